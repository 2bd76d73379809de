"""asd_sample against its 64-bit form: tokens equal, probabilities to a rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2608_03447_amd as asd
from oracle import decode

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def check(logits, u, t=None, k=None, p=None, m=None, **kw):
    rows = logits.shape[0]
    prob = torch.full((rows,), 7.0, device=DEV)

    def dev(x, dtype):
        return None if x is None else torch.tensor(x, dtype=dtype).expand(rows).contiguous().to(DEV)

    u = torch.as_tensor(u, dtype=torch.float32).to(DEV).expand(rows).contiguous()
    args = [dev(t, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32)]
    token = asd.asd_sample(logits, u, temperature=args[0], top_k=args[1], top_p=args[2],
                           min_p=args[3], out_prob=prob, **kw)
    torch.cuda.synchronize()
    z = logits.float().cpu().numpy()
    a = [[d] * rows if x is None else x.cpu().double().tolist() for x, d in zip(args, (1.0, 0, 1.0, 0.0))]
    uu = u.cpu().double().tolist()
    want = [decode.sample_row(z[r], uu[r], *(x[r] for x in a)) for r in range(rows)]
    assert token.cpu().tolist() == [w[0] for w in want]
    exact = np.array([w[1] for w in want])
    # one rounding to binary32, the weights' 2^-44
    assert (np.abs(prob.cpu().double().numpy() - exact) <= exact * 2.0 ** -23 + 2.0 ** -40).all()
    return token


def rows_of(rows, vocab, dtype, seed, sigma=2.0, pad=0):
    gen = torch.Generator().manual_seed(seed)
    z = sigma * torch.randn((rows, vocab + pad), generator=gen)
    likely = torch.randint(vocab, (rows, 8), generator=gen)
    z.scatter_add_(1, likely, 10 * torch.rand((rows, 1), generator=gen).expand(rows, 8))
    return z.to(dtype).to(DEV)[:, :vocab], torch.rand(rows, generator=gen)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 1), (63, 0), (64, 3), (257, 0), (1000, 24),
                                       (4097, 1), (32000, 0), (50257, 7), (151936, 0)])
def test_every_filter_over_the_sizes(dtype, vocab, pad):
    rows = 12
    z, u = rows_of(rows, vocab, dtype, vocab + pad, pad=pad)
    check(z, u)
    check(z, u, t=0.7)
    check(z, u, k=[0, 1, 2, 3, 5, 20, 50, 100, 1000, 5000, 1 << 30, -1])
    check(z, u, p=[1.0, 0.99, 0.95, 0.9, 0.8, 0.7, 0.5, 0.3, 0.1, 0.0, -1.0, 2.0])
    check(z, u, m=[0.0, 1.0, 0.9, 0.5, 0.3, 0.1, 0.05, 0.02, 0.01, 1e-4, 1e-9, 2.0])
    check(z, u, t=[0.8, 1.2, 0.3, 1.0] * 3, k=[50, 0, 7, 300] * 3, p=[0.95, 0.9, 1.0, 0.6] * 3,
          m=[0.0, 0.05, 0.01, 0.0] * 3)


@pytest.mark.parametrize("dtype", TYPES)
def test_flat_rows_keep_many_tokens(dtype):
    """The nucleus of a flat row is most of the vocabulary, with long ties in 16 bits."""
    gen = torch.Generator().manual_seed(5)
    z = (0.5 * torch.randn((16, 60001), generator=gen)).to(dtype).to(DEV)
    u = torch.linspace(0, 0.999, 16)
    check(z, u)
    check(z, u, p=[0.9, 0.5, 0.99, 0.05] * 4)
    check(z, u, k=[30000, 10, 60000, 9999] * 4, p=[0.9, 0.5, 0.99, 0.05] * 4)
    check(z, u, m=[0.5, 0.01, 0.9, 0.2] * 4, t=[1.0, 2.0, 0.1, 100.0] * 4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [8, 1024, 40960])
def test_ties_go_to_the_lowest_index_and_edges_are_exact(dtype, vocab):
    """Equal logits: every running sum is a whole number, so u and p on an edge are exact."""
    z = torch.zeros((8, vocab), dtype=dtype, device=DEV)
    u = torch.arange(8) / 8.0
    assert check(z, u).tolist() == [vocab * j // 8 for j in range(8)]
    assert check(z, u, p=0.5).tolist() == [vocab * j // 16 for j in range(8)]
    assert check(z, u, k=8).tolist() == list(range(8))
    assert check(z, u, k=8, p=0.25).tolist() == [j // 4 for j in range(8)]
    z[:, 1::2] = -3.0
    assert check(z, u, m=0.5).tolist() == [2 * (vocab // 2 * j // 8) for j in range(8)]


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_unusual_values(dtype):
    lowest, big = torch.finfo(dtype).min, torch.finfo(dtype).max
    inf, nan = math.inf, math.nan
    rows = [[nan, 0, 0, 0], [0, 1, 2, nan], [-inf] * 4, [inf, 0, inf, -inf], [inf, nan, 0, 0],
            [lowest] * 4, [lowest, 0, lowest, lowest], [big, lowest, 0, big], [-inf, -inf, lowest, -inf],
            [-0.0, 0.0, -0.0, 0.0], [-inf, 5, -inf, 5], [-nan, 0, 0, 0]]
    z = torch.tensor(rows, dtype=torch.float64).to(dtype).to(DEV)
    asd.asd_device_error(clear=True)
    for u in (0.0, 0.4, 0.6, 0.999999):
        for t in (None, 0.0, 1e-30, 1e30, inf, nan, -1.0, 1e-45):
            check(z, u, t=t)
        check(z, u, k=2)
        check(z, u, p=0.6)
        check(z, u, m=0.5)
        check(z, u, k=3, p=0.9, m=0.1)
        check(z, u, p=nan, m=nan)
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_SAMPLE
    check(z[9:11], 0.5)
    assert asd.asd_device_error(clear=True) == 0


def test_u_outside_its_range():
    z, _ = rows_of(6, 1000, torch.float32, 3)
    check(z, torch.tensor([-1.0, 0.0, 1.0, 2.0, math.inf, math.nan]), t=0.9)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_at_any_address_and_apart(dtype):
    base = torch.zeros(64 + 7 * 1303, dtype=dtype, device=DEV)
    for start in (0, 1, 2, 3, 5, 7):
        for stride in (1300, 1301, 1303):
            z, u = rows_of(5, 1300, dtype, start + stride)
            view = base[start:start + 5 * stride].as_strided((5, 1300), (stride, 1))
            view.copy_(z)
            check(view, u, t=0.9, k=40, p=0.9)
            check(view, u, p=0.95)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_draws_the_same_in_any_batch(dtype):
    z, u = rows_of(300, 20011, dtype, 11, sigma=1.0)
    u = u.to(DEV)
    p = torch.rand(300).to(DEV)
    whole = asd.asd_sample(z, u, top_p=p, temperature=1.1)
    for a, b in ((0, 1), (17, 20), (100, 300)):
        part = asd.asd_sample(z[a:b], u[a:b], top_p=p[a:b].contiguous(), temperature=1.1)
        assert torch.equal(part, whole[a:b])


def test_draws_follow_the_distribution():
    z = torch.tensor([0.0, 1.0, 2.0, 3.0, -1.0], device=DEV).expand(20000, 5).contiguous()
    u = (torch.arange(20000, device=DEV) + 0.5) / 20000
    token = asd.asd_sample(z, u, temperature=0.9)
    share = torch.bincount(token.long(), minlength=5).double() / 20000
    # evenly spaced u: each token's share to the one draw at either edge
    assert ((share - torch.softmax(z[0].double() / 0.9, 0)).abs() <= 1.0 / 20000).all()


def test_other_streams_graphs_and_workspaces():
    z, u = rows_of(40, 50001, torch.bfloat16, 2)
    u = u.to(DEV)
    want = asd.asd_sample(z, u, top_p=0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    size = max(1, asd.asd_sample_workspace_bytes(torch.bfloat16, 50001, 40))
    space = torch.empty(size, dtype=torch.uint8, device=DEV)
    with torch.cuda.stream(side):
        assert torch.equal(asd.asd_sample(z, u, top_p=0.9), want)
        p = torch.full((40,), 0.9, device=DEV)
        out = torch.zeros(40, dtype=torch.int32, device=DEV)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            asd.asd_sample(z, u, top_p=p, out_token=out, workspace=space)
    torch.cuda.synchronize()
    for turn in range(4):
        zz, uu = rows_of(40, 50001, torch.bfloat16, 100 + turn)
        z.copy_(zz)
        u.copy_(uu)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(asd.asd_sample(z, u, top_p=p), replayed)


def test_empty_and_scalar_arguments():
    z, u = rows_of(4, 100, torch.float32, 1)
    u = u.to(DEV)
    assert asd.asd_sample(z[:0], u[:0]).shape == (0,)
    a = asd.asd_sample(z, u, temperature=0.5, top_k=10, top_p=0.9, min_p=0.01)
    full = [torch.full((4,), x, dtype=d, device=DEV) for x, d in
            ((0.5, torch.float32), (10, torch.int32), (0.9, torch.float32), (0.01, torch.float32))]
    b = asd.asd_sample(z, u, temperature=full[0], top_k=full[1], top_p=full[2], min_p=full[3])
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,pad", [(65537, 0), (70001, 3), (129280, 0), (262130, 0), (262144, 0)])
def test_flat_rows_of_wide_vocabularies(dtype, vocab, pad):
    """Rows that many workgroups read in parts, and the widths beside which one does."""
    z, u = rows_of(6, vocab, dtype, vocab, sigma=1.5, pad=pad)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    check(z, u, p=[0.5, 0.9, 0.95, 0.99, 0.999999, 0.3])
    check(z, u, m=[1e-2, 1e-3, 1e-4, 1e-6, 2e-3, 1e-9])
    check(z, u, t=[0.9, 1.0, 1.3, 2.0, 8.0, 1e3], p=0.9, m=[0.0, 1e-3, 1e-4, 0.0, 0.05, 0.5])


@pytest.mark.parametrize("dtype", TYPES)
def test_wide_rows_of_few_values_and_in_order(dtype):
    vocab = 80000
    gen = torch.Generator().manual_seed(11)
    z = torch.zeros(9, vocab)
    z[1, ::3] = -1.0                                              # two values
    z[2] = torch.randint(0, 9, (vocab,), generator=gen).float()   # nine: more ties than a list holds
    z[3] = torch.linspace(-6, 6, vocab)                           # in order
    z[4] = torch.linspace(6, -6, vocab)
    z[5] = torch.randn(vocab, generator=gen)
    z[5, 1000:70000] = -math.inf                                  # sub-blocks of nothing
    z[6] = torch.randn(vocab, generator=gen)
    z[6, 777] = math.inf
    z[7] = torch.randn(vocab, generator=gen) * 1e4                # nearly greedy
    z[8, :64] = 1.0                                               # one sub-block stands out
    z = z.to(dtype).to(DEV)
    u = torch.rand(9, generator=gen)
    for p in (0.2, 0.7, 0.95, 0.9999):
        check(z, u, p=p)
        check(z, u, p=p, m=0.01)
    for m in (0.5, 0.01, 1e-5):
        check(z, u, m=m)


def test_wide_flat_rows_in_a_graph():
    z, u = rows_of(40, 100003, torch.bfloat16, 5)
    uniform = u.to(DEV)
    p = torch.full((40,), 0.95, device=DEV)
    want = [asd.asd_sample(z, uniform, top_p=p).tolist()]
    out = torch.empty(40, dtype=torch.int32, device=DEV)
    space = torch.empty(asd.asd_sample_workspace_bytes(z.dtype, 100003, 40), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asd.asd_sample(z, uniform, top_p=p, out_token=out, workspace=space)
    uniform.copy_(uniform.flip(0))
    want.append(asd.asd_sample(z, uniform, top_p=p).tolist())
    for turn in (1, 0, 1, 0):
        uniform.copy_((u if turn == 0 else u.flip(0)).to(DEV))
        space.fill_(0xa5)
        graph.replay()
        assert out.tolist() == want[turn]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [300, 2048, 2049, 3001, 20000, 65000, 100000])
def test_counts_next_to_the_width(dtype, vocab):
    """Top-k of few and of most tokens, where neighbouring logits tie or one stands far out."""
    z, u = rows_of(7, vocab, dtype, vocab + 1)
    z[1] = z[1].float().round().to(dtype)
    z[2] = 0.5
    z[3, 5] = 3e4
    z[4, vocab // 2:] = -math.inf
    z[5] += 1000
    k = [vocab - 1, 1000, 1500, 600, 1900, 1921, vocab // 3]
    for p in (1.0, 0.9, 0.3):
        check(z, u, k=k, p=p)
        check(z, u, k=k[::-1], p=p, m=1e-3, t=1.5)


def test_more_rows_than_a_launch_takes():
    """Each row's token is that of the same row in a small batch."""
    base, vocab, rows = 1000, 40, (1 << 20) + 1234        # rows of 40 binary16 logits keep their alignment
    z, u = rows_of(base, vocab, torch.float16, 17)
    gen = torch.Generator().manual_seed(18)
    u = u.to(DEV)
    p = torch.rand(base, generator=gen).to(DEV)
    k = torch.randint(0, 30, (base,), generator=gen).to(torch.int32).to(DEV)
    want = asd.asd_sample(z, u, top_k=k, top_p=p)
    many = torch.arange(rows, device=DEV) % base
    prob = torch.zeros(rows, device=DEV)
    got = asd.asd_sample(z[many], u[many], top_k=k[many], top_p=p[many], out_prob=prob)
    assert torch.equal(got, want[many])
    assert bool((prob > 0).all())


def test_repeated_calls_give_the_same():
    z, u = rows_of(300, 90001, torch.bfloat16, 23)
    p = torch.full((300,), 0.97, device=DEV)
    probs = [torch.empty(300, device=DEV) for _ in range(4)]
    tokens = [asd.asd_sample(z, u.to(DEV), top_p=p, out_prob=x).tolist() for x in probs]
    assert all(t == tokens[0] for t in tokens) and all(torch.equal(x, probs[0]) for x in probs)


@pytest.mark.parametrize("vocab", [500, 5000, 70000])
def test_temperatures_at_the_ends(vocab):
    z, u = rows_of(8, vocab, torch.float32, vocab)
    t = [1e-38, 1e-30, 1e-6, 1e-3, 1e6, 1e30, 3e38, math.inf]
    check(z, u, t=t)
    check(z, u, t=t, p=0.6)
    check(z, u, t=t, k=30, p=0.6, m=0.2)
    check(z, u, t=t, k=vocab // 2, p=0.6)


def test_two_streams_at_once():
    """Each stream has a library workspace of its own."""
    z = [rows_of(64, 100000, torch.bfloat16, s) for s in (1, 2)]
    args = [(x[0], x[1].to(DEV)) for x in z]
    p = torch.full((64,), 0.95, device=DEV)
    want = [asd.asd_sample(*a, top_p=p).tolist() for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(asd.asd_sample(*args[i], top_p=p))
    torch.cuda.synchronize()
    assert all(t.tolist() == want[i] for i in range(2) for t in got[i])
