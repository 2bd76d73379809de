"""asd_sample on rows whose tails hold little mass in many tokens, and on vocabularies beyond 2^18: every token is
the definition's, to 2^-40 of the row's mass at an edge, by sums in 80-bit floating point."""
import numpy as np
import pytest
import torch

import paper_2608_03447_amd as asd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EDGE = 2.0 ** -40


def kept_weights(z, t=1.0, k=0, p=1.0, m=0.0):
    """The kept weights of a row (80-bit): one array, or several where the top-p cut is so near an edge that one
    token more or less may be kept."""
    z = z.astype(np.longdouble)
    w = np.exp((z - z.max()) / np.longdouble(t))
    order = np.argsort(-z, kind="stable")
    ranked = w[order]
    n = z.size if k <= 0 else min(int(k), z.size)
    counts = [n]
    if p < 1:
        run = np.cumsum(ranked[:n])
        goal = np.longdouble(p) * run[-1]
        near = EDGE * run[-1]
        first = max(1, int(np.searchsorted(run, goal - near, side="left")) + 1)
        last = max(1, int(np.searchsorted(run, goal + near, side="left")) + 1)
        counts = range(first, min(last, n) + 1)
        assert len(counts) <= 8, "the cut's tokens are too small to test"
    out = []
    for n in counts:
        if m > 0:
            n = min(n, int(np.sum(ranked >= np.longdouble(np.float32(m)))))
        kept = np.zeros_like(w)
        kept[order[:n]] = ranked[:n]
        out.append(kept)
    return out


def fits(kept, run, token, prob, u):
    """Whether the token may be drawn with u, and the probability is its own."""
    if not kept[token] > 0:
        return False
    low, high = float((run[token] - kept[token]) / run[-1]), float(run[token] / run[-1])
    share = float(kept[token] / run[-1])
    # one rounding to binary32, the weight's 2^-44 and the sum's 2^-40
    near = abs(prob - share) <= share * (2.0 ** -24 * 1.01 + 2.0 ** -38)
    return near and low - EDGE <= u < high + EDGE


def check(z, uniform, t=1.0, k=0, p=1.0, m=0.0):
    """One row of logits, drawn from with every u of `uniform`."""
    rows = len(uniform)
    u = torch.tensor(uniform, dtype=torch.float32)
    prob = torch.empty(rows, device=DEV)
    logits = z.to(DEV).expand(rows, -1).contiguous()
    token = asd.asd_sample(logits, u.to(DEV), temperature=t, top_k=k, top_p=p, min_p=m, out_prob=prob)
    torch.cuda.synchronize()
    sets = [(x, np.cumsum(x)) for x in
            kept_weights(z.float().numpy(), float(np.float32(t)), k, float(np.float32(p)), m)]
    for r, (at, x, share) in enumerate(zip(token.tolist(), u.tolist(), prob.tolist())):
        assert any(fits(*s, at, share, x) for s in sets), "u %g gives token %d of %g" % (x, at, share)


def draws(top, n, seed):
    """u over [0, top), evenly in all, and at both ends of [0, 1)."""
    rng = np.random.default_rng(seed)
    return [0.0, 2.0 ** -149, 1 - 2.0 ** -24] + list(rng.random(n) * top)


@pytest.mark.parametrize("vocab", [20000, 100000, 151936, 262145, 600001])
def test_equal_tails_that_a_nucleus_cuts(vocab):
    z = torch.full((1, vocab), -20.79)
    z[0, -1] = 0.0
    tail = vocab * 2.0 ** -30
    check(z[0], draws(tail, 30, vocab), p=1 - 2.0 ** -24)
    check(z[0], draws(tail, 30, vocab + 1), k=vocab - 1)
    check(z[0], draws(tail, 12, vocab + 2), k=vocab - 1, p=1 - 2.0 ** -24)


@pytest.mark.parametrize("vocab,low", [(20000, -31.01), (151936, -31.01), (300000, -30.8), (1 << 22, -28.2), (1 << 24, -26.8)])
def test_tails_of_weights_below_a_billionth(vocab, low):
    """Each weight is some 2^-39 to 2^-45, all of them 2^-30 to 2^-14 of the mass."""
    z = torch.full((vocab,), low)
    z[-1] = 0.0
    tail = vocab * np.exp(low)
    check(z, draws(1.5 * tail, 8, vocab), k=vocab - 1)
    check(z, draws(1.5 * tail, 4, vocab))
    check(z, draws(1.5 * tail, 4, vocab), m=1e-20)


@pytest.mark.parametrize("vocab", [20000, 80000, 300000])
def test_tails_of_many_values(vocab):
    """Weights of 4 to 12 units of 2^-44 and 0.45 more, none like another, around the cut."""
    rng = np.random.default_rng(vocab)
    units = rng.integers(4, 13, vocab) + 0.45 + 0.02 * (rng.random(vocab) - 0.5)
    z = torch.from_numpy((np.log(units) - 44 * np.log(2.0)).astype(np.float32))
    scale = 2.0 ** -22 / (vocab * 8.45 * 2.0 ** -44)               # a tail of 2^-22 of the mass
    z += float(np.log(scale))
    z[vocab // 3] = 0.0
    for p in (1 - 2.0 ** -24, 1 - 2.0 ** -23):
        check(z, draws(2.0 ** -22, 12, vocab), p=p)
        check(z, draws(2.0 ** -22, 12, vocab), p=p, m=1e-30)
    check(z, draws(2.0 ** -22, 12, vocab), m=float(torch.exp(z.median())))


@pytest.mark.parametrize("vocab", [20000, 80000])
def test_the_first_token_of_no_mass_to_speak_of(vocab):
    z = torch.full((vocab,), -34.0)                                # exp(-34) = 1.7e-15
    z[0], z[-1] = -40.0, 0.0                                       # 4.2e-18
    for m in (1e-20, 3e-17):
        check(z, [0.0], m=m)
    check(z, [0.0])
    check(z, [0.0], k=vocab - 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [262145, 600001, 1500007])
def test_vocabularies_beyond_the_shared_rows(vocab, dtype):
    gen = torch.Generator().manual_seed(vocab)
    z = 2.5 * torch.randn(vocab, generator=gen)
    z[torch.randint(vocab, (8,), generator=gen)] += 10.0
    z = z.to(dtype)
    u = [0.0, 0.3, 0.77, 1 - 2.0 ** -24]
    check(z, u)
    check(z, u, t=0.7, k=50)
    check(z, u, k=100000)
    check(z, u, p=0.95)
    check(z, u, k=30000, p=0.9, m=1e-4)
    check(z, u, m=1e-3)


def test_shared_rows_with_both_cuts():
    """Top-p and min-p of one row, either of them the stricter."""
    gen = torch.Generator().manual_seed(3)
    z = 1.5 * torch.randn(120000, generator=gen)
    u = draws(1.0, 10, 4)
    for p in (0.9, 0.99, 0.999999):
        for m in (1e-1, 1e-2, 1e-3, 1e-5, 1e-8):
            check(z, u, p=p, m=m)


@pytest.mark.parametrize("vocab,rows,calls", [(60001, 7, 60), (100000, 420, 1), (300000, 100, 1)])
def test_cuts_between_any_two_tokens_above_a_far_tail(vocab, rows, calls):
    """Top-p as near as binary32 has it to where the cut passes from one token to the next, over a tail of tokens that
    are 0.45 units of 2^-44 each: of all rows, some cuts lie within the tail's mass of the next token's."""
    rng = np.random.default_rng(vocab)
    few = 3000
    z = np.full(vocab, np.log(0.45) - 44 * np.log(2.0), dtype=np.float32)
    at = rng.permutation(vocab)[:few + 1]
    z[at[0]] = 0.0
    z[at[1:]] = (np.log(1.0 / few) + rng.uniform(-0.5, 0.5, few)).astype(np.float32)
    w = np.exp(z.astype(np.longdouble))
    order = np.argsort(-z, kind="stable")
    run = np.cumsum(w[order])
    rank = np.empty(vocab, dtype=np.int64)
    rank[order] = np.arange(vocab)
    places = np.sort(at)                                            # the tokens that can be kept, by index
    logits = torch.from_numpy(z).to(DEV).expand(rows, vocab).contiguous()
    picked = iter(rng.permutation(np.arange(20, few - 20))[:rows * calls])
    cut_short = 0
    for _ in range(calls):
        p = np.array([np.float32(run[next(picked)] / run[-1]) for _ in range(rows)])
        u = rng.random(rows).astype(np.float32)
        prob = torch.empty(rows, device=DEV)
        token = asd.asd_sample(logits, torch.from_numpy(u).to(DEV), top_p=torch.from_numpy(p).to(DEV), out_prob=prob)
        torch.cuda.synchronize()
        for r in range(rows):
            goal = np.longdouble(p[r]) * run[-1]
            counts = {int(np.searchsorted(run, goal + d * EDGE * run[-1], side="left")) + 1 for d in (-1, 1)}
            cut_short += int(np.searchsorted(run, goal - np.longdouble(p[r]) * w[w < 1e-9].sum(), side="left")) + 1 not in counts
            kept = [np.where(rank[places] < n, w[places], 0) for n in counts]
            where = int(np.searchsorted(places, int(token[r])))
            assert places[where] == int(token[r])
            assert any(fits(k, np.cumsum(k), where, float(prob[r]), float(u[r])) for k in kept), (r, float(p[r]))
    assert cut_short >= 1, "no cut lies within the tail's mass of the next token's"


def test_equal_logits_of_a_very_wide_row():
    """Every running sum is a whole number, so that each token is known."""
    vocab = (1 << 26) + 3
    z = torch.zeros((2, vocab), dtype=torch.float16, device=DEV)
    for kept, args in ((vocab, {}), ((vocab + 1) // 2, dict(top_p=0.5)), (12345677, dict(top_k=12345677)),
                       (6172839, dict(top_k=12345677, top_p=0.5)), (vocab, dict(min_p=1.0))):
        for u in ([0.0, 0.5], [0.625, 1 - 2.0 ** -24]):
            token = asd.asd_sample(z, torch.tensor(u, device=DEV), **args)
            assert token.tolist() == [int(np.floor(np.longdouble(x) * kept)) for x in u]
