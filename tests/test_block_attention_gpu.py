"""asd_block_attention against its 64-bit form, within the bound of its roundings."""
import math

import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch, check_attention

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def queries(b, scale=2.0):
    return b.randn(b.rows, b.hq, b.d, scale=scale)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (7, 1), (20, 4), (16, 16)])
def test_single_tokens(hq, hkv, d, dtype):
    b = Batch([0] * 7, [0, 1, 15, 31, 32, 127, 300], hq, hkv, d, dtype, 16, seed=d + hq)
    check_attention(b, queries(b))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens", [[1, 8, 16], [63, 2, 31], [40], [100, 0]])
def test_chains_and_trees(lens, d, dtype):
    cached = [0, 130, 77, 5][:len(lens)]
    b = Batch(lens, cached, 8, 2, d, dtype, 16, seed=sum(lens))
    q = queries(b)
    check_attention(b, q)
    check_attention(b, q, mask=b.trees(2))


@pytest.mark.parametrize("layout,page", [("nhd", 1), ("nhd", 7), ("hnd", 24), ("both", 16),
                                         ("nhd", 512), ("hnd", 3)])
def test_pages_of_any_size_and_order(layout, page):
    b = Batch([5, 0, 20], [200, 513, 31], 6, 3, 64, BF16, page, seed=page, layout=layout)
    check_attention(b, queries(b))


@pytest.mark.parametrize("cached", [1000, 5000, 20011])
def test_long_caches_of_few_rows(cached):
    b = Batch([0, 8], [cached, 3], 4, 1, 128, BF16, 16, seed=cached)
    check_attention(b, queries(b))


def test_many_requests():
    lens = [j % 4 for j in range(700)]
    b = Batch(lens, [(j * 37) % 90 for j in range(700)], 4, 2, 64, BF16, 16)
    check_attention(b, queries(b))


def test_large_groups():
    b = Batch([12, 3], [40, 100], 48, 1, 64, F16, 16)
    check_attention(b, queries(b))


def test_rows_that_see_nothing_give_zeros():
    b = Batch([3, 2], [0, 0], 4, 2, 64, BF16, 16)
    mask = torch.zeros((b.rows, 1), dtype=torch.int64, device=DEV)
    out = check_attention(b, queries(b), mask=mask)
    assert (out == 0).all()
    mask[2] = 2
    check_attention(b, queries(b), mask=mask)
    mask.fill_(-1)
    check_attention(b, queries(b), mask=mask)


def test_blocks_longer_than_the_mask():
    b = Batch([90], [10], 4, 2, 64, BF16, 16)
    check_attention(b, queries(b), mask=b.trees(1))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan, 6e4])
@pytest.mark.parametrize("d", [64, 128])
def test_hidden_tokens_hold_anything(bad, d):
    """Nothing of a hidden token reaches a row: in the tree, after the block, in other pages."""
    b = Batch([6, 30, 0], [40, 7, 20], 8, 2, d, F16, 16, seed=9)
    q = queries(b)
    mask = b.trees(1)
    mask[0] = 1
    for i, (k, c) in enumerate(zip(b.lens, b.cached)):
        used = c + k + 1
        for t in range(used, b.page_table.shape[1] * 16):      # behind the block
            if t // 16 < (used + 15) // 16:
                page = b.page_table[i, t // 16].long()
                b.k_cache[page, t % 16] = bad
                b.v_cache[page, t % 16] = bad
    free = set(range(b.pages)) - set(b.page_table.flatten().tolist())
    for page in free:
        b.k_cache[page] = bad
        b.v_cache[page] = bad
    check_attention(b, q, mask=mask)
    # tokens of the block itself, hidden from every row but some
    for j in (2, 5):
        page = b.page_table[0, (40 + j) // 16].long()
        b.k_cache[page, (40 + j) % 16] = bad
        b.v_cache[page, (40 + j) % 16] = bad
    first = mask[:7, 0]
    mask[:7, 0] = first & ~(1 << 2) & ~(1 << 5)
    check_attention(b, q, mask=mask)
    chain = Batch([6], [40], 8, 2, d, F16, 16, seed=9)
    page = chain.page_table[0, 46 // 16].long()
    chain.v_cache[page, 46 % 16] = bad
    chain.k_cache[page, 46 % 16] = bad
    qq = queries(chain)
    out = asd.asd_block_attention(qq, chain.k_cache, chain.v_cache, chain.page_table,
                                  chain.cache_lens, chain.block_lens)
    assert torch.isfinite(out[:6]).all()
    chain.v_cache[page, 46 % 16] = 0
    chain.k_cache[page, 46 % 16] = 0
    same = asd.asd_block_attention(qq, chain.k_cache, chain.v_cache, chain.page_table,
                                   chain.cache_lens, chain.block_lens)
    assert torch.equal(out[:6], same[:6])


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_visible_infinity_reaches_the_rows_that_see_it(d):
    b = Batch([3], [50], 4, 2, d, BF16, 16)
    q = queries(b)
    page = b.page_table[0, 51 // 16].long()
    b.v_cache[page, 51 % 16, 0, 5] = math.inf
    out = asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens)
    out = out.float().cpu()
    assert torch.isfinite(out[0]).all()                       # row 0 does not see row 1
    assert (out[1:, :2, 5] == math.inf).all()
    out[1:, :2, 5] = 0
    assert torch.isfinite(out).all()
    b.v_cache[page, 51 % 16, 0, 5] = 0
    b.k_cache[page, 51 % 16, 1] = math.nan
    out = asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens)
    out = out.float().cpu()
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[:, :2]).all()
    assert out[1:, 2:].isnan().all()


def test_scores_far_apart_and_growing():
    """The maximum moves with nearly every token, by more than a weight can hold."""
    for order in (1, -1):
        b = Batch([2], [400], 4, 1, 64, F16, 16)
        q = torch.zeros((b.rows, 4, 64), dtype=F16, device=DEV)
        q[..., 0] = 30.0
        for t in range(403):
            page = b.page_table[0, t // 16].long()
            b.k_cache[page, t % 16, 0, 0] = 0.25 * order * t
        check_attention(b, q, scale=1.0)
        check_attention(b, q, scale=-0.5)
        check_attention(b, q, scale=0.0)


def test_offsets_and_strided_queries():
    b = Batch([2, 0, 3], [9, 4, 0], 4, 2, 64, BF16, 8, offsets=[10, 2, 5], total_rows=20)
    check_attention(b, queries(b))
    wide = b.randn(b.rows, 10, 64)
    check_attention(b, wide[:, 3:7])


def test_requests_that_do_not_fit_are_skipped():
    asd.asd_device_error(clear=True)
    b = Batch([2, 2, -4, 2], [5, -1, 9, 14], 4, 2, 64, BF16, 4, width=4)
    check_attention(b, queries(b))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_NEGATIVE_K | asd.ASD_DEVERR_CACHE
    b = Batch([2, 2, 2], [5, 1, 1], 4, 2, 64, BF16, 4, offsets=[0, 4, -1], total_rows=6)
    check_attention(b, queries(b))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_ROWS
    b = Batch([2, 2, 0], [30, 200, 3], 4, 2, 64, BF16, 4)
    b.page_table[0, 3], b.page_table[1, 20], b.page_table[2, 0] = -1, b.pages, -7
    check_attention(b, queries(b))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_CACHE


def test_workspaces_may_hold_anything():
    """Stretches without work, and items that no stretch cuts, say so themselves."""
    for lens, cached in (([0], [5]), ([8, 0, 16], [900, 3000, 100]), ([0] * 40, [700] * 40)):
        b = Batch(lens, cached, 8, 2, 128, BF16, 16)
        q = queries(b)
        size = asd.asd_block_attention_workspace_bytes(8, 2, 128, b.n, b.rows)
        check_attention(b, q, workspace=torch.full((size,), 0x5a, dtype=torch.uint8, device=DEV))


def test_a_cache_past_32_bits():
    """Pages 2^31 elements and more into the cache, through strides that leave holes."""
    stride = 1 << 23
    pages = 300
    base = torch.empty(stride * pages, dtype=BF16, device=DEV)
    b = Batch([2], [4700], 2, 1, 64, BF16, 16)
    k = base.as_strided((pages, 16, 1, 64), (stride, 64, 64, 1))
    v = base[16 * 64:].as_strided((pages, 16, 1, 64), (stride, 64, 64, 1))
    k.copy_(b.k_cache[:pages] if b.pages >= pages else b.k_cache.repeat(2, 1, 1, 1)[:pages])
    v.copy_(b.v_cache[:pages] if b.pages >= pages else b.v_cache.repeat(2, 1, 1, 1)[:pages])
    b.page_table.remainder_(pages)
    b.k_cache, b.v_cache, b.pages = k, v, pages
    check_attention(b, queries(b))


def test_streams_graphs_and_workspaces():
    b = Batch([8, 0, 16], [900, 3000, 100], 8, 2, 128, BF16, 16)
    q = queries(b)
    call = (b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens)
    want = asd.asd_block_attention(q, *call)
    size = max(1, asd.asd_block_attention_workspace_bytes(8, 2, 128, 3, b.rows))
    space = torch.empty(size, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    with torch.cuda.stream(side):
        assert torch.equal(asd.asd_block_attention(q, *call), want)
        assert torch.equal(asd.asd_block_attention(q, *call, workspace=space), want)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            asd.asd_block_attention(q, *call, out=out, workspace=space)
    torch.cuda.synchronize()
    for turn in range(4):
        q.copy_(queries(b))
        b.cache_lens.copy_(torch.tensor([900 - 300 * turn, 3000 - 999 * turn, turn]))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(asd.asd_block_attention(q, *call), replayed)


def test_an_empty_batch_is_a_no_op():
    b = Batch([0], [4], 4, 2, 64, BF16, 8)
    out = torch.full((0, 4, 64), 7.0, dtype=BF16, device=DEV)
    got = asd.asd_block_attention(queries(b)[:0], b.k_cache, b.v_cache, b.page_table[:0],
                                  b.cache_lens[:0], b.block_lens[:0], out=out)
    assert got.shape == (0, 4, 64)


def test_repeated_calls_and_two_streams_give_the_same():
    b = Batch([8, 0, 40], [30000, 5000, 77], 16, 4, 128, BF16, 16, seed=31)
    c = Batch([0] * 20, list(range(100, 8100, 400)), 16, 4, 128, BF16, 64, seed=32)
    calls = []
    for x in (b, c):
        q = queries(x)
        calls.append(lambda x=x, q=q: asd.asd_block_attention(q, x.k_cache, x.v_cache, x.page_table,
                                                              x.cache_lens, x.block_lens))
    want = [call() for call in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(calls[i]())
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])
