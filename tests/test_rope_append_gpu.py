"""asd_rope_append against its 64-bit form, within the bound of its roundings."""
import math

import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch, check_append

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def freq(rot, theta=1e4):
    return (theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV)


def qkv(b, apart=True):
    """Three parts of one projection's rows, or three dense tensors."""
    if apart:
        x = b.randn(b.rows, (b.hq + 2 * b.hkv) * b.d, scale=1.5)
        q, k, v = x.split([b.hq * b.d, b.hkv * b.d, b.hkv * b.d], 1)
        return [t.unflatten(1, (-1, b.d)) for t in (q, k, v)]
    return [b.randn(b.rows, h, b.d, scale=1.5) for h in (b.hq, b.hkv, b.hkv)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (64, 64), (128, 24), (256, 64), (80, 80),
                                   (8, 6), (96, 2), (104, 0), (256, 256), (128, 96), (200, 120)])
def test_head_sizes_and_parts_of_them(d, rot, interleaved, dtype):
    b = Batch([3, 0, 5], [17, 0, 100], 6, 2, d, dtype, 16, seed=d + rot)
    weight = [(1 + 0.3 * b.randn(d).float()).to(dtype) for _ in range(2)]
    for norm in (weight, (None, None), (weight[0], None), (None, weight[1])):
        q, k, v = qkv(b)
        check_append(b, q, k, v, inv_freq=freq(rot) if rot else None, q_norm=norm[0], k_norm=norm[1],
                     interleaved=interleaved)


@pytest.mark.parametrize("layout,page", [("nhd", 1), ("nhd", 7), ("hnd", 16), ("hnd", 5),
                                         ("both", 16), ("nhd", 300)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (12, 4), (5, 5), (32, 8)])
def test_cache_layouts_and_head_counts(layout, page, hq, hkv):
    b = Batch([0, 8, 1, 40], [0, 1, 63, 200], hq, hkv, 64, BF16, page, seed=page, layout=layout)
    q, k, v = qkv(b, apart=False)
    check_append(b, q, k, v, inv_freq=freq(64))


def test_positions_of_a_tree_and_far_ones():
    b = Batch([6, 2], [10, 20], 4, 2, 128, BF16, 16)
    q, k, v = qkv(b)
    for positions in ([10, 11, 11, 12, 12, 12, 13, 20, 21, 21],
                      [2 ** 31 + j for j in range(10)], [10 ** 6 - 17 * j for j in range(10)],
                      [-5 * j for j in range(10)]):
        check_append(b, q, k, v, inv_freq=freq(128, 1e6),
                     positions=torch.tensor(positions, dtype=torch.int64, device=DEV))


def test_long_blocks_and_many_requests():
    b = Batch([700, 0, 33], [5, 900, 0], 8, 2, 64, F16, 24, seed=3)
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))
    lens = [j % 3 for j in range(1500)]
    b = Batch(lens, [j % 11 for j in range(1500)], 2, 1, 64, BF16, 16, seed=4)
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))


@pytest.mark.parametrize("d", [16, 24])
def test_more_requests_than_workgroups(d):
    n, size = 70000, 4
    k = torch.randn(n, 1, d, device=DEV).to(BF16)
    v = torch.randn(n, 1, d, device=DEV).to(BF16)
    pages = torch.randperm(n, device=DEV)
    lens = torch.arange(n, device=DEV) % size
    k_cache, v_cache = (torch.zeros(n, size, 1, d, dtype=BF16, device=DEV) for _ in range(2))
    asd.asd_rope_append(None, k, v, k_cache, v_cache, pages.to(torch.int32)[:, None], lens,
                        torch.zeros(n, dtype=torch.int32, device=DEV), None)
    for cache, rows in ((k_cache, k), (v_cache, v)):
        want = torch.zeros_like(cache)
        want[pages, lens] = rows
        assert torch.equal(cache, want)


def test_offsets_leave_other_rows_as_they_were():
    b = Batch([2, 0, 3], [9, 4, 0], 4, 2, 64, BF16, 8, offsets=[10, 2, 5], total_rows=20)
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))


def test_in_place_and_without_queries():
    b = Batch([4, 4], [30, 3], 8, 2, 128, BF16, 16)
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(128), out_q=q)
    check_append(b, None, k, v, inv_freq=freq(128))


def test_requests_that_do_not_fit_are_skipped():
    asd.asd_device_error(clear=True)
    b = Batch([2, 2, -4, 2], [5, -1, 9, 14], 4, 2, 64, BF16, 4, width=4)    # room for 16 tokens
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_NEGATIVE_K | asd.ASD_DEVERR_CACHE
    b = Batch([2, 2, 2], [5, 1, 1], 4, 2, 64, BF16, 4, offsets=[0, 4, -1], total_rows=6)
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_ROWS
    b = Batch([2, 2, 2], [2, 1, 1], 4, 2, 64, BF16, 4)
    b.page_table[0, 0], b.page_table[1, 0] = -1, b.pages
    q, k, v = qkv(b)
    check_append(b, q, k, v, inv_freq=freq(64))
    assert asd.asd_device_error(clear=True) == asd.ASD_DEVERR_CACHE


def test_values_are_copied_as_they_are():
    b = Batch([3], [2], 2, 1, 64, F16, 4)
    q, k, v = qkv(b)
    v[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, -0.0], dtype=F16)
    check_append(b, q, k, v, inv_freq=freq(64))
    assert torch.signbit(b.v_cache[b.page_table[0, 0].long(), 2, 0, 3])


def test_a_captured_append_follows_its_buffers():
    b = Batch([4, 0, 7], [30, 3, 100], 8, 2, 128, BF16, 16)
    q, k, v = qkv(b)
    out = torch.empty((b.rows, 8, 128), dtype=BF16, device=DEV)
    f = freq(128)

    def call(into):
        asd.asd_rope_append(q, k, v, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens,
                            f, out_q=into)

    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for turn in range(4):
        q.copy_(b.randn(*q.shape))
        k.copy_(b.randn(*k.shape))
        b.cache_lens.copy_(torch.tensor([30 + turn, 3 - turn, 96 + turn]))
        b.k_cache.zero_()
        graph.replay()
        torch.cuda.synchronize()
        keys = b.k_cache.clone()
        b.k_cache.zero_()
        want = torch.empty_like(out)
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(keys, b.k_cache)
