"""asd_block_attention divides by the weights as they enter the product, so that their rounding
moves a row only as far as its values differ."""
import numpy as np
import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch, exact64, half_step, host, smallest
from oracle import decode

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
SHAPES = [([0] * 5, [0, 1, 40, 300, 700], 8, 2), ([12, 3, 0], [500, 31, 90], 8, 2),
          ([63, 20], [130, 260], 8, 1), ([0], [5000], 4, 1)]


def attend(b, q, mask=None):
    out = asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens,
                                  mask=mask)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,cached,hq,hkv", SHAPES)
def test_rows_of_equal_values_give_that_value(lens, cached, hq, hkv, d, dtype):
    """No sum here passes through more than 200 roundings to binary32 (40 products of 32 tokens a wavefront,
    32 tokens in each, then the joins): 2^-16 of the sum, and the value is 2^-12 of itself or more away from
    where another one would be the nearest."""
    b = Batch(lens, cached, hq, hkv, d, dtype, 16, seed=d + len(lens))
    q = b.randn(b.rows, hq, d, scale=1.5)
    for value in (1.2890625, -0.0059814453125):
        b.v_cache.fill_(value)
        want = torch.tensor(value, dtype=dtype)
        for mask in (None, b.trees(2)):
            assert bool((attend(b, q, mask).cpu() == want).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,cached,hq,hkv", SHAPES)
def test_values_next_to_each_other(lens, cached, hq, hkv, d, dtype):
    """With weights w (1 + e), |e| at most half a step and the scores' errors, the quotient is off by
    sum p |e| |V - mean| to first order, beside the binary32 sums and the one rounding of the result."""
    b = Batch(lens, cached, hq, hkv, d, dtype, 16, seed=3 * d + len(lens))
    q = b.randn(b.rows, hq, d, scale=1.5)
    values = 8.0 + 0.125 * torch.randn(b.v_cache.shape, generator=b.gen)
    b.v_cache.copy_(values.to(dtype))
    got = exact64(attend(b, q))
    args = [host(b.page_table), b.cached, b.lens, d ** -0.5]
    keys, v = exact64(b.k_cache), exact64(b.v_cache)
    want, mean, reach = decode.block_attention(exact64(q), keys, v, *args)
    _, apart, _ = decode.block_attention(exact64(q), keys, v - 8.0, *args)     # sum p |V - 8|
    apart = apart + np.abs(want - 8.0)                                         # at least sum p |V - mean|
    eps = 2.0 ** -24
    tokens = max(c + max(k, 0) + 1 for c, k in zip(cached, lens))
    score = (d + 4) * eps * reach[..., None]
    bound = (apart * (half_step(dtype) * 1.02 + 2 * score) + (tokens + 64) * eps * mean
             + half_step(dtype) * np.abs(want) * 1.01 + smallest(dtype))
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), "off by %g beyond the bound" % over.max()
