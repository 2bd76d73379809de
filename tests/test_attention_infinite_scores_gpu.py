"""Rows of asd_block_attention whose scores are all -infinity, and rows of which some are."""
import math

import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,cached,hq,hkv", [([0, 5], [40, 3], 4, 2), ([2], [6000], 4, 1)])
def test_scores_of_minus_infinity_weigh_nothing(lens, cached, hq, hkv, dtype):
    b = Batch(lens, cached, hq, hkv, 64, dtype, 16, seed=len(lens))
    q = b.randn(b.rows, hq, 64)
    q[..., 0] = 1.0
    b.k_cache[..., 0] = -math.inf

    def attend():
        out = asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens)
        torch.cuda.synchronize()
        return out

    assert bool((attend() == 0).all())
    # the first token of every sequence alone has a finite score
    first = b.page_table[:, 0].long()
    b.k_cache[first, 0, :, 0] = 0.0
    want = torch.empty_like(q)
    at = 0
    for i, k in enumerate(lens):
        value = b.v_cache[first[i], 0].repeat_interleave(hq // hkv, 0)
        want[at:at + k + 1] = value
        at += k + 1
    assert torch.equal(attend(), want)
