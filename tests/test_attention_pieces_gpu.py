"""asd_block_attention over prompt pieces, alone and among single tokens, against products in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch, attention_bound, exact64

pytestmark = pytest.mark.gpu


def exact(b, q, mask):
    """(out, weighted |V|, the scores' reach) of every row and head."""
    rows, heads, d = q.shape
    out = torch.zeros((rows, heads, d), dtype=torch.float64, device=DEV)
    mean, reach = torch.zeros_like(out), torch.zeros((rows, heads), dtype=torch.float64, device=DEV)
    group, scale, first = heads // b.hkv, d ** -0.5, 0
    for i, (k, cached) in enumerate(zip(b.lens, b.cached)):
        count = k + 1
        token = torch.arange(cached + count, device=DEV)
        page, slot = b.page_table[i, token // b.page].long(), token % b.page
        if mask is None:
            seen = torch.ones((count, count), dtype=torch.bool, device=DEV).tril()
        else:
            j = torch.arange(count, device=DEV)
            seen = (mask[first:first + count][:, j // 64] >> (j % 64)) & 1 != 0
        seen = torch.cat([torch.ones((count, cached), dtype=torch.bool, device=DEV), seen], 1)
        for h in range(heads):
            x = q[first:first + count, h].double()
            keys, values = (c[page, slot, h // group].double() for c in (b.k_cache, b.v_cache))
            w = torch.softmax((scale * (x @ keys.T.contiguous())).masked_fill(~seen, float("-inf")), 1)
            out[first:first + count, h] = w @ values
            mean[first:first + count, h] = w @ values.abs()
            reach[first:first + count, h] = scale * (x.abs() @ keys.abs().T.contiguous()).amax(1)
        first += count
    return (t.cpu().numpy() for t in (out, mean, reach))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (32, 1, 64), (4, 2, 256)])
@pytest.mark.parametrize("lens,cached", [([1499], [100]), ([0, 1203, 0, 700, 3, 0], [4000, 77, 0, 1, 800, 129]),
                                         ([511] * 4 + [0] * 60, [0, 64, 200, 1000] + [37 * j for j in range(60)])])
def test_prompt_pieces_among_single_tokens(lens, cached, hq, hkv, d, dtype):
    b = Batch(lens, cached, hq, hkv, d, dtype, 16, seed=d + len(lens))
    q = b.randn(b.rows, hq, d, scale=1.5)
    tokens = max(c + k + 1 for c, k in zip(cached, lens))
    for mask in (None, b.trees(24)):
        out = asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens, mask=mask)
        torch.cuda.synchronize()
        want, mean, reach = exact(b, q, mask)
        over = np.abs(exact64(out) - want) - attention_bound(b, want, mean, reach, tokens)
        assert (over <= 0).all(), "off by %g beyond the bound" % over.max()
