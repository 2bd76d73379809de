"""asd_block_attention at the end of the accepted lengths: the last tokens of a sequence of 2^31 - 2."""
import math

import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, half_step

pytestmark = pytest.mark.gpu


def test_the_last_tokens_of_the_longest_sequence_count():
    """All pages but the last are one page of one token, whose slots lie on each other; the last page's
    tokens share another one, whose weight is about that of all others together."""
    page, entries, rows, d = 126, 17043521, 3, 64            # 126 * 17,043,521 = 2^31 - 2
    assert page * entries == 2 ** 31 - 2
    table = torch.zeros((1, entries), dtype=torch.int32, device=DEV)
    table[0, -1] = 1
    keys = torch.zeros((2, 1, 1, d), dtype=torch.float16, device=DEV)
    values = torch.zeros_like(keys)
    score = 16.59375
    keys[1, ..., 0] = score
    values[1] = 1.0
    q = torch.zeros((rows, 1, d), dtype=torch.float16, device=DEV)
    q[..., 0] = math.sqrt(d)
    cached = page * entries - rows
    asd.asd_device_error(clear=True)
    out = asd.asd_block_attention(
        q, keys.expand(2, page, 1, d), values.expand(2, page, 1, d), table,
        torch.tensor([cached], device=DEV), torch.tensor([rows - 1], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert asd.asd_device_error(clear=True) == 0
    others = float(page * (entries - 1))
    for p in range(rows):
        last = (cached + p + 1 - others) * math.exp(score)
        want = last / (others + last)
        # the score's difference in binary32 (24 octaves, two roundings), and the result's rounding; one
        # token more or less would be off by 0.002
        bound = half_step(torch.float16) * want + 24 * 2.0 ** -22
        assert (out[p].double() - want).abs().max().item() <= bound
