"""Helpers of the decoding operators' tests: batches of blocks over a paged cache, and the
comparison of a call's outputs with the 64-bit forms of ``oracle/decode.py``."""
import numpy as np
import torch

import paper_2608_03447_amd as asd
from oracle import decode

DEV = "cuda:0"


def half_step(dtype):
    """The greatest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Half the spacing of the subnormal numbers: the absolute error of a rounding near zero."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def exact64(t):
    return t.detach().double().cpu().numpy()


def host(t):
    return None if t is None else t.cpu().numpy()


class Batch:
    """Blocks of `lens` drafts over caches of `cached` tokens, in pages that lie in any order."""

    def __init__(self, lens, cached, hq, hkv, d, dtype, page, seed=0, layout="nhd", offsets=None,
                 total_rows=None, spare=2, width=None):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.cached = list(lens), list(cached)
        self.n, self.page, self.hq, self.hkv, self.d, self.dtype = len(self.lens), page, hq, hkv, d, dtype
        counts = [max(k, 0) + 1 for k in self.lens]
        self.rows = total_rows if total_rows is not None else sum(counts)
        need = [(max(c, 0) + m + page - 1) // page for c, m in zip(self.cached, counts)]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=gen)
        table = torch.zeros((self.n, width or max(need + [1])), dtype=torch.int32)
        at = 0
        for i, m in enumerate(need):
            m = min(m, table.shape[1])
            table[i, :m] = order[at:at + m].to(torch.int32)
            at += m
        self.gen = gen
        self.page_table = table.to(DEV)
        self.block_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.cache_lens = torch.tensor(self.cached, dtype=torch.int64, device=DEV)
        self.row_offsets = None if offsets is None else torch.tensor(offsets, dtype=torch.int64,
                                                                     device=DEV)
        self.k_cache, self.v_cache = self._cache(layout), self._cache(layout)
        if layout == "both":      # keys and values of a page next to each other in one array
            both = torch.stack([self.k_cache, self.v_cache], 1)
            self.k_cache, self.v_cache = both[:, 0], both[:, 1]

    def randn(self, *shape, scale=1.0):
        return (scale * torch.randn(shape, generator=self.gen)).to(self.dtype).to(DEV)

    def _cache(self, layout):
        if layout == "hnd":
            return self.randn(self.pages, self.hkv, self.page, self.d).transpose(1, 2)
        return self.randn(self.pages, self.page, self.hkv, self.d)

    def trees(self, words=1):
        """A random ancestor mask: every row sees itself and the rows above it in its tree."""
        mask = np.zeros((self.rows, words), dtype=np.uint64)
        first = 0
        rng = np.random.default_rng(7)
        for k in self.lens:
            seen = []
            for j in range(max(k, 0) + 1):
                bits = (seen[int(rng.integers(j))] if j else 0) | 1 << j
                seen.append(bits)
                for w in range(words):
                    mask[first + j, w] = bits >> (64 * w) & (1 << 64) - 1
            first += max(k, 0) + 1
        return torch.from_numpy(mask.view(np.int64)).to(DEV)


def check_append(b, q, k, v, **kw):
    """asd_rope_append against the 64-bit form: every element of q_out and of both caches."""
    before_k, before_v = b.k_cache.clone(), b.v_cache.clone()
    args = {name: kw.get(name) for name in ("q_norm", "k_norm", "positions")}
    inv_freq, eps = kw.get("inv_freq"), kw.get("eps", 1e-6)
    out = kw.get("out_q")
    if q is not None and out is None:
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    q64 = None if q is None else exact64(q)
    ref = decode.rope_append(
        q64, exact64(k), exact64(v), exact64(before_k), exact64(before_v), host(b.page_table),
        b.cached, b.lens, host(inv_freq), eps=eps, interleaved=kw.get("interleaved", False),
        row_offsets=host(b.row_offsets), positions=host(args["positions"]),
        q_norm=None if args["q_norm"] is None else exact64(args["q_norm"]),
        k_norm=None if args["k_norm"] is None else exact64(args["k_norm"]))
    got = asd.asd_rope_append(q, k, v, b.k_cache, b.v_cache, b.page_table, b.cache_lens,
                              b.block_lens, inv_freq, eps=eps, row_offsets=b.row_offsets,
                              interleaved=kw.get("interleaved", False), out_q=out, **args)
    torch.cuda.synchronize()
    # binary32 before the one rounding: the norm's sum of d squares, its root and the products
    # (d + 8 roundings at most), the angle's sine and cosine and the turn (24 with a margin)
    near = (b.d + 32) * 2.0 ** -24

    def close(name, x, want, size):
        x = exact64(x)
        bound = half_step(b.dtype) * np.abs(want) * (1 + near) + near * size + smallest(b.dtype)
        worst = np.abs(x - want) - bound
        assert not (worst > 0).any(), "%s: off by %g beyond its bound at %s" % (
            name, worst.max(), np.unravel_index(worst.argmax(), worst.shape))

    if q is None:
        assert got is None
    else:
        written = ~np.isnan(ref[0])
        x = exact64(got)
        assert (x[~written] == 7.0).all() or kw.get("out_q") is not None
        close("q", got, np.where(written, ref[0], x), ref[3])
    untouched = (ref[4] == 0).all(-1)
    same = (b.k_cache == before_k) | (b.k_cache.isnan() & before_k.isnan())
    assert same.cpu().numpy()[untouched].all()
    close("keys", b.k_cache, ref[1], ref[4])
    assert np.array_equal(exact64(b.v_cache), ref[2], equal_nan=True)


def attention_bound(b, out, mean, reach, tokens):
    """What the roundings of the operator amount to: scores and sums in binary32, weights rounded
    once to dtype, the result rounded once."""
    eps = 2.0 ** -24
    score = (b.d + 4) * eps * reach[..., None]         # of one score; the maximum's adds as much
    weights = half_step(b.dtype) * 1.01 + 2 * score + (tokens + 64) * eps
    return mean * weights + half_step(b.dtype) * np.abs(out) * 1.01 + smallest(b.dtype)


def check_attention(b, q, mask=None, scale=None, **kw):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    asd.asd_block_attention(q, b.k_cache, b.v_cache, b.page_table, b.cache_lens, b.block_lens,
                            scale=scale, mask=mask, row_offsets=b.row_offsets, out=out, **kw)
    torch.cuda.synchronize()
    ref, mean, reach = decode.block_attention(
        exact64(q), exact64(b.k_cache), exact64(b.v_cache), host(b.page_table), b.cached, b.lens,
        b.d ** -0.5 if scale is None else scale, None if mask is None else host(mask),
        host(b.row_offsets))
    got = exact64(out)
    written = ~np.isnan(ref).all(-1)
    assert (got[~written] == 7.0).all(), "rows of no request were written"
    bound = attention_bound(b, ref, mean, reach, max(c + max(k, 0) + 1 for c, k in
                                                     zip(b.cached, b.lens)))
    over = (np.abs(got - ref) - bound)[written]
    assert not np.isnan(over).any() and (over <= 0).all(), "off by %g beyond the bound" % over.max()
    return out
