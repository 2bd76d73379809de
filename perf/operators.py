"""The decoding operators beside the verifier, as cases that can be timed.

A case is a dict of plain values.  ``prepare`` makes on the GPU what a serving
program holds before the call, ``run`` makes one pass through one operator, in
its plain form (elementary torch operations in 32 bits, in 64 where 32 lose
what matters) or, where ``own`` is true, as the public call of the framework;
``exact`` gives the same outputs in 64 bits, from the definitions alone.

Three operators of a decoding round:

append   ``asd_rope_append``: the norms of queries and keys, the position
         rotation, and the append of keys and values to a paged cache
attend   ``asd_block_attention``: attention of draft blocks (chains) or draft
         trees over that cache; a block of one row is single-token decoding
sample   ``asd_sample``: one token per logit row by temperature, top-k, top-p
         and min-p, from given random numbers

The vocabularies and block lengths are those of the repository's workloads
(blocks of 0 to 32 drafts, 32,000 / 129,280 / 151,936 tokens); head layouts
are generic.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # One request decoding alone enters its block of 8 drafts and the token
        # before them into the cache, the smallest append: latency is all.
        {"name": "append-1x9-bf16", "kind": "append", "n": 1, "k": 8, "ragged": False,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 900, "page": 16, "tree": False,
         "norm": True, "interleaved": False, "rot": 128, "theta": 1e6, "layout": "nhd"},
        # Single tokens of a batch without drafts: small heads, pairs next to
        # each other, half of each head rotated, pages of odd size, head-major.
        {"name": "append-61x1-f16-d64", "kind": "append", "n": 61, "k": 0, "ragged": False,
         "hq": 24, "hkv": 24, "d": 64, "dtype": "f16", "ctx": 500, "page": 7, "tree": False,
         "norm": False, "interleaved": True, "rot": 32, "theta": 1e4, "layout": "hnd"},
        # The headline batch of the verifier: 256 blocks of 16 drafts.
        {"name": "append-256x17-bf16", "kind": "append", "n": 256, "k": 16, "ragged": False,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 300, "page": 16, "tree": False,
         "norm": True, "interleaved": False, "rot": 128, "theta": 1e6, "layout": "nhd"},
        # Prompts that enter the cache in long ragged pieces, the largest.
        {"name": "append-8xlong-bf16", "kind": "append", "n": 8, "k": 2300, "ragged": True,
         "hq": 64, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 1000, "page": 64, "tree": False,
         "norm": True, "interleaved": False, "rot": 128, "theta": 5e5, "layout": "nhd"},
        # One token of one request over a short cache: latency.
        {"name": "attend-1x1-bf16", "kind": "attend", "n": 1, "k": 0, "ragged": False,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 700, "spread": False, "page": 16,
         "tree": False, "layout": "nhd"},
        # One long sequence decoding alone: few rows, the cache split over the chip.
        {"name": "attend-1x9-long-bf16", "kind": "attend", "n": 1, "k": 8, "ragged": False,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 65000, "spread": False, "page": 64,
         "tree": False, "layout": "nhd"},
        # Single tokens of a batch whose sequences are anything up to 8,192 long.
        {"name": "attend-64x1-ragged-bf16", "kind": "attend", "n": 64, "k": 0, "ragged": False,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 8192, "spread": True, "page": 16,
         "tree": False, "layout": "nhd"},
        # Ragged draft blocks of a batch, small heads, odd pages, head-major.
        {"name": "attend-32xragged-f16-d64", "kind": "attend", "n": 32, "k": 16, "ragged": True,
         "hq": 24, "hkv": 4, "d": 64, "dtype": "f16", "ctx": 4001, "spread": True, "page": 24,
         "tree": False, "layout": "hnd"},
        # Trees of 64 drafts over long caches: rows enough for the matrix cores.
        {"name": "attend-16xtree64-bf16", "kind": "attend", "n": 16, "k": 63, "ragged": False,
         "hq": 64, "hkv": 8, "d": 128, "dtype": "bf16", "ctx": 16000, "spread": False, "page": 16,
         "tree": True, "layout": "nhd"},
        # One row, the usual filters together: latency.
        {"name": "sample-1x32000-f32", "kind": "sample", "rows": 1, "vocab": 32000, "pad": 0,
         "dtype": "f32", "mode": "usual"},
        # A small batch, rows padded, every combination of filters, greedy rows too.
        {"name": "sample-67x129280-bf16", "kind": "sample", "rows": 67, "vocab": 129280, "pad": 96,
         "dtype": "bf16", "mode": "mixed"},
        # The rows of 64 blocks of 32 drafts in float32 with every combination, the largest.
        {"name": "sample-2112x151936-f32", "kind": "sample", "rows": 2112, "vocab": 151936,
         "pad": 0, "dtype": "f32", "mode": "mixed"},
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


# No drawn case moves or computes more than the largest listed one of its kind.
_LIMITS = {}


def _limit(kind):
    if not _LIMITS:
        for case in listed():
            w = work(case)
            b, f = _LIMITS.get(case["kind"], (0, 0))
            _LIMITS[case["kind"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    return _LIMITS[kind]


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["append", "attend", "sample"])
    while True:
        if kind == "sample":
            case = {"kind": kind, "rows": _log_int(rng, 1, 2112), "vocab": _log_int(rng, 300, 151936),
                    "pad": rng.choice([0, 0, 1, 64]), "dtype": rng.choice(["f32", "bf16", "f16"]),
                    "mode": rng.choice(["usual", "mixed", "mixed"])}
        else:
            group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 16])
            hkv = rng.choice([1, 2, 4, 5, 8, 16])
            case = {"kind": kind, "n": _log_int(rng, 1, 256), "ragged": rng.random() < 0.5,
                    "hq": hkv * group, "hkv": hkv, "d": rng.choice([64, 128, 128, 128]),
                    "dtype": rng.choice(["bf16", "f16"]), "page": rng.choice([1, 7, 16, 24, 64, 256]),
                    "layout": rng.choice(["nhd", "hnd"])}
            if kind == "append":
                case.update(k=_log_int(rng, 1, 2300) - 1, ctx=_log_int(rng, 1, 1000),
                            norm=rng.random() < 0.5, interleaved=rng.random() < 0.5,
                            theta=rng.choice([1e4, 5e5, 1e6]))
                case["rot"] = case["d"] // rng.choice([1, 1, 2, 4])
                case["tree"] = case["k"] < 64 and rng.random() < 0.3
            else:
                case.update(k=rng.choice([0, _log_int(rng, 1, 64) - 1]), ctx=_log_int(rng, 1, 65000),
                            spread=rng.random() < 0.5)
                case["tree"] = rng.random() < 0.4
            # what the caches hold in all, so that a state stays small beside the card
            if case["n"] * (case["ctx"] + case["k"] + 1 + case["page"]) * hkv * case["d"] > 1 << 30:
                continue
        w, (b, f) = work(case), _limit(kind)
        if w["bytes"] <= b and w["flops"] <= f:
            return case


# ---------------------------------------------------------------- inputs

def _spread(low, high, n):
    """n whole numbers over [low, high], the same for every seed (a case's work is
    its own), in an order that mixes short and long."""
    if n == 1:
        return [high]
    step = 1
    for s in (7, 5, 11, 13, 3, 17, 19, 23):     # one that visits every index
        if math.gcd(s, n) == 1:
            step = s
            break
    return [low + (high - low) * ((i * step) % n) // (n - 1) for i in range(n)]


def _blocks(case):
    """(K_i, cached tokens) of every request."""
    n, k, ctx = case["n"], case["k"], case["ctx"]
    lens = _spread(0, k, n) if case["ragged"] else [k] * n
    spread = case.get("spread", False)
    cached = _spread(0, ctx, n) if spread else [ctx - (i % 5 if ctx > 4 else 0) for i in range(n)]
    return lens, cached


def _tree(size, gen):
    """Ancestors (the node itself among them) and depth of every node of a random
    draft tree: node 0 is the last committed token, each node hangs under an
    earlier one."""
    parent = [-1] + [int(x) for x in
                     (torch.rand(size, generator=gen) * torch.arange(1, size + 1)).tolist()][:size - 1]
    seen, depth = [], []
    for j in range(size):
        above = seen[parent[j]] if j else 0
        seen.append(above | (1 << j))
        depth.append(depth[parent[j]] + 1 if j else 0)
    return seen, depth


def _signed(bits):
    return bits - (1 << 64) if bits >= 1 << 63 else bits


def _cache(case, pages, gen, dtype):
    """[pages, page, hkv, d] keys or values, as they lie in memory token-major or head-major."""
    p, h, d = case["page"], case["hkv"], case["d"]
    if case["layout"] == "hnd":
        return torch.randn((pages, h, p, d), generator=gen, device=DEVICE).to(dtype).transpose(1, 2)
    return torch.randn((pages, p, h, d), generator=gen, device=DEVICE).to(dtype)


def _prepare_blocks(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    lens, cached = _blocks(case)
    rows = sum(lens) + len(lens)
    need = [(c + k + 1 + page - 1) // page for c, k in zip(cached, lens)]
    width = max(need)
    pages = sum(need) + 3                                  # three that no request owns
    order = torch.randperm(pages, generator=host)
    table = torch.zeros((case["n"], width), dtype=torch.int32)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m].to(torch.int32)
        at += m
    state = {"case": case, "lens": lens, "cached": cached,
             "block_lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE),
             "cache_lens": torch.tensor(cached, dtype=torch.int64, device=DEVICE),
             "page_table": table.to(DEVICE),
             "k_cache": _cache(case, pages, gen, dtype), "v_cache": _cache(case, pages, gen, dtype),
             "mask": None, "positions": None}
    if case["tree"]:
        words, places = [], []
        for k, c in zip(lens, cached):
            seen, depth = _tree(k + 1, host)
            words += [_signed(b) for b in seen]
            places += [c + x for x in depth]
        state["mask"] = torch.tensor(words, dtype=torch.int64, device=DEVICE).reshape(rows, 1)
        state["positions"] = torch.tensor(places, dtype=torch.int64, device=DEVICE)
    if case["kind"] == "attend":
        # queries that make some keys stand out, as trained heads do
        state["q"] = (2.0 * torch.randn((rows, hq, d), generator=gen, device=DEVICE)).to(dtype)
        return state
    # the three parts of one projection's output, as views of its rows
    fused = (1.5 * torch.randn((rows, (hq + 2 * hkv) * d), generator=gen, device=DEVICE)).to(dtype)
    state["q"] = fused[:, :hq * d].unflatten(1, (hq, d))
    state["k"] = fused[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    state["v"] = fused[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
    state["q_norm"] = state["k_norm"] = None
    if case["norm"]:
        state["q_norm"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE)).to(dtype)
        state["k_norm"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE)).to(dtype)
    half = torch.arange(case["rot"] // 2, dtype=torch.float64)
    state["inv_freq"] = (case["theta"] ** (-2.0 * half / case["rot"])).to(torch.float32).to(DEVICE)
    return state


def _prepare_sample(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    # N(0, 2) noise with 48 likelier tokens a row: by how much they stand out
    # differs from row to row, so some rows are nearly decided and some flat
    z = torch.randn((rows, vocab + case["pad"]), generator=gen, device=DEVICE).mul_(2.0)
    likely = torch.randint(vocab, (rows, 48), generator=gen, device=DEVICE)
    height = 14.0 * torch.rand((rows, 1), generator=gen, device=DEVICE)
    z.scatter_add_(1, likely, height * torch.rand((rows, 48), generator=gen, device=DEVICE))
    logits = z.to(DTYPES[case["dtype"]])[:, :vocab]
    u = torch.rand(rows, generator=gen, device=DEVICE)
    if case["mode"] == "usual":
        t = torch.full((rows,), 0.8, device=DEVICE)
        k = torch.full((rows,), 50, dtype=torch.int32, device=DEVICE)
        p = torch.full((rows,), 0.95, device=DEVICE)
        m = torch.zeros(rows, device=DEVICE)
    else:
        def pick(values, dtype):
            at = torch.randint(len(values), (rows,), generator=gen, device=DEVICE)
            return torch.tensor(values, dtype=dtype, device=DEVICE)[at]
        t = pick([0.0, 0.5, 0.7, 0.8, 1.0, 1.0, 1.0, 1.3], torch.float32)
        k = pick([0, 0, 0, 1, 20, 50, 100, 1000], torch.int32)
        p = pick([1.0, 1.0, 0.95, 0.9, 0.8, 0.5], torch.float32)
        m = pick([0.0, 0.0, 0.0, 0.02, 0.05, 0.1], torch.float32)
    return {"case": case, "logits": logits, "u": u, "temperature": t, "top_k": k, "top_p": p,
            "min_p": m}


def prepare(case, seed):
    return _prepare_sample(case, seed) if case["kind"] == "sample" else _prepare_blocks(case, seed)


# ---------------------------------------------------------------- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_append(s):
    import paper_2608_03447_amd as asd
    q = asd.asd_rope_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"],
                            s["cache_lens"], s["block_lens"], s["inv_freq"], q_norm=s["q_norm"],
                            k_norm=s["k_norm"], eps=EPS, positions=s["positions"],
                            interleaved=s["case"]["interleaved"])
    return q, s["k_cache"], s["v_cache"]


def _own_attend(s):
    import paper_2608_03447_amd as asd
    return asd.asd_block_attention(s["q"], s["k_cache"], s["v_cache"], s["page_table"],
                                   s["cache_lens"], s["block_lens"], mask=s["mask"])


def _own_sample(s):
    import paper_2608_03447_amd as asd
    prob = torch.empty_like(s["u"])
    token = asd.asd_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                           top_p=s["top_p"], min_p=s["min_p"], out_prob=prob)
    return token, prob


def _rows_of(s):
    """Request and place in its block of every row (packed blocks)."""
    count = s["block_lens"].long() + 1
    request = torch.repeat_interleave(torch.arange(len(count), device=DEVICE), count,
                                      output_size=s["q"].shape[0])
    first = torch.cumsum(count, 0) - count
    return request, torch.arange(len(request), device=DEVICE) - first[request]


def _plain_append(s):
    case = s["case"]
    dtype, rot, page = DTYPES[case["dtype"]], case["rot"], case["page"]
    request, place = _rows_of(s)
    at = s["cache_lens"][request] + place                     # the token's place in its cache
    position = at if s["positions"] is None else s["positions"]
    # the angle in 64 bits: at far positions 32 would lose it
    angle = position.double()[:, None] * s["inv_freq"].double()[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def turn(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        out = x.clone()
        if case["interleaved"]:
            a, b = slice(0, rot, 2), slice(1, rot, 2)
        else:
            a, b = slice(0, rot // 2), slice(rot // 2, rot)
        out[..., a] = x[..., a] * cos - x[..., b] * sin
        out[..., b] = x[..., a] * sin + x[..., b] * cos
        return out.to(dtype)

    where = s["page_table"][request, at // page].long()
    s["k_cache"][where, at % page] = turn(s["k"], s["k_norm"])
    s["v_cache"][where, at % page] = s["v"]
    return turn(s["q"], s["q_norm"]), s["k_cache"], s["v_cache"]


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    scale = 1.0 / math.sqrt(d)
    out = torch.empty_like(s["q"])
    first = 0
    for i, (k, cached) in enumerate(zip(s["lens"], s["cached"])):
        rows, total = k + 1, cached + k + 1
        token = torch.arange(total, device=DEVICE)
        where = s["page_table"][i, token // page].long()
        keys = s["k_cache"][where, token % page].float().permute(1, 2, 0).contiguous()
        values = s["v_cache"][where, token % page].float().permute(1, 0, 2).contiguous()
        q = s["q"][first:first + rows].float().reshape(rows, hkv, hq // hkv, d)
        q = q.permute(1, 0, 2, 3).reshape(hkv, rows * (hq // hkv), d).contiguous()
        score = (torch.matmul(q, keys) * scale).reshape(hkv, rows, hq // hkv, total)
        node = torch.arange(rows, device=DEVICE)
        if s["mask"] is None:
            seen = node[None, :] <= node[:, None]
        else:
            seen = (s["mask"][first:first + rows, :1] >> node[None, :]) & 1 == 1
        score[..., cached:] = score[..., cached:].masked_fill(~seen[None, :, None, :], -math.inf)
        weight = torch.exp(score - score.amax(-1, keepdim=True))
        weight = weight / weight.sum(-1, keepdim=True)
        o = torch.matmul(weight.reshape(hkv, -1, total), values)
        o = o.reshape(hkv, rows, hq // hkv, d).permute(1, 0, 2, 3).reshape(rows, hq, d)
        out[first:first + rows] = o.to(out.dtype)
        first += rows
    return out


def _plain_sample(s):
    vocab = s["case"]["vocab"]
    z, order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    # 64 bits: a draw or a nucleus' edge next to a running sum of 10^5 terms
    weight = torch.exp((z.double() - z[:, :1].double()) / torch.where(greedy, 1.0, t))
    place = torch.arange(vocab, device=DEVICE)[None, :]
    k = s["top_k"].long()[:, None]
    keep = (place < torch.where(k <= 0, vocab, k))
    mass = torch.where(keep, weight, 0.0)
    below = torch.cumsum(mass, 1)
    p = s["top_p"].double()[:, None]
    whole = mass.sum(1, keepdim=True)
    keep &= ((below - mass) < p * whole) | (p >= 1)
    keep &= weight >= s["min_p"].double()[:, None]
    keep[:, 0] = True
    keep &= ~greedy | (place == 0)
    kept = torch.zeros_like(weight).scatter_(1, order, torch.where(keep, weight, 0.0))
    del mass, below, weight
    run_sum = torch.cumsum(kept, 1)
    target = s["u"].double()[:, None] * run_sum[:, -1:]
    above = (run_sum > target) & (kept > 0)
    token = torch.argmax(above.to(torch.int8), dim=1, keepdim=True)
    prob = kept.gather(1, token) / run_sum[:, -1:]
    return token[:, 0].to(torch.int32), prob[:, 0].float()


_OWN = {"append": _own_append, "attend": _own_attend, "sample": _own_sample}
_PLAIN = {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}


# ---------------------------------------------------------------- work

def work(case):
    if case["kind"] == "sample":
        cells = case["rows"] * case["vocab"]
        return {"bytes": cells * SIZES[case["dtype"]] + case["rows"] * 28, "flops": 3 * cells}
    lens, cached = _blocks(case)
    rows = sum(lens) + len(lens)
    size, d, hq, hkv = SIZES[case["dtype"]], case["d"], case["hq"], case["hkv"]
    if case["kind"] == "append":
        cells = rows * (hq + 2 * hkv) * d
        turned = rows * (hq + hkv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))
        return {"bytes": 2 * cells * size + rows * 12, "flops": turned}
    pairs = sum((k + 1) * c + (k + 1) * (k + 2) // 2 for k, c in zip(lens, cached))
    tokens = sum(k + 1 + c for k, c in zip(lens, cached))
    return {"bytes": (2 * tokens * hkv + 2 * rows * hq) * d * size, "flops": 4 * pairs * hq * d}


# ---------------------------------------------------------------- 64 bits

def _exact_append(case, seed):
    s = prepare(case, seed)
    rot, page = case["rot"], case["page"]
    freq = s["inv_freq"].double()
    keys, values = s["k_cache"].double(), s["v_cache"].double()
    queries = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    pair = torch.arange(rot // 2, device=DEVICE)
    a, b = (2 * pair, 2 * pair + 1) if case["interleaved"] else (pair, pair + rot // 2)

    def turned(x, weight, angle):
        x = x.double()
        if weight is not None:
            x = weight.double() * x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        z = torch.polar(torch.ones_like(angle), angle)[:, None, :] * torch.complex(x[..., a], x[..., b])
        y = x.clone()
        y[..., a], y[..., b] = z.real, z.imag
        return y

    first = 0
    for i, (k, cached) in enumerate(zip(s["lens"], s["cached"])):
        part = slice(first, first + k + 1)
        token = torch.arange(cached, cached + k + 1, device=DEVICE)
        place = token if s["positions"] is None else s["positions"][part]
        angle = torch.outer(place.double(), freq)
        queries[part] = turned(s["q"][part], s["q_norm"], angle)
        where = s["page_table"][i].long()[token // page]
        keys[where, token % page] = turned(s["k"][part], s["k_norm"], angle)
        values[where, token % page] = s["v"][part].double()
        first += k + 1
    return queries, keys, values


def _exact_attend(case, seed):
    s = prepare(case, seed)
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    group = hq // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    first = 0
    for i, (k, cached) in enumerate(zip(s["lens"], s["cached"])):
        rows, total = k + 1, cached + k + 1
        slot = s["page_table"][i].long().repeat_interleave(page)[:total]
        inside = torch.arange(total, device=DEVICE) % page
        hidden = torch.zeros((rows, total), dtype=torch.bool, device=DEVICE)
        for r in range(rows):
            if s["mask"] is None:
                hidden[r, cached + r + 1:] = True
            else:
                bits = int(s["mask"][first + r, 0]) & ((1 << 64) - 1)
                hidden[r, cached:] = torch.tensor([bits >> j & 1 == 0 for j in range(rows)],
                                                  device=DEVICE)
        for h in range(hkv):
            keys = s["k_cache"][slot, inside, h].double()
            values = s["v_cache"][slot, inside, h].double()
            for x in range(h * group, (h + 1) * group):
                score = s["q"][first:first + rows, x].double() @ keys.T.contiguous() / d ** 0.5
                score[hidden] = -math.inf
                out[first:first + rows, x] = torch.softmax(score, 1) @ values
        first += rows
    return out


def _exact_sample(case, seed):
    s = prepare(case, seed)
    rows = case["rows"]
    token = torch.empty(rows, dtype=torch.int32, device=DEVICE)
    prob = torch.empty(rows, dtype=torch.float64, device=DEVICE)
    t, k, p, m, u = (s[name].double().tolist()
                     for name in ("temperature", "top_k", "top_p", "min_p", "u"))
    for r in range(rows):
        z = s["logits"][r].double()
        if t[r] <= 0:
            token[r], prob[r] = (z == z.max()).nonzero()[0, 0], 1.0
            continue
        # by the distinct values, greatest first: how many tokens have each and what they weigh
        value, count = torch.unique(z, return_counts=True)
        value, count = value.flip(0), count.flip(0).double()
        weight = torch.exp((value - value[0]) / t[r])
        limit = k[r] if k[r] > 0 else float(case["vocab"])
        before = torch.cumsum(count, 0) - count
        taken = torch.minimum(count, (limit - before).clamp(min=0.0))
        mass = torch.cumsum(taken * weight, 0)
        if p[r] < 1:
            # the value on which the nucleus ends, and how many tokens of it are needed
            goal = p[r] * mass[-1]
            end = int((mass < goal).sum())
            rest = goal - (mass[end - 1] if end else 0.0)
            taken[end] = torch.minimum(taken[end], torch.ceil(rest / weight[end]).clamp(min=1.0))
            taken[end + 1:] = 0
        taken[1:] *= weight[1:] >= m[r]
        last = int((taken > 0).nonzero()[-1, 0])
        kept = torch.where(z > value[last], torch.exp((z - value[0]) / t[r]), 0.0)
        kept[(z == value[last]).nonzero()[:int(taken[last]), 0]] = weight[last]
        total = torch.cumsum(kept, 0)
        at = int((total <= u[r] * total[-1]).sum())
        token[r], prob[r] = at, kept[at] / total[-1]
    return token, prob


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[
        case["kind"]](case, seed)
