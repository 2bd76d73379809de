"""The decoding operators' native marshalling: the results of the Python marshalling for the
ordinary arguments, and no others taken."""
import pytest
import torch

import paper_2608_03447_amd as asd
from decode_gpu import DEV, Batch

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


class _Counts:
    """The native module, counting the calls it takes."""
    def __init__(self, fast):
        self.fast, self.taken = fast, 0

    def __getattr__(self, name):
        def call(*args):
            r = getattr(self.fast, name)(*args)
            self.taken += r is not None
            return r
        return call


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


class _Calls:
    """A batch and logits; each call's arguments by name, to be changed before it."""
    def __init__(self, dtype=BF16, layout="nhd"):
        b = Batch([3, 0, 5], [7, 30, 0], 4, 2, 64, dtype, 8, seed=2, layout=layout)
        freq = torch.rand(32, generator=torch.Generator().manual_seed(1)).to(DEV)
        rows = b.randn(b.rows, 8 * 64).unflatten(1, (8, 64))
        paged = dict(k_cache=b.k_cache, v_cache=b.v_cache, page_table=b.page_table,
                     cache_lens=b.cache_lens, block_lens=b.block_lens)
        self.append = dict(q=rows[:, :4], k=rows[:, 4:6], v=rows[:, 6:], inv_freq=freq, **paged)
        self.attend = dict(q=b.randn(b.rows, 4, 64), **paged)
        gen = torch.Generator().manual_seed(3)
        self.sample = dict(logits=torch.randn(5, 999, generator=gen).to(DEV),
                           uniform=torch.rand(5, generator=gen).to(DEV))
        self.batch = b

    def run(self, call):
        if call == "append":
            out = [asd.asd_rope_append(**self.append), self.batch.k_cache, self.batch.v_cache]
        elif call == "attend":
            out = [asd.asd_block_attention(**self.attend)]
        else:
            out = [asd.asd_sample(**self.sample), self.sample.get("out_prob")]
        torch.cuda.synchronize()
        return [None if t is None else t.cpu() for t in out]


def _norms(c):
    c.append.update(q_norm=torch.full((64,), 1.5, dtype=BF16, device=DEV),
                    k_norm=torch.full((64,), 0.5, dtype=BF16, device=DEV), eps=1e-5)


TAKEN = {
    "append": lambda c: None,
    "append, norms": _norms,
    "append, pairs side by side": lambda c: c.append.update(interleaved=True),
    "append, keys alone": lambda c: c.append.update(q=None),
    "append, no rotation": lambda c: c.append.update(inv_freq=None),
    "append, in place": lambda c: c.append.update(out_q=c.append["q"]),
    "append, places": lambda c: c.append.update(
        positions=torch.arange(c.batch.rows, device=DEV) * 3),
    "append, offsets": lambda c: c.append.update(
        row_offsets=torch.tensor([7, 0, 1], device=DEV),       # the last row is nobody's
        out_q=torch.zeros(c.batch.rows, 4, 64, dtype=BF16, device=DEV)) or c.append["block_lens"].copy_(
            torch.tensor([2, 0, 5])),
    "attend": lambda c: None,
    "attend, scale": lambda c: c.attend.update(scale=0.25),
    "attend, trees": lambda c: c.attend.update(mask=c.batch.trees(2)),
    "attend, given": lambda c: c.attend.update(
        out=torch.zeros_like(c.attend["q"]),
        workspace=torch.empty(asd.asd_block_attention_workspace_bytes(4, 2, 64, 3, c.batch.rows),
                              dtype=torch.uint8, device=DEV)),
    "sample": lambda c: None,
    "sample, bfloat16": lambda c: c.sample.update(logits=c.sample["logits"].bfloat16()),
    "sample, half": lambda c: c.sample.update(logits=c.sample["logits"].half()),
    "sample, rows apart": lambda c: c.sample.update(logits=c.sample["logits"][:, 3:900]),
    "sample, all": lambda c: c.sample.update(
        temperature=torch.full((5,), 0.7, device=DEV), top_p=torch.full((5,), 0.9, device=DEV),
        top_k=torch.full((5,), 20, dtype=torch.int32, device=DEV),
        min_p=torch.full((5,), 0.01, device=DEV), out_prob=torch.empty(5, device=DEV)),
}


@pytest.mark.parametrize("layout", ["nhd", "hnd", "both"])
@pytest.mark.parametrize("name", sorted(TAKEN))
def test_native_calls_equal_python_calls(name, layout, monkeypatch):
    results = []
    for fast in (_Counts(asd._load_fast()), _Declines()):
        monkeypatch.setattr(asd, "_fast", fast)
        c = _Calls(layout=layout)
        TAKEN[name](c)
        results.append(c.run(name.split(",")[0]))
        if isinstance(fast, _Counts):
            assert fast.taken == 1
    for a, b in zip(*results):
        assert (a is None and b is None) or torch.equal(a, b)


def test_half_blocks_and_given_outputs(monkeypatch):
    for fast in (_Counts(asd._load_fast()), _Declines()):
        monkeypatch.setattr(asd, "_fast", fast)
        c = _Calls(F16)
        out = torch.zeros(c.batch.rows, 4, 64, dtype=F16, device=DEV)
        assert asd.asd_rope_append(**c.append, out_q=out) is out
        other = torch.zeros_like(out)
        assert asd.asd_block_attention(**c.attend, out=other) is other
        token = torch.zeros(5, dtype=torch.int32, device=DEV)
        assert asd.asd_sample(**c.sample, out_token=token) is token
        if isinstance(fast, _Counts):
            assert fast.taken == 3


def _put(call, **values):
    return lambda c: getattr(c, call).update(values)


def _change(call, name, f):
    return lambda c: getattr(c, call).update({name: f(getattr(c, call)[name])})


LEFT = {
    "append, a norm of another type": _put("append", q_norm=torch.ones(64)),
    "append, an output without queries": lambda c: c.append.update(
        out_q=c.append["q"], q=None),
    "append, heads that do not match": _change("append", "v", lambda t: t[:, :1]),
    "append, heads apart": _change("append", "k", lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)),
    "append, too wide a turn": _change(
        "append", "inv_freq", lambda t: t.repeat(2)),
    "append, a table of long": _change("append", "page_table", lambda t: t.long()),
    "append, lengths on the host": _change("append", "block_lens", lambda t: t.cpu()),
    "append, short lengths": _change("append", "cache_lens", lambda t: t[:2]),
    "append, an integer eps": _put("append", eps=1),
    "attend, a cache of another type": _change("attend", "v_cache", lambda t: t.half()),
    "attend, elements apart": _change("attend", "k_cache", lambda t: t.repeat_interleave(2, 3)[..., ::2]),
    "attend, strided lengths": _change("attend", "block_lens", lambda t: t.repeat_interleave(2)[::2]),
    "attend, a mask of few rows": lambda c: c.attend.update(mask=c.batch.trees()[:-1]),
    "attend, float queries": _change("attend", "q", lambda t: t.float()),
    "attend, rows that are not dense": _change("attend", "q", lambda t: t.repeat(1, 2, 1)[:, ::2]),
    "attend, an output of another shape": lambda c: c.attend.update(out=c.attend["q"][:, :2]),
    "sample, scalars": _put("sample", temperature=0.5, top_k=10, top_p=0.9, min_p=0.01),
    "sample, columns": _change("sample", "logits", lambda t: t.t().contiguous().t()),
    "sample, doubles": _change("sample", "logits", lambda t: t.double()),
    "sample, too few numbers": _change("sample", "uniform", lambda t: t[:4]),
    "sample, no numbers": _put("sample", uniform=None),
    "sample, no rows": lambda c: c.sample.update(logits=c.sample["logits"][:0],
                                                 uniform=c.sample["uniform"][:0]),
}


@pytest.mark.parametrize("name", sorted(LEFT))
def test_other_arguments_are_left_to_python(name, monkeypatch):
    """The native function declines them: converted or refused by the Python code."""
    results = []
    for fast in (_Counts(asd._load_fast()), _Declines()):
        monkeypatch.setattr(asd, "_fast", fast)
        c = _Calls()
        LEFT[name](c)
        try:
            results.append(c.run(name.split(",")[0]))
        except ValueError as e:
            results.append(str(e))
        if isinstance(fast, _Counts):
            assert fast.taken == 0
    if isinstance(results[0], str) or isinstance(results[1], str):
        assert results[0] == results[1]
    else:
        for a, b in zip(*results):
            assert (a is None and b is None) or torch.equal(a, b)


def test_failing_status_raises():
    c = _Calls()
    with pytest.raises(asd.AsdError) as e:
        asd.asd_block_attention(**{**c.attend, "q": c.attend["q"].repeat(1, 2, 1)[:, :5].contiguous()})
    assert e.value.status == 1          # 5 query heads over 2 key heads
