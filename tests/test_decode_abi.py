"""The decoding operators refuse what the host can see to be wrong, with nothing launched (CPU)."""
import ctypes
import math

import pytest
import torch

import paper_2608_03447_amd as asd
from paper_2608_03447_amd import decode


def vp(v):
    return None if v is None else ctypes.c_void_p(v)


CACHE = dict(keys=0x1000, values=0x2000, num_pages=10, page_stride=2048, token_stride=128,
             head_stride=64, page_table=0x3000, max_pages=4, page_size=16, num_heads=2, head_dim=64)


def paged(changes):
    c = dict(CACHE, **{k: v for k, v in changes.items() if k in CACHE})
    return decode._PagedCache(*[c[name] for name, _ in decode._PagedCache._fields_])


def append(**kw):
    a = dict(q=0x4000, k=0x5000, v=0x6000, dtype=1, qs=512, ks=512, vs=512, hq=4, qn=None, kn=None,
             eps=1e-6, freq=0x7000, rot=64, flags=0, pos=None, n=1, rows=2, lens=0x8000, offs=None,
             cl=0x9000, out=0xa000, os=256)
    a.update(kw)
    cache = paged(kw)
    return asd._load().asd_rope_append(
        vp(a["q"]), vp(a["k"]), vp(a["v"]), a["dtype"], a["qs"], a["ks"], a["vs"], a["hq"], vp(a["qn"]),
        vp(a["kn"]), a["eps"], vp(a["freq"]), a["rot"], a["flags"], vp(a["pos"]),
        None if kw.get("cache") == 0 else ctypes.byref(cache), a["n"], a["rows"], vp(a["lens"]),
        vp(a["offs"]), vp(a["cl"]), vp(a["out"]), a["os"], None)


def attend(**kw):
    a = dict(q=0x4000, dtype=1, qs=256, hq=4, scale=0.1, n=1, rows=2, lens=0x8000, offs=None,
             cl=0x9000, mask=None, words=0, out=0xa000, ws=None, wsb=0)
    a.update(kw)
    cache = paged(kw)
    return asd._load().asd_block_attention(
        vp(a["q"]), a["dtype"], a["qs"], a["hq"], a["scale"],
        None if kw.get("cache") == 0 else ctypes.byref(cache), a["n"], a["rows"], vp(a["lens"]),
        vp(a["offs"]), vp(a["cl"]), vp(a["mask"]), a["words"], vp(a["out"]), None, vp(a["ws"]),
        a["wsb"])


def sample(**kw):
    a = dict(z=0x1000, dtype=1, vocab=100, rows=2, stride=100, t=None, k=None, p=None, m=None,
             u=0x2000, tok=0x3000, prob=None, ws=None, wsb=0)
    a.update(kw)
    return asd._load().asd_sample(vp(a["z"]), a["dtype"], a["vocab"], a["rows"], a["stride"],
                                  vp(a["t"]), vp(a["k"]), vp(a["p"]), vp(a["m"]), vp(a["u"]),
                                  vp(a["tok"]), vp(a["prob"]), None, vp(a["ws"]), a["wsb"])


BAD_CACHE = [dict(cache=0), dict(keys=None), dict(values=None), dict(page_table=None),
             dict(keys=0x1008), dict(values=0x2002), dict(num_pages=0), dict(num_pages=1 << 31),
             dict(page_stride=-8), dict(token_stride=12), dict(head_stride=4), dict(max_pages=0),
             dict(page_size=0), dict(max_pages=1 << 20, page_size=1 << 11), dict(num_heads=0),
             dict(num_heads=4097), dict(page_stride=1 << 60), dict(head_dim=0)]
BAD_BATCH = [dict(n=-1), dict(n=3), dict(rows=1 << 31), dict(lens=None), dict(cl=None)]


@pytest.mark.parametrize("kw", BAD_CACHE + BAD_BATCH + [
    dict(head_dim=12), dict(head_dim=264), dict(hq=-1), dict(hq=4097), dict(q=None),
    dict(out=None), dict(hq=0), dict(q=None, out=None), dict(k=None), dict(v=None), dict(rot=66),
    dict(rot=7), dict(rot=-2), dict(freq=None), dict(flags=2), dict(eps=-1.0), dict(eps=math.nan),
    dict(eps=math.inf), dict(q=0x4008), dict(k=0x5004), dict(v=0x6002), dict(out=0xa008),
    dict(qn=0x7008), dict(kn=0x7004), dict(qs=100), dict(ks=100), dict(vs=-8), dict(qs=128),
    dict(ks=64), dict(os=8)])
def test_rope_append_refuses(kw):
    assert append(**kw) == 1


@pytest.mark.parametrize("kw", BAD_CACHE + BAD_BATCH + [
    dict(head_dim=96), dict(hq=0), dict(hq=3), dict(hq=65538), dict(scale=math.nan),
    dict(scale=math.inf), dict(mask=0x5000), dict(words=1), dict(mask=0x5000, words=-1),
    dict(mask=0x5004, words=1), dict(q=None), dict(out=None), dict(q=0x4008), dict(out=0xa004),
    dict(qs=100), dict(qs=128), dict(ws=0x10010, wsb=1 << 20)])
def test_block_attention_refuses(kw):
    assert attend(**kw) == 1


@pytest.mark.parametrize("kw", [
    dict(vocab=0), dict(vocab=1 << 30, stride=1 << 30), dict(rows=-1), dict(rows=1 << 31),
    dict(stride=99), dict(z=None), dict(u=None), dict(tok=None), dict(z=0x1001),
    dict(z=0x1002, dtype=0), dict(ws=0x10010, wsb=1 << 20), dict(stride=1 << 60)])
def test_sample_refuses(kw):
    assert sample(**kw) == 1


@pytest.mark.parametrize("dtype", [-1, 3, 7])
def test_unknown_types_are_refused(dtype):
    assert sample(dtype=dtype) == 2
    assert append(dtype=dtype) == 2 and append(dtype=0) == 2
    assert attend(dtype=dtype) == 2 and attend(dtype=0) == 2


def test_verifying_calls_still_refuse_binary16():
    assert asd._load().asd_workspace_bytes(asd.ASD_F16, 100, 1, 2) == 0


def test_empty_batches_are_no_ops():
    assert append(n=0, rows=0, k=None, keys=None, page_table=None) == 0
    assert attend(n=0, rows=0, q=None, keys=None, page_table=None) == 0
    assert sample(rows=0, z=None, u=None) == 0


def test_workspace_sizes_of_refused_shapes_are_zero():
    lib = asd._load()
    assert lib.asd_block_attention_workspace_bytes(4, 3, 64, 1, 2) == 0
    assert lib.asd_block_attention_workspace_bytes(4, 2, 96, 1, 2) == 0
    assert lib.asd_block_attention_workspace_bytes(4, 2, 64, 3, 2) == 0
    assert lib.asd_sample_workspace_bytes(9, 100, 1) == 0
    assert lib.asd_sample_workspace_bytes(1, 0, 1) == 0


def test_the_binding_refuses_host_tensors_and_wrong_layouts():
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    c = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    t = torch.zeros((1, 3), dtype=torch.int32)
    n = torch.zeros(1, dtype=torch.int64)
    k = torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        asd.asd_rope_append(x, x, x, c, c, t, n, k, None)
    with pytest.raises(ValueError, match="GPU"):
        asd.asd_block_attention(x, c, c, t, n, k)
    with pytest.raises(ValueError, match="GPU"):
        asd.asd_sample(torch.zeros(2, 10), torch.zeros(2))
    with pytest.raises(ValueError, match="same shape and strides"):
        decode._cache(c, c.transpose(0, 1).contiguous().transpose(0, 1), t, 1, torch.bfloat16,
                      torch.device("cpu"), 64)
    with pytest.raises(ValueError, match="page_table"):
        decode._cache(c, c, t.long(), 1, torch.bfloat16, torch.device("cpu"), 64)
    with pytest.raises(ValueError, match="dense"):
        wide = torch.zeros((3, 16, 2, 128), dtype=torch.bfloat16)[..., ::2]
        decode._cache(wide, wide, t, 1, torch.bfloat16, torch.device("cpu"), 64)
    with pytest.raises(ValueError, match="cache_lens"):
        decode._batch(k, None, None, torch.device("cpu"))
