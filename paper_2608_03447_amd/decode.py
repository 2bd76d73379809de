"""The operators of a decoding round around the verifier: a block's tokens enter
the paged cache (``asd_rope_append``), its rows attend to the cache
(``asd_block_attention``), and tokens are drawn from logit rows (``asd_sample``).

Like the rest of the binding these only marshal torch tensors and the current
HIP stream into the C calls of ``include/asd.h``, the ordinary arguments in
``_asd_binding``.
"""
import ctypes
import math

import torch

import paper_2608_03447_amd as _asd

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}


class _PagedCache(ctypes.Structure):
    """``asd_paged_cache`` of ``include/asd.h``."""

    _fields_ = [("keys", ctypes.c_void_p), ("values", ctypes.c_void_p),
                ("num_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("page_table", ctypes.c_void_p), ("max_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(dev):
    return torch.cuda.current_stream(dev.index).cuda_stream


def _heads(t, name, dtype=None, dev=None, rows=None, dim=None):
    """The row stride of [rows, heads, D] with dense heads (rows may be apart, as
    parts of one projection's rows are)."""
    if t.dim() != 3 or t.dtype not in _HALF or not t.is_cuda:
        raise ValueError("%s must be a 3-D bfloat16 or float16 tensor [rows, heads, D] on a GPU" % name)
    if (dtype is not None and t.dtype != dtype) or (dev is not None and t.device != dev):
        raise ValueError("%s must be a %s tensor on %s" % (name, dtype, dev))
    if (rows is not None and t.shape[0] != rows) or (dim is not None and t.shape[2] != dim):
        raise ValueError("%s must have %s rows of heads of %s elements" % (name, rows, dim))
    if t.numel() and ((t.shape[2] > 1 and t.stride(2) != 1)
                      or (t.shape[1] > 1 and t.stride(1) != t.shape[2])):
        raise ValueError("the heads of each row of %s must be dense" % name)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _cache(k_cache, v_cache, page_table, n, dtype, dev, dim):
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        if t.dim() != 4 or t.dtype != dtype or t.device != dev or t.shape[3] != dim:
            raise ValueError("%s must be a %s tensor [pages, page_size, heads, %d] on %s"
                             % (name, dtype, dim, dev))
        if t.numel() and dim > 1 and t.stride(3) != 1:
            raise ValueError("the elements of each head of %s must be dense" % name)
    if k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
        raise ValueError("k_cache and v_cache must have the same shape and strides")
    if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.shape[0] != n \
            or page_table.device != dev or not page_table.is_contiguous():
        raise ValueError("page_table must be a contiguous int32 (%d, pages) tensor on %s" % (n, dev))
    if page_table.shape[1] > 0x7fffffff or k_cache.shape[1] > 0x7fffffff:
        raise ValueError("page_table and pages must have fewer than 2^31 entries a row")
    pages, size, heads = k_cache.shape[:3]
    # a stride over one entry is never used; torch leaves it with any value
    steps = [s if c > 1 else 0 for s, c in zip(k_cache.stride()[:3], (pages, size, heads))]
    return _PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), pages, *steps, page_table.data_ptr(),
                       page_table.shape[1], size, heads, dim)


def _batch(block_lens, cache_lens, row_offsets, dev):
    if block_lens.dtype != torch.int32 or block_lens.dim() != 1 or block_lens.device != dev:
        raise ValueError("block_lens must be an int32 vector on %s" % dev)
    n = block_lens.shape[0]
    _asd._check_vector(cache_lens, n, torch.int64, dev, "cache_lens")
    if cache_lens is None:
        raise ValueError("cache_lens must be an int64 tensor of shape (%d,) on %s" % (n, dev))
    _asd._check_vector(row_offsets, n, torch.int64, dev, "row_offsets")
    return n


def _workspace(workspace, dev):
    if workspace is None:
        return None, 0
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError("workspace must be a contiguous uint8 tensor on %s" % dev)
    return workspace.data_ptr(), workspace.numel()


def asd_rope_append(q, k, v, k_cache, v_cache, page_table, cache_lens, block_lens, inv_freq, *,
                    q_norm=None, k_norm=None, eps=1e-6, positions=None, interleaved=False,
                    row_offsets=None, out_q=None):
    """Norm and rotate queries and keys, and append keys and values to the paged cache
    (``asd_rope_append`` of ``include/asd.h``).

    q, k, v      [total_rows, heads, D] bfloat16 or float16, the heads of a row dense (views of
                 one projection's rows will do); q may be None
    k_cache, v_cache  [pages, page_size, kv_heads, D], any strides with dense heads
    page_table   int32 [num_requests, max_pages]
    cache_lens   int64 [num_requests]: tokens in the cache before the block
    block_lens   int32 [num_requests] (K_i): request i has K_i + 1 rows
    inv_freq     float32 [rot_dim / 2], or None for no rotation
    q_norm, k_norm  [D] norm weights of q's type, or None for no norm
    positions    int64 [total_rows], or None: cache_lens[i] + p
    out_q        None or [total_rows, q_heads, D] with dense heads; may be q
    Returns the rotated queries (None without q); the cache is written in place.  Rows that no
    request owns are not written.
    """
    r = (_asd._fast or _asd._load_fast()).rope_append(
        k, q, v, k_cache, v_cache, page_table, cache_lens, block_lens, row_offsets, inv_freq, q_norm,
        k_norm, eps, positions, interleaved, out_q)
    if r is not None:
        return None if r is True else _asd._result(r, "asd_rope_append")
    if k.dim() != 3 or not k.is_cuda or k.dtype not in _HALF:
        raise ValueError("k must be a 3-D bfloat16 or float16 tensor [rows, heads, D] on a GPU")
    dev, dtype = k.device, k.dtype
    rows, heads, dim = k.shape
    k_stride = _heads(k, "k")
    v_stride = _heads(v, "v", dtype, dev, rows, dim)
    if v.shape[1] != heads or k_cache.dim() != 4 or k_cache.shape[2] != heads:
        raise ValueError("k, v and the caches must have the same number of heads")
    n = _batch(block_lens, cache_lens, row_offsets, dev)
    cache = _cache(k_cache, v_cache, page_table, n, dtype, dev, dim)
    q_heads = q_stride = out_stride = 0
    if q is not None:
        q_stride, q_heads = _heads(q, "q", dtype, dev, rows, dim), q.shape[1]
        if out_q is None:
            out_q = torch.empty((rows, q_heads, dim), dtype=dtype, device=dev)
        out_stride = _heads(out_q, "out_q", dtype, dev, rows, dim)
        if out_q.shape != q.shape:
            raise ValueError("out_q must have q's shape")
    elif out_q is not None:
        raise ValueError("out_q needs q")
    _asd._check_vector(q_norm, dim, dtype, dev, "q_norm")
    _asd._check_vector(k_norm, dim, dtype, dev, "k_norm")
    rot = 0
    if inv_freq is not None:
        _asd._check_vector(inv_freq, inv_freq.numel(), torch.float32, dev, "inv_freq")
        rot = 2 * inv_freq.numel()
        if rot > dim:
            raise ValueError("inv_freq must have at most D / 2 entries")
    _asd._check_vector(positions, rows, torch.int64, dev, "positions")
    block_lens = block_lens.contiguous()
    with _asd._on(dev):
        st = _asd._load().asd_rope_append(
            _ptr(q), k.data_ptr(), v.data_ptr(), _HALF[dtype], q_stride, k_stride, v_stride, q_heads,
            _ptr(q_norm), _ptr(k_norm), float(eps), _ptr(inv_freq), rot, 1 if interleaved else 0,
            _ptr(positions), ctypes.byref(cache), n, rows, block_lens.data_ptr(), _ptr(row_offsets),
            cache_lens.data_ptr(), _ptr(out_q), out_stride, _stream(dev))
    if st != 0:
        raise _asd.AsdError(st, "asd_rope_append")
    return out_q


def asd_block_attention(q, k_cache, v_cache, page_table, cache_lens, block_lens, *, scale=None,
                        mask=None, row_offsets=None, out=None, workspace=None):
    """Attention of draft blocks or trees over the paged cache, which holds the block's own
    tokens already (``asd_block_attention`` of ``include/asd.h``).

    q            [total_rows, q_heads, D] bfloat16 or float16, the heads of a row dense;
                 D 64, 128 or 256
    k_cache, v_cache, page_table, cache_lens, block_lens  as for :func:`asd_rope_append`
    scale        of the scores; None: 1 / sqrt(D)
    mask         int64 [total_rows, words]: bit j % 64 of word j // 64 lets the row see the
                 block's row j; None: row p sees rows 0..p (a chain of drafts)
    out          None or a contiguous tensor of q's shape
    workspace    None (library workspace) or a uint8 tensor as for :func:`asd_verify_ws`
    Returns out, [total_rows, q_heads, D]; rows that no request owns are not written.
    """
    r = (_asd._fast or _asd._load_fast()).block_attention(
        q, k_cache, v_cache, page_table, cache_lens, block_lens, row_offsets, scale, mask, out,
        workspace)
    if r is not None:
        return _asd._result(r, "asd_block_attention")
    stride = _heads(q, "q")
    dev, dtype = q.device, q.dtype
    rows, q_heads, dim = q.shape
    n = _batch(block_lens, cache_lens, row_offsets, dev)
    cache = _cache(k_cache, v_cache, page_table, n, dtype, dev, dim)
    words = 0
    if mask is not None:
        if mask.dtype != torch.int64 or mask.dim() != 2 or mask.shape[0] != rows \
                or mask.shape[1] < 1 or mask.device != dev or not mask.is_contiguous():
            raise ValueError("mask must be a contiguous int64 (%d, words) tensor on %s" % (rows, dev))
        words = mask.shape[1]
    if out is None:
        out = torch.empty((rows, q_heads, dim), dtype=dtype, device=dev)
    elif out.dtype != dtype or out.shape != q.shape or out.device != dev or not out.is_contiguous():
        raise ValueError("out must be a contiguous %s tensor of q's shape on %s" % (dtype, dev))
    space, space_bytes = _workspace(workspace, dev)
    block_lens = block_lens.contiguous()
    with _asd._on(dev):
        st = _asd._load().asd_block_attention(
            q.data_ptr(), _HALF[dtype], stride, q_heads,
            1.0 / math.sqrt(dim) if scale is None else float(scale), ctypes.byref(cache), n, rows,
            block_lens.data_ptr(), _ptr(row_offsets), cache_lens.data_ptr(), _ptr(mask), words,
            out.data_ptr(), _stream(dev), space, space_bytes)
    if st != 0:
        raise _asd.AsdError(st, "asd_block_attention")
    return out


def asd_block_attention_workspace_bytes(num_q_heads, num_kv_heads, head_dim, num_requests,
                                        total_rows):
    """Bytes of a ``workspace`` for :func:`asd_block_attention` on the current device."""
    return int(_asd._load().asd_block_attention_workspace_bytes(
        int(num_q_heads), int(num_kv_heads), int(head_dim), int(num_requests), int(total_rows)))


def asd_sample(logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None,
               out_token=None, out_prob=None, workspace=None):
    """Draw a token from every logit row by temperature, top-k, top-p and min-p
    (``asd_sample`` of ``include/asd.h``).

    logits       [rows, V] float32, bfloat16 or float16, rows dense (they may be apart)
    uniform      float32 [rows], uniform on [0, 1): the row's random number
    temperature, top_p, min_p  float or float32 [rows]; None: 1, 1 and 0
    top_k        int or int32 [rows]; None: all
    out_prob     None or float32 [rows]: takes the drawn token's share of the kept weights
    workspace    None (library workspace) or a uint8 tensor as for :func:`asd_verify_ws`
    Returns the tokens, int32 [rows].
    """
    r = (_asd._fast or _asd._load_fast()).sample(
        logits, uniform, temperature, top_k, top_p, min_p, out_token, out_prob, workspace)
    if r is not None:
        return _asd._result(r, "asd_sample")
    if logits.dim() != 2 or logits.dtype not in _DTYPES or not logits.is_cuda:
        raise ValueError("logits must be a 2-D float32, bfloat16 or float16 tensor on a GPU")
    rows, vocab = logits.shape
    if logits.numel() and ((vocab > 1 and logits.stride(1) != 1)
                           or (rows > 1 and logits.stride(0) < vocab)):
        raise ValueError("the rows of logits must be dense and must not overlap")
    dev = logits.device
    if uniform is None:
        raise ValueError("uniform must be a contiguous float32 tensor of shape (%d,) on %s" % (rows, dev))
    _asd._check_vector(uniform, rows, torch.float32, dev, "uniform")
    _asd._check_vector(out_token, rows, torch.int32, dev, "out_token")
    _asd._check_vector(out_prob, rows, torch.float32, dev, "out_prob")
    with _asd._on(dev):
        args = []
        for value, dtype, name in ((temperature, torch.float32, "temperature"),
                                   (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"),
                                   (min_p, torch.float32, "min_p")):
            args.append(None if value is None else
                        _asd._per_request(value, rows, dtype, dev, name))
        if out_token is None:
            out_token = torch.empty(rows, dtype=torch.int32, device=dev)
        space, space_bytes = _workspace(workspace, dev)
        st = _asd._load().asd_sample(
            logits.data_ptr(), _DTYPES[logits.dtype], vocab, rows,
            logits.stride(0) if rows > 1 else vocab, *[_ptr(t) for t in args], uniform.data_ptr(),
            out_token.data_ptr(), _ptr(out_prob), _stream(dev), space, space_bytes)
    del args
    if st != 0:
        raise _asd.AsdError(st, "asd_sample")
    return out_token


def asd_sample_workspace_bytes(dtype, vocab, rows):
    """Bytes of a ``workspace`` for :func:`asd_sample` on the current device."""
    code = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    return int(_asd._load().asd_sample_workspace_bytes(code, int(vocab), int(rows)))
