"""Python binding of ``include/kvx_attend.h``: operators on a replica's paged KV cache (argument marshalling only).

Every step runs in the HIP library that ``kvx`` binds (``libkvx.so``); caches are ``kvx.Cache`` handles, errors
``kvx.KvError``, ``stream`` a torch stream, a raw handle, or None for the current one.  The names are the C ABI's.

A batch of sequences is ``tables`` (int32 [B][pages]: block tables), ``lens`` (int32 [B]: tokens in the cache, the new
ones among them) and ``starts`` (int32 [B + 1]: where each sequence's new tokens start among all; None: one each).  All
three are device tensors; ``max_q`` and ``max_len`` are the host's bounds of new tokens and tokens per sequence, by
default (and at most) what the shapes allow.  Tight bounds size the launches better; numbers beyond them are refused on
the device (``kv_attend_async_error``), and such a sequence's rows of the outputs hold what they held before.

There is no backward pass: tensors that require a gradient are refused while torch records one.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from .kvx import Cache, KvCache, _in_use_on, _lib, _raise

KV_DTYPE_BF16 = 1
KV_DTYPE_F16 = 2
KV_DTYPE_E4M3 = 3
KV_DTYPE_F32 = 4
KV_ASYNC_BAD_BATCH = 2

_DTYPES = {torch.bfloat16: KV_DTYPE_BF16, torch.float16: KV_DTYPE_F16, torch.float8_e4m3fn: KV_DTYPE_E4M3}

EXPORTS = ("kv_append", "kv_append_scaled", "kv_rotate", "kv_attend", "kv_attend_workspace", "kv_attend_pages",
           "kv_attend_pages_workspace", "kv_bounds", "kv_score", "kv_keep", "kv_keep_workspace", "kv_compact",
           "kv_attend_async_error")


class KvRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class KvBatch(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("max_queries", ctypes.c_int32), ("num_queries", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("table_len", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("block_tables", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("starts", ctypes.c_void_p)]


class KvAttendOptions(ctypes.Structure):
    _fields_ = [("cache_dtype", ctypes.c_int32), ("window", ctypes.c_int32), ("scale", ctypes.c_float),
                ("softcap", ctypes.c_float), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float),
                ("slopes", ctypes.c_void_p), ("weights_in", ctypes.c_void_p), ("weights_out", ctypes.c_void_p),
                ("weights_seq_stride", ctypes.c_int64), ("weights_head_stride", ctypes.c_int64),
                ("full_weights", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class KvPageScales(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("block_stride", ctypes.c_int64), ("kv_stride", ctypes.c_int64)]


class KvPageList(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("budget", ctypes.c_int32)]


class KvRotateOptions(ctypes.Structure):
    _fields_ = [("cache_dtype", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("weight_dtype", ctypes.c_int32), ("freqs", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("weight_offset", ctypes.c_float), ("magnitude", ctypes.c_float), ("k_scale", ctypes.c_float),
                ("v_scale", ctypes.c_float), ("reserved", ctypes.c_int32), ("scales", ctypes.POINTER(KvPageScales))]


class KvScoreOptions(ctypes.Structure):
    _fields_ = [("cache_dtype", ctypes.c_int32), ("block_size", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("scales", ctypes.POINTER(KvPageScales)),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


def _declare(lib):
    P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    cache, batch, rows = ctypes.POINTER(KvCache), ctypes.POINTER(KvBatch), ctypes.POINTER(KvRows)
    options = ctypes.POINTER(KvAttendOptions)
    scales, pages = ctypes.POINTER(KvPageScales), ctypes.POINTER(KvPageList)
    for name, args, res in (
            ("kv_append", [cache, i32, batch, rows, rows, i32, f32, f32, P], i32),
            ("kv_append_scaled", [cache, i32, batch, rows, rows, scales, P], i32),
            ("kv_rotate", [cache, i32, batch, ctypes.POINTER(KvRotateOptions), rows, rows, rows, rows, P], i32),
            ("kv_attend", [cache, i32, batch, options, rows, rows, P, P, i64, P], i32),
            ("kv_attend_workspace", [cache, batch, options, rows], i64),
            ("kv_attend_pages", [cache, i32, batch, options, scales, pages, rows, rows, P, P, i64, P], i32),
            ("kv_attend_pages_workspace", [cache, batch, options, scales, pages, rows], i64),
            ("kv_bounds", [cache, i32, batch, i32, cache, P], i32),
            ("kv_score", [cache, i32, batch, ctypes.POINTER(KvScoreOptions), rows, P, P, P], i32),
            ("kv_keep", [P, i64, i64, P, i32, i32, i32, i32, i32, i32, P, P, P, P, i64, P], i32),
            ("kv_keep_workspace", [i32, i32, i32, i32], i64),
            ("kv_compact", [cache, i32, i32, P, i64, i32, P, i32, i32, P, P, i64, i32, P], i32),
            ("kv_attend_async_error", [ctypes.c_int], i32)):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res


_declare(_lib)


# A decoding step makes a call per layer, and short calls are bound by this module: checks read each property once, and
# what only the numbers decide is remembered by them.


def _ints(t, name: str, dims: int, device: int, rows=None):
    """A tensor of int32 on the call's device whose last dimension is dense."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.dim() != dims or \
            (t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel()):
        raise TypeError(f"{name} must be a {dims}-dimensional int32 device tensor with a dense last dimension")
    if t.get_device() != device:
        _elsewhere(t, name, device)
    if rows is not None and t.shape[0] != rows:
        raise ValueError(f"{name} has {t.shape[0]} rows; {rows} are needed")
    return t


def _elsewhere(t, name: str, device: int) -> None:
    raise TypeError(f"{name} must be a device tensor on device {device}, where the call works (it is on {t.device})")


def _on(t, name: str, device: int) -> None:
    if t.get_device() != device:
        _elsewhere(t, name, device)


def _floats(t, name: str, device: int, shape) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous float32 device tensor of {tuple(shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        _no_gradient(name)
    _on(t, name, device)


def _weights(t, name: str, device: int, rows=None) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.dim() != 3 or \
            (t.stride(2) != 1 and t.shape[2] > 1 and t.numel()) or (rows is not None and t.shape[:2] != rows):
        raise TypeError(f"{name} must be a [sequences][heads][tokens] float32 device tensor with dense rows"
                        f"{'' if rows is None else f' ({rows} of them)'}")
    if t.requires_grad and torch.is_grad_enabled():
        _no_gradient(name)
    _on(t, name, device)


def _no_gradient(name: str):
    raise RuntimeError(f"{name} requires a gradient, and these operators have none: detach it, or call under "
                       "torch.no_grad()")


def _rows(t, name: str, head_dim: int, device: int) -> KvRows:
    if not isinstance(t, torch.Tensor) or len(shape := t.shape) != 3 or \
            (dtype := t.dtype) not in (torch.bfloat16, torch.float16):
        raise TypeError(f"{name} must be a [tokens][heads][D] device tensor of bfloat16 or float16")
    if t.requires_grad and torch.is_grad_enabled():
        _no_gradient(name)
    if t.get_device() != device:
        _elsewhere(t, name, device)
    _, heads, width = shape
    token, head, column = t.stride()
    if width != head_dim or (column != 1 and t.numel()):
        raise ValueError(f"{name}: rows of {width} elements {column} apart; dense rows of {head_dim} are needed")
    return KvRows(t.data_ptr(), token, head, heads, _DTYPES[dtype])


def _factor(x, name: str) -> float:
    """A factor that the caller named; the ABI takes 0 in 32 bits for its default, which is not what 0 means here."""
    if -2.0**-150 <= x <= 2.0**-150:
        raise ValueError(f"{name} must be above 0 in 32 bits (got {x})")
    return float(x)


def _int32(x, name: str) -> int:
    """ctypes would cut a longer number to its low 32 bits."""
    if not -2**31 <= x < 2**31:
        raise ValueError(f"{name} must fit 32 bits (got {x})")
    return int(x)


def _batch(cache: Cache, tables, lens, starts, tokens: int, max_q, max_len) -> KvBatch:
    device = cache.struct.device
    B, pages = _ints(tables, "tables", 2, device).shape
    if tokens >= 2**31:
        _int32(tokens, "the number of new tokens")
    _ints(lens, "lens", 1, device, B)
    if starts is None:
        if tokens != B:
            raise ValueError(f"{tokens} new tokens for {B} sequences of one each: starts is needed")
        max_q, starts_at = 1, None
    else:
        starts_at = _ints(starts, "starts", 1, device, B + 1).data_ptr()
        max_q = max(1, tokens if max_q is None else min(tokens, int(max_q)))
    most = min(pages * cache.layout.block_size, 2**31 - 1024)
    if max_len is not None:
        most = min(most, max(int(max_len), -1))
    return KvBatch(B, max_q, tokens, most, pages, 0, tables.stride(0), tables.data_ptr(), lens.data_ptr(), starts_at)


def _cache_dtype(cache: Cache, dtype, rows) -> int:
    """KV_DTYPE of the cache: ``dtype``, or by its element size the rows' type or e4m3."""
    if dtype is None:
        dtype = torch.float8_e4m3fn if cache.layout.elem_bytes == 1 else rows.dtype
    if dtype not in _DTYPES:
        raise TypeError(f"caches are bfloat16, float16 or float8_e4m3fn, not {dtype}")
    return _DTYPES[dtype]


def _call_stream(stream):
    """(the stream's handle, the context in which the call's own tensors are made): they belong to the call's stream,
    which may be another than the current one."""
    if stream is None:
        return torch.cuda.current_stream(torch.cuda.current_device()).cuda_stream, _HERE
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    return stream.cuda_stream, torch.cuda.stream(stream)


_HERE = contextlib.nullcontext()


def _used(stream, *tensors) -> None:
    """Tensors used on a stream that was named: as with a store's block table, torch must not hand their memory out again
    before the call's work is done there.  (With no stream named the call is like torch's own on the current stream.)"""
    if stream is not None:
        for t in tensors:
            if t is not None:
                _in_use_on(t, stream)


def _page_scales(t, cache: Cache, device: int) -> KvPageScales:
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.uint8, torch.float8_e8m0fnu) or t.dim() != 3:
        raise TypeError("scales must be a [blocks][2][heads] uint8 or float8_e8m0fnu device tensor")
    _on(t, "scales", device)
    blocks, two, heads = t.shape
    if two != 2 or heads != cache.layout.num_kv_heads or blocks < cache.struct.num_blocks:
        raise ValueError(f"scales of {tuple(t.shape)} for a cache of {cache.struct.num_blocks} blocks of "
                         f"{cache.layout.num_kv_heads} heads")
    block, kv, head = t.stride()
    if head != 1 and heads > 1:
        raise TypeError("scales must have a dense last dimension")
    # (Strides over a single block lead nowhere.)
    return KvPageScales(t.data_ptr(), block if blocks > 1 else max(block, kv + heads), kv)


def kv_append(cache: Cache, layer: int, k, v, tables, lens, starts=None, *, max_q=None, max_len=None, dtype=None,
              k_scale: float = 1.0, v_scale: float = 1.0, scales=None, stream=None) -> None:
    """Write the new tokens' rows ``k`` and ``v`` ([tokens][H][D], token and head strides of whole 16 bytes) into layer
    ``layer``.

    ``dtype``: the cache's; by default that of ``k``, or float8_e4m3fn in a cache of 1-byte elements, where x is stored
    as e4m3(x / scale).  ``scales``: kv_append_scaled.
    """
    if scales is not None:
        if k_scale != 1.0 or v_scale != 1.0:
            raise ValueError("k_scale and v_scale beside scales of pages")
        if dtype not in (None, torch.float8_e4m3fn):
            raise TypeError(f"scales of pages for a cache of {dtype}")
        return kv_append_scaled(cache, layer, k, v, tables, lens, scales, starts, max_q=max_q, max_len=max_len,
                                stream=stream)
    D = cache.layout.head_dim
    device = cache.struct.device
    kr, vr = _rows(k, "k", D, device), _rows(v, "v", D, device)
    if k.shape != v.shape:
        raise ValueError(f"k and v differ in shape: {tuple(k.shape)} and {tuple(v.shape)}")
    batch = _batch(cache, tables, lens, starts, k.shape[0], max_q, max_len)
    handle, _ = _call_stream(stream)
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    else:
        k_scale = v_scale = 1.0
    _raise(_lib.kv_append(ctypes.byref(cache.struct), _int32(layer, "layer"), ctypes.byref(batch), ctypes.byref(kr),
                          ctypes.byref(vr), _cache_dtype(cache, dtype, k), k_scale, v_scale, handle))
    _used(stream, k, v, tables, lens, starts)


def kv_append_scaled(cache: Cache, layer: int, k, v, tables, lens, scales, starts=None, *, max_q=None, max_len=None,
                     stream=None) -> None:
    """kv_append into a float8_e4m3fn cache whose pages have ``scales`` (float8_e8m0fnu, or its bytes as uint8,
    [blocks][2][H]: K's and V's of each head): the new rows' pages take the smallest power of two that brings them, and what a
    page already held, to 448 or less."""
    D = cache.layout.head_dim
    device = cache.struct.device
    kr, vr = _rows(k, "k", D, device), _rows(v, "v", D, device)
    if k.shape != v.shape:
        raise ValueError(f"k and v differ in shape: {tuple(k.shape)} and {tuple(v.shape)}")
    batch = _batch(cache, tables, lens, starts, k.shape[0], max_q, max_len)
    by = _page_scales(scales, cache, device)
    handle, _ = _call_stream(stream)
    _raise(_lib.kv_append_scaled(ctypes.byref(cache.struct), _int32(layer, "layer"), ctypes.byref(batch),
                                 ctypes.byref(kr), ctypes.byref(vr), ctypes.byref(by), handle))
    _used(stream, k, v, tables, lens, starts, scales)


def kv_rotate(cache: Cache, layer: int, q, k, v, tables, lens, starts=None, *, freqs=None, positions=None, q_weight=None,
              k_weight=None, eps: float = 1e-6, weight_offset: float = 0.0, interleaved: bool = False,
              magnitude: float = 1.0, max_q=None, max_len=None, dtype=None, k_scale: float = 1.0, v_scale: float = 1.0,
              scales=None, out=None, stream=None):
    """Norm the new tokens' ``q`` and ``k`` for each head, rotate them by their position, and append K and V to layer
    ``layer``; returns the rotated queries.

    ``q_weight``, ``k_weight`` ([D], float32 or the rows' type; None: no norm): x / sqrt(mean x^2 + eps) * (weight_offset +
    weight).  ``freqs`` (float64 [n], None: no rotation): radians per position of the pairs (i, i + n) of a row's first 2n
    columns, or (2i, 2i + 1) if ``interleaved``; cosine and sine are multiplied by ``magnitude``.  ``positions`` (int32
    [tokens]): by default each token's place in its sequence.  ``dtype``, ``k_scale``, ``v_scale`` and ``scales`` are
    kv_append's.  ``out`` (like ``q``) is made if not given, and may be ``q`` itself; rows of no sequence are left as they
    were."""
    D = cache.layout.head_dim
    device = cache.struct.device
    qr, kr, vr = _rows(q, "q", D, device), _rows(k, "k", D, device), _rows(v, "v", D, device)
    if k.shape != v.shape or q.shape[0] != k.shape[0]:
        raise ValueError(f"q, k and v differ in shape: {tuple(q.shape)}, {tuple(k.shape)} and {tuple(v.shape)}")
    batch = _batch(cache, tables, lens, starts, q.shape[0], max_q, max_len)
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    options = KvRotateOptions(_cache_dtype(cache, dtype, k), eps=float(eps), weight_offset=float(weight_offset),
                              interleaved=1 if interleaved else 0, magnitude=_factor(magnitude, "magnitude"),
                              k_scale=k_scale, v_scale=v_scale)
    if freqs is not None:
        if not isinstance(freqs, torch.Tensor) or freqs.dtype is not torch.float64 or freqs.dim() != 1 or \
                not freqs.is_contiguous():
            raise TypeError("freqs must be a contiguous 1-dimensional float64 device tensor")
        if freqs.requires_grad and torch.is_grad_enabled():
            _no_gradient("freqs")
        _on(freqs, "freqs", device)
        options.rotary_dim, options.freqs = _int32(2 * freqs.shape[0], "twice the number of freqs"), freqs.data_ptr()
    if positions is not None:
        if not _ints(positions, "positions", 1, device, q.shape[0]).is_contiguous():
            raise TypeError("positions must be contiguous")
        options.positions = positions.data_ptr()
    for weight, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if weight is None:
            continue
        if not isinstance(weight, torch.Tensor) or weight.shape != (D,) or not weight.is_contiguous() or \
                weight.dtype not in (torch.float32, q.dtype):
            raise TypeError(f"{name} must be a contiguous [{D}] device tensor of float32 or {q.dtype}")
        if weight.requires_grad and torch.is_grad_enabled():
            _no_gradient(name)
        _on(weight, name, device)
        setattr(options, name, weight.data_ptr())
        options.weight_dtype = KV_DTYPE_F32 if weight.dtype is torch.float32 else _DTYPES[weight.dtype]
    if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
        raise TypeError("q_weight and k_weight have different types")
    if scales is not None:
        by = _page_scales(scales, cache, device)
        options.scales = ctypes.pointer(by)
    if out is not None and (out.dtype != q.dtype or out.shape != q.shape):
        raise TypeError("out must have the type and shape of q")
    handle, here = _call_stream(stream)
    if out is None:
        with here:
            out = q.new_empty(q.shape)
    outr = _rows(out, "out", D, device)
    _raise(_lib.kv_rotate(ctypes.byref(cache.struct), _int32(layer, "layer"), ctypes.byref(batch), ctypes.byref(options),
                          ctypes.byref(qr), ctypes.byref(outr), ctypes.byref(kr), ctypes.byref(vr), handle))
    _used(stream, q, k, v, tables, lens, starts, freqs, positions, q_weight, k_weight, scales, out)
    return out


def kv_attend(cache: Cache, layer: int, q, tables, lens, starts=None, *, max_q=None, max_len=None, dtype=None,
              scale=None, softcap: float = 0.0, window: int = 0, slopes=None, k_scale: float = 1.0, v_scale: float = 1.0,
              weights=None, prior=None, full_weights: bool = False, scales=None, pages=None, counts=None, out=None,
              lse=None, stream=None):
    """Attention of the new tokens' queries ``q`` ([tokens][query heads][D], token and head strides of whole 16 bytes)
    over layer ``layer``; returns (out, lse).

    ``weights`` (float32 [B][H][>= max_len]): receives ``prior`` (same shape and strides; None: 0) plus what each cached
    token got in this call; ``prior=weights`` accumulates in place.  ``full_weights``: sequences of more than 64 rows
    (new tokens times query heads) per KV head take exp(s) to V as two numbers of q's type, as shorter ones always do,
    for up to 1.3 times the time; then the output's rounding alone shows.  ``out`` (like ``q``) and ``lse`` (float32
    [tokens][query heads]) are made if not given, and overlap no input; rows that belong to no sequence are left as
    they were.

    ``scales``: those of a float8_e4m3fn cache's pages, as kv_append_scaled leaves them.  ``pages`` (int32 [tokens][H or 1]
    [budget], dense rows) and ``counts`` (int32 [tokens]): each new token attends over the first ``counts`` of its
    ``pages`` alone, which are places in its sequence's table, as kv_keep chooses them from kv_score's scores.  Neither
    goes with ``weights``.
    """
    device = cache.struct.device
    qr = _rows(q, "q", cache.layout.head_dim, device)
    batch = _batch(cache, tables, lens, starts, q.shape[0], max_q, max_len)
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    else:
        k_scale = v_scale = 1.0
    options = KvAttendOptions(_cache_dtype(cache, dtype, q), _int32(window, "window") if window else 0,
                              0.0 if scale is None else _factor(scale, "scale"),
                              _factor(softcap, "softcap") if softcap else 0.0, k_scale, v_scale)
    if full_weights:
        options.full_weights = 1
    if slopes is not None:
        _floats(slopes, "slopes", device, (q.shape[1],))
        options.slopes = slopes.data_ptr()
    if weights is not None:
        _weights(weights, "weights", device, (tables.shape[0], cache.layout.num_kv_heads))
        if max_len is None:
            batch.max_len = min(batch.max_len, weights.shape[2])
        elif weights.shape[2] < batch.max_len:
            raise ValueError(f"weights of {weights.shape[2]} tokens for sequences of up to {batch.max_len}")
        options.weights_out = weights.data_ptr()
        options.weights_seq_stride, options.weights_head_stride = weights.stride(0), weights.stride(1)
        if prior is not None:
            _weights(prior, "prior", device)
            if prior.shape != weights.shape or prior.stride() != weights.stride():
                raise TypeError("prior must have the shape and strides of weights")
            options.weights_in = prior.data_ptr()
    elif prior is not None:
        raise ValueError("prior without weights")
    by = chosen = None
    if scales is not None:
        by = ctypes.byref(_page_scales(scales, cache, device))
    if pages is not None:
        chosen = ctypes.byref(_page_list(pages, counts, cache, q.shape[0], device))
    elif counts is not None:
        raise ValueError("counts without pages")
    heads = (q.shape[0], q.shape[1])
    if out is not None and (out is q or out.dtype != q.dtype or out.shape != q.shape):
        raise TypeError("out must have the type and shape of q, and be another tensor")
    if lse is not None:
        _floats(lse, "lse", device, heads)
    layout = cache.layout
    key = (layout.num_kv_heads, layout.head_dim, layout.elem_bytes, layout.block_size, batch.num_seqs, batch.max_queries,
           batch.num_queries, batch.max_len, options.window, weights is None, q.shape[1],
           -1 if pages is None else pages.shape[2])
    need = _attend_bytes.get(key)
    if need is None:
        args = (ctypes.byref(cache.struct), ctypes.byref(batch), ctypes.byref(options))
        need = _lib.kv_attend_workspace(*args, ctypes.byref(qr)) if by is None and chosen is None else \
            _lib.kv_attend_pages_workspace(*args, by, chosen, ctypes.byref(qr))
        if need < 0:
            _raise(need)
        if len(_attend_bytes) >= 4096:
            _attend_bytes.clear()
        _attend_bytes[key] = need
    handle, here = _call_stream(stream)
    with here:
        if out is None:
            out = q.new_empty(q.shape)
        if lse is None:
            lse = torch.empty(heads, dtype=torch.float32, device=q.device)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    outr = _rows(out, "out", layout.head_dim, device)
    args = (ctypes.byref(cache.struct), _int32(layer, "layer"), ctypes.byref(batch), ctypes.byref(options))
    more = (ctypes.byref(qr), ctypes.byref(outr), lse.data_ptr(), workspace.data_ptr() if need else None, need, handle)
    if by is None and chosen is None:
        _raise(_lib.kv_attend(*args, *more))
    else:
        _raise(_lib.kv_attend_pages(*args, by, chosen, *more))
    _used(stream, q, tables, lens, starts, slopes, weights, prior, out, lse, scales, pages, counts)
    return out, lse


def kv_attend_pages(cache: Cache, layer: int, q, tables, lens, starts=None, *, scales=None, pages=None, counts=None,
                    **options):
    """kv_attend with ``scales`` of pages, or over chosen ``pages``, or both."""
    if scales is None and pages is None:
        raise ValueError("neither scales nor pages")
    return kv_attend(cache, layer, q, tables, lens, starts, scales=scales, pages=pages, counts=counts, **options)


def _page_list(pages, counts, cache: Cache, tokens: int, device: int) -> KvPageList:
    _ints(pages, "pages", 3, device, tokens)
    if counts is None:
        raise ValueError("pages without counts")
    if not _ints(counts, "counts", 1, device, tokens).is_contiguous():
        raise TypeError("counts must be contiguous")
    _, heads, budget = pages.shape
    return KvPageList(pages.data_ptr(), counts.data_ptr(), pages.stride(0), pages.stride(1), heads, budget)


_attend_bytes = {}  # kv_attend_workspace by the numbers that it depends on


def kv_bounds(cache: Cache, layer: int, bounds: Cache, tables, lens, starts=None, *, max_q=None, max_len=None, dtype=None,
              stream=None) -> None:
    """For the pages of layer ``layer`` that new tokens lie in: the lowest and the highest stored K of every column over
    the page's tokens, into the same block of ``bounds``, a cache of the same heads, head_dim and element size with one token
    a block (lowest as K, highest as V).  Without ``starts`` each sequence has one new token; for a restored prefix, name as
    many rows as it has tokens.

    ``dtype``: the cache's, which 2-byte elements alone do not say."""
    device = cache.struct.device
    if starts is None:
        rows, starts_at = tables.shape[0] if isinstance(tables, torch.Tensor) and tables.dim() else 0, None
    else:
        # (How many rows there are only the device knows: as many as sequences may have tokens.)
        rows, starts_at = 2**31 - 1, starts
        if max_q is None:
            max_q = 2**31 - 1
    batch = _batch(cache, tables, lens, starts_at, rows, max_q, max_len)
    if dtype is None:
        if cache.layout.elem_bytes != 1:
            raise TypeError("dtype is needed: bfloat16 or float16")
        dtype = torch.float8_e4m3fn
    handle, _ = _call_stream(stream)
    _raise(_lib.kv_bounds(ctypes.byref(cache.struct), _int32(layer, "layer"), ctypes.byref(batch),
                          _cache_dtype(cache, dtype, None), ctypes.byref(bounds.struct), handle))
    _used(stream, tables, lens, starts)


def kv_score(bounds: Cache, layer: int, q, tables, lens, starts=None, *, block_size: int, max_q=None, max_len=None,
             dtype=None, scale: float = 1.0, scales=None, out=None, counts=None, stream=None):
    """What no token of a page can exceed in scale * (q . k): for each new token, KV head and page up to the token's own the
    largest over the head's queries ``q`` ([tokens][query heads][D]) of q's positive part times the page's highest K and its
    negative part times the lowest, from kv_bounds's ``bounds`` of pages of ``block_size`` tokens.

    Returns (scores float32 [tokens][H][pages], counts int32 [tokens]: pages up to the token's own), which are kv_keep's
    weights and lens.  ``out`` and ``counts`` are made if not given; scores of pages beyond ``counts``, and rows of no
    sequence, are left as they were (in made ones, scores hold anything and counts 0)."""
    device = bounds.struct.device
    qr = _rows(q, "q", bounds.layout.head_dim, device)
    block_size = _int32(block_size, "block_size")
    batch = _batch(bounds, tables, lens, starts, q.shape[0], max_q, None)
    most = min(tables.shape[1] * block_size, 2**31 - 1024)
    batch.max_len = most if max_len is None else min(most, max(int(max_len), -1))
    heads = bounds.layout.num_kv_heads
    pages = -(-max(batch.max_len, 0) // block_size) if block_size > 0 else 0
    handle, here = _call_stream(stream)
    with here:
        if out is None:
            out = torch.empty((q.shape[0], heads, pages), dtype=torch.float32, device=q.device)
        if counts is None:
            counts = torch.empty(q.shape[0], dtype=torch.int32, device=q.device) if starts is None else \
                torch.zeros(q.shape[0], dtype=torch.int32, device=q.device)
    _weights(out, "out", device, (q.shape[0], heads))
    if out.shape[2] < pages:
        raise ValueError(f"out of {out.shape[2]} pages for sequences of up to {pages}")
    if not _ints(counts, "counts", 1, device, q.shape[0]).is_contiguous():
        raise TypeError("counts must be contiguous")
    options = KvScoreOptions(_cache_dtype(bounds, dtype, q), block_size, _factor(scale, "scale"))
    options.token_stride, options.head_stride = out.stride(0), out.stride(1)
    if scales is not None:
        by = _page_scales(scales, bounds, device)
        options.scales = ctypes.pointer(by)
    _raise(_lib.kv_score(ctypes.byref(bounds.struct), _int32(layer, "layer"), ctypes.byref(batch), ctypes.byref(options),
                         ctypes.byref(qr), out.data_ptr(), counts.data_ptr(), handle))
    _used(stream, q, tables, lens, starts, scales, out, counts)
    return out, counts


def kv_keep(weights, lens, budget: int, *, sinks: int = 0, recent: int = 0, max_len=None, stream=None):
    """The tokens that each sequence keeps under ``budget``: its first ``sinks``, its last ``recent`` and the heaviest
    others by ``weights`` (float32 [B][H or 1][tokens], dense rows).  Returns (keep int32 [B][H][budget], ascending and
    then -1; kept_lens int32 [B]; kept_weights float32 like keep, then 0)."""
    device = torch.cuda.current_device() if torch.cuda.is_available() else -2
    _weights(weights, "weights", device)
    B, H, L = weights.shape
    _ints(lens, "lens", 1, device, B)
    if max_len is not None and int(max_len) > L:
        raise ValueError(f"weights of {L} tokens for sequences of up to {max_len}")
    budget, sinks, recent = _int32(budget, "budget"), _int32(sinks, "sinks"), _int32(recent, "recent")
    if budget < 1:
        raise ValueError(f"budget must be positive (got {budget})")
    most = _int32(L if max_len is None else max_len, "max_len")
    need = _lib.kv_keep_workspace(B, H, most, budget)
    if need < 0:
        _raise(need)
    handle, here = _call_stream(stream)
    with here:
        workspace = torch.empty(need, dtype=torch.uint8, device=weights.device) if need else None
        keep = torch.empty((B, H, budget), dtype=torch.int32, device=weights.device)
        kept_lens = torch.empty(B, dtype=torch.int32, device=weights.device)
        kept_weights = torch.empty((B, H, budget), dtype=torch.float32, device=weights.device)
    _raise(_lib.kv_keep(weights.data_ptr(), weights.stride(0), weights.stride(1), lens.data_ptr(), B, H,
                        most, budget, sinks, recent, keep.data_ptr(), kept_lens.data_ptr(),
                        kept_weights.data_ptr(), workspace.data_ptr() if need else None, need, handle))
    _used(stream, weights, lens)
    return keep, kept_lens, kept_weights


def kv_compact(cache: Cache, layer: int, tables, keep, kept_lens, dst_tables, *, stream=None) -> None:
    """Copy the kept tokens' rows of layer ``layer`` into the pages of ``dst_tables``: token ``keep[b][h][j]`` becomes
    token j (``keep`` int32 [B][H or 1][budget], contiguous; ``kept_lens`` int32 [B] of them count).  The destination's
    pages are distinct and none of the sources'.  ``window`` and ``slopes`` of later calls count in the new places."""
    device = cache.struct.device
    B = _ints(tables, "tables", 2, device).shape[0]
    if not _ints(keep, "keep", 3, device, B).is_contiguous():
        raise TypeError("keep must be contiguous")
    _ints(kept_lens, "kept_lens", 1, device, B)
    _ints(dst_tables, "dst_tables", 2, device, B)
    handle, _ = _call_stream(stream)
    _raise(_lib.kv_compact(ctypes.byref(cache.struct), _int32(layer, "layer"), B, tables.data_ptr(), tables.stride(0),
                           tables.shape[1], keep.data_ptr(), keep.shape[1], keep.shape[2], kept_lens.data_ptr(),
                           dst_tables.data_ptr(), dst_tables.stride(0), dst_tables.shape[1], handle))
    _used(stream, tables, keep, kept_lens, dst_tables)


def kv_attend_async_error(clear: bool = False) -> int:
    """Device-side faults of these operators on the current device since the last clear (KV_ASYNC_* bits)."""
    mask = int(_lib.kv_attend_async_error(1 if clear else 0))
    if mask < 0:
        _raise(mask)
    return mask
