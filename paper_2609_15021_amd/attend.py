"""Python binding of ``include/kvx_attend.h``: operators on a replica's paged KV cache (argument marshalling only).

Every step runs in the HIP library that ``kvx`` binds (``libkvx.so``); caches are ``kvx.Cache`` handles, errors
``kvx.KvError``, ``stream`` a torch stream, a raw handle, or None for the current one.  The names are the C ABI's.

A batch of sequences is ``tables`` (int32 [B][pages]: block tables), ``lens`` (int32 [B]: tokens in the cache, the new
ones among them) and ``starts`` (int32 [B + 1]: where each sequence's new tokens start among all; None: one each).  All
three are device tensors; ``max_q`` and ``max_len`` are the host's bounds of new tokens and tokens per sequence, by
default (and at most) what the shapes allow.  Tight bounds size the launches better; numbers beyond them are refused on
the device (``kv_attend_async_error``), and such a sequence's rows of the outputs hold what they held before.

There is no backward pass: tensors that require a gradient are refused while torch records one, and those that carry a
forward-mode tangent always.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct

import torch
from torch.autograd import forward_ad

from .kvx import Cache, KvCache, _in_use_on, _lib, _raise

try:
    from . import _tensors
except ImportError as e:
    raise ImportError("the binding's module _tensors is not built; run __graft_entry__.build()") from e

KV_DTYPE_BF16 = 1
KV_DTYPE_F16 = 2
KV_DTYPE_E4M3 = 3
KV_DTYPE_F32 = 4
KV_ASYNC_BAD_BATCH = 2

_ROW_TYPES = {torch.bfloat16: KV_DTYPE_BF16, torch.float16: KV_DTYPE_F16}
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


# The same structures as bytes, which take a third of the time to make; a call reads them before it returns.
_pack_rows = struct.Struct("qqqii").pack
_pack_batch = struct.Struct("iiiiiiqqqq").pack
_pack_attend = struct.Struct("iiffffqqqqqii").pack
_pack_scales = struct.Struct("qqq").pack
_pack_list = struct.Struct("qqqqii").pack
_pack_rotate = struct.Struct("iiiiqqqqfffffiP").pack
_pack_score = struct.Struct("iifiPqq").pack


def _declare(lib):
    P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    # Structures: a pointer, or bytes.
    cache, batch, rows, options, scales, pages = ctypes.POINTER(KvCache), P, P, P, P, P
    for name, args, res in (
            ("kv_append", [cache, i32, batch, rows, rows, i32, f32, f32, P], i32),
            ("kv_append_scaled", [cache, i32, batch, rows, rows, scales, P], i32),
            ("kv_rotate", [cache, i32, batch, options, rows, rows, rows, rows, P], i32),
            ("kv_attend", [cache, i32, batch, options, rows, rows, P, P, i64, P], i32),
            ("kv_attend_workspace", [cache, batch, options, rows], i64),
            ("kv_attend_pages", [cache, i32, batch, options, scales, pages, rows, rows, P, P, i64, P], i32),
            ("kv_attend_pages_workspace", [cache, batch, options, scales, pages, rows], i64),
            ("kv_bounds", [cache, i32, batch, i32, cache, P], i32),
            ("kv_score", [cache, i32, batch, options, rows, P, P, P], i32),
            ("kv_keep", [P, i64, i64, P, i32, i32, i32, i32, i32, i32, P, P, P, P, i64, P], i32),
            ("kv_keep_workspace", [i32, i32, i32, i32], i64),
            ("kv_compact", [cache, i32, i32, P, i64, i32, P, i32, i32, P, P, i64, i32, P], i32),
            ("kv_attend_async_error", [ctypes.c_int], i32)):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res


_declare(_lib)


# A decoding step makes a call per layer, and short calls are bound by this module: a tensor that is as it should be is
# looked at by _tensors, in one call; where that answers None, the checks here say what is wrong.  What only the numbers
# decide is remembered by them.


def _ints(t, name: str, dims: int, device: int, rows=None):
    """A tensor of int32 on the call's device whose last dimension is dense: its shape and strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or len(shape := t.shape) != dims or \
            ((strides := t.stride())[-1] != 1 and shape[-1] > 1 and t.numel()):
        raise TypeError(f"{name} must be a {dims}-dimensional int32 device tensor with a dense last dimension")
    if t.get_device() != device:
        _elsewhere(t, name, device)
    if rows is not None and shape[0] != rows:
        raise ValueError(f"{name} has {shape[0]} rows; {rows} are needed")
    return shape, strides


def _dense_ints(t, name: str, dims: int, device: int, rows: int) -> int:
    """The address of a contiguous one."""
    at = _tensors.ints(t, dims, device, rows)
    if at is not None:
        return at
    _ints(t, name, dims, device, rows)
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _elsewhere(t, name: str, device: int) -> None:
    raise TypeError(f"{name} must be a device tensor on device {device}, where the call works (it is on {t.device})")


def _on(t, name: str, device: int) -> None:
    if t.get_device() != device:
        _elsewhere(t, name, device)


def _floats(t, name: str, device: int, shape) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous float32 device tensor of {tuple(shape)}")
    _plain(t, name)
    _on(t, name, device)


def _weights(t, name: str, device: int, rows=None) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.dim() != 3 or \
            (t.stride(2) != 1 and t.shape[2] > 1 and t.numel()) or (rows is not None and t.shape[:2] != rows):
        raise TypeError(f"{name} must be a [sequences][heads][tokens] float32 device tensor with dense rows"
                        f"{'' if rows is None else f' ({rows} of them)'}")
    _plain(t, name)
    _on(t, name, device)


def _plain(t, name: str) -> None:
    """These operators have no derivatives: what asks for one is refused."""
    if t.requires_grad and torch.is_grad_enabled():
        raise RuntimeError(f"{name} requires a gradient, and these operators have none: detach it, or call under "
                           "torch.no_grad()")
    if forward_ad.unpack_dual(t).tangent is not None:
        raise RuntimeError(f"{name} carries a tangent, and these operators have no forward-mode derivative: pass its "
                           "primal")


def _rows(t, name: str, head_dim: int, device: int):
    """(kv_rows, the tensor's shape)."""
    found = _tensors.rows(t, head_dim, device)
    if found is not None:
        return found
    if not isinstance(t, torch.Tensor) or len(shape := t.shape) != 3 or (dtype := _ROW_TYPES.get(t.dtype)) is None:
        raise TypeError(f"{name} must be a [tokens][heads][D] device tensor of bfloat16 or float16")
    _plain(t, name)
    if t.get_device() != device:
        _elsewhere(t, name, device)
    _, heads, width = shape
    token, head, column = t.stride()
    if width != head_dim or (column != 1 and t.numel()):
        raise ValueError(f"{name}: rows of {width} elements {column} apart; dense rows of {head_dim} are needed")
    return _pack_rows(t.data_ptr(), token, head, heads, dtype), shape


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


def _batch(block_size: int, device: int, tables, lens, starts, tokens: int, max_q, max_len):
    """(kv_batch, its num_seqs, max_queries and max_len)."""
    found = _tensors.batch(block_size, device, tables, lens, starts, tokens, max_q, max_len)
    if found is not None:
        return found
    (B, pages), (stride, _) = _ints(tables, "tables", 2, device)
    if tokens >= 2**31:
        _int32(tokens, "the number of new tokens")
    _ints(lens, "lens", 1, device, B)
    if starts is None:
        if tokens != B:
            raise ValueError(f"{tokens} new tokens for {B} sequences of one each: starts is needed")
        max_q, starts_at = 1, 0
    else:
        _ints(starts, "starts", 1, device, B + 1)
        starts_at = starts.data_ptr()
        max_q = max(1, tokens if max_q is None else min(tokens, int(max_q)))
    most = min(pages * block_size, 2**31 - 1024)
    if max_len is not None:
        most = min(most, max(int(max_len), -1))
    batch = _pack_batch(B, max_q, tokens, most, pages, 0, stride, tables.data_ptr(), lens.data_ptr(), starts_at)
    return batch, B, max_q, most


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
        return _current_stream(), _HERE
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    return stream.cuda_stream, torch.cuda.stream(stream)


_HERE = contextlib.nullcontext()


def _current_stream() -> int:
    device = torch.cuda.current_device()
    return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device)


# (Torch's own way to the handle, without a Stream around it, where it has one.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _used(stream, *tensors) -> None:
    """Tensors used on a stream that was named: as with a store's block table, torch must not hand their memory out again
    before the call's work is done there.  (With no stream named the call is like torch's own on the current stream.)"""
    if stream is not None:
        for t in tensors:
            if t is not None:
                _in_use_on(t, stream)


def _page_scales(t, cache: Cache, device: int):
    """kv_page_scales: (address, block stride, K to V)."""
    found = _tensors.scales(t, cache.layout.num_kv_heads, cache.struct.num_blocks, device)
    if found is not None:
        return found
    if not isinstance(t, torch.Tensor) or (t.dtype is not torch.uint8 and t.dtype is not torch.float8_e8m0fnu) or \
            len(shape := t.shape) != 3:
        raise TypeError("scales must be a [blocks][2][heads] uint8 or float8_e8m0fnu device tensor")
    _plain(t, "scales")
    if t.get_device() != device:
        _elsewhere(t, "scales", device)
    blocks, two, heads = shape
    if two != 2 or heads != cache.layout.num_kv_heads or blocks < cache.struct.num_blocks:
        raise ValueError(f"scales of {tuple(shape)} for a cache of {cache.struct.num_blocks} blocks of "
                         f"{cache.layout.num_kv_heads} heads")
    block, kv, head = t.stride()
    if head != 1 and heads > 1:
        raise TypeError("scales must have a dense last dimension")
    # (A stride over a single block leads nowhere.)
    return t.data_ptr(), block if blocks > 1 else max(block, kv + heads), kv


def _page_list(pages, counts, tokens: int, device: int):
    """(kv_page_list, its budget)."""
    found = _tensors.lists(pages, counts, tokens, device)
    if found is not None:
        return found
    (_, heads, budget), (token, head, _) = _ints(pages, "pages", 3, device, tokens)
    if counts is None:
        raise ValueError("pages without counts")
    counts_at = _dense_ints(counts, "counts", 1, device, tokens)
    return _pack_list(pages.data_ptr(), counts_at, token, head, heads, budget), budget


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
    layout = cache.layout
    D = layout.head_dim
    device = cache.struct.device
    (kr, shape), (vr, v_shape) = _rows(k, "k", D, device), _rows(v, "v", D, device)
    if shape != v_shape:
        raise ValueError(f"k and v differ in shape: {tuple(shape)} and {tuple(v_shape)}")
    batch = _batch(layout.block_size, device, tables, lens, starts, shape[0], max_q, max_len)[0]
    handle, _ = _call_stream(stream)
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    else:
        k_scale = v_scale = 1.0
    _raise(_lib.kv_append(ctypes.byref(cache.struct), _int32(layer, "layer"), batch, kr, vr,
                          _cache_dtype(cache, dtype, k), k_scale, v_scale, handle))
    if stream is not None:
        _used(stream, k, v, tables, lens, starts)


def kv_append_scaled(cache: Cache, layer: int, k, v, tables, lens, scales, starts=None, *, max_q=None, max_len=None,
                     stream=None) -> None:
    """kv_append into a float8_e4m3fn cache whose pages have ``scales`` (float8_e8m0fnu, or its bytes as uint8,
    [blocks][2][H]: K's and V's of each head): the new rows' pages take the smallest power of two that brings them, and
    what a page already held, to 448 or less."""
    layout = cache.layout
    D = layout.head_dim
    device = cache.struct.device
    (kr, shape), (vr, v_shape) = _rows(k, "k", D, device), _rows(v, "v", D, device)
    if shape != v_shape:
        raise ValueError(f"k and v differ in shape: {tuple(shape)} and {tuple(v_shape)}")
    batch = _batch(layout.block_size, device, tables, lens, starts, shape[0], max_q, max_len)[0]
    by = _pack_scales(*_page_scales(scales, cache, device))
    handle, _ = _call_stream(stream)
    _raise(_lib.kv_append_scaled(ctypes.byref(cache.struct), _int32(layer, "layer"), batch, kr, vr, by, handle))
    if stream is not None:
        _used(stream, k, v, tables, lens, starts, scales)


def kv_rotate(cache: Cache, layer: int, q, k, v, tables, lens, starts=None, *, freqs=None, positions=None,
              q_weight=None, k_weight=None, eps: float = 1e-6, weight_offset: float = 0.0, interleaved: bool = False,
              magnitude: float = 1.0, max_q=None, max_len=None, dtype=None, k_scale: float = 1.0, v_scale: float = 1.0,
              scales=None, out=None, stream=None):
    """Norm the new tokens' ``q`` and ``k`` for each head, rotate them by their position, and append K and V to layer
    ``layer``; returns the rotated queries.

    ``q_weight``, ``k_weight`` ([D], float32 or the rows' type; None: no norm): x / sqrt(mean x^2 + eps) *
    (weight_offset + weight).  ``freqs`` (float64 [n], None: no rotation): radians per position of the pairs (i, i + n)
    of a row's first 2n columns, or (2i, 2i + 1) if ``interleaved``; cosine and sine are multiplied by ``magnitude``.
    ``positions`` (int32 [tokens]): by default each token's place in its sequence.  ``dtype``, ``k_scale``, ``v_scale``
    and ``scales`` are kv_append's.  ``out`` (like ``q``) is made if not given, and may be ``q`` itself; rows of no
    sequence are left as they were."""
    layout = cache.layout
    D = layout.head_dim
    device = cache.struct.device
    qr, q_shape = _rows(q, "q", D, device)
    (kr, shape), (vr, v_shape) = _rows(k, "k", D, device), _rows(v, "v", D, device)
    if shape != v_shape or q_shape[0] != shape[0]:
        raise ValueError(f"q, k and v differ in shape: {tuple(q_shape)}, {tuple(shape)} and {tuple(v_shape)}")
    tokens = q_shape[0]
    batch = _batch(layout.block_size, device, tables, lens, starts, tokens, max_q, max_len)[0]
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    rotary, weight_dtype, *at = _rotate_arguments(q.dtype, D, tokens, device, freqs, positions, q_weight, k_weight)
    by = None if scales is None else KvPageScales(*_page_scales(scales, cache, device))
    options = _pack_rotate(_cache_dtype(cache, dtype, k), rotary, 1 if interleaved else 0, weight_dtype, *at, eps,
                           weight_offset, _factor(magnitude, "magnitude"), k_scale, v_scale, 0,
                           0 if by is None else ctypes.addressof(by))
    handle, here = _call_stream(stream)
    if out is None:
        with here:
            out, outr = _new_rows(q, q_shape)
    elif not isinstance(out, torch.Tensor) or out.dtype != q.dtype or out.shape != q_shape:
        raise TypeError("out must have the type and shape of q")
    else:
        outr, _ = _rows(out, "out", D, device)
    _raise(_lib.kv_rotate(ctypes.byref(cache.struct), _int32(layer, "layer"), batch, options, qr, outr, kr, vr, handle))
    if stream is not None:
        _used(stream, q, k, v, tables, lens, starts, freqs, positions, q_weight, k_weight, scales, out)
    return out


def _rotate_arguments(rows_dtype, head_dim: int, tokens: int, device: int, freqs, positions, q_weight, k_weight):
    """(rotary_dim, weight_dtype, freqs, positions, q_weight, k_weight) of kv_rotate_options."""
    found = _tensors.rotation(_ROW_TYPES[rows_dtype], head_dim, tokens, device, freqs, positions, q_weight, k_weight)
    if found is not None:
        return found
    rotary = freqs_at = weight_dtype = 0
    if freqs is not None:
        if not isinstance(freqs, torch.Tensor) or freqs.dtype is not torch.float64 or freqs.dim() != 1 or \
                not freqs.is_contiguous():
            raise TypeError("freqs must be a contiguous 1-dimensional float64 device tensor")
        _plain(freqs, "freqs")
        _on(freqs, "freqs", device)
        rotary, freqs_at = _int32(2 * freqs.shape[0], "twice the number of freqs"), freqs.data_ptr()
    positions_at = 0 if positions is None else _dense_ints(positions, "positions", 1, device, tokens)
    at = []
    for weight, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if weight is None:
            at.append(0)
            continue
        if not isinstance(weight, torch.Tensor) or weight.shape != (head_dim,) or not weight.is_contiguous() or \
                (weight.dtype is not torch.float32 and weight.dtype is not rows_dtype):
            raise TypeError(f"{name} must be a contiguous [{head_dim}] device tensor of float32 or {rows_dtype}")
        _plain(weight, name)
        _on(weight, name, device)
        of = KV_DTYPE_F32 if weight.dtype is torch.float32 else _DTYPES[weight.dtype]
        if weight_dtype not in (0, of):
            raise TypeError("q_weight and k_weight have different types")
        weight_dtype = of
        at.append(weight.data_ptr())
    return rotary, weight_dtype, freqs_at, positions_at, *at


def _new_rows(like, shape):
    """(a contiguous tensor like the rows `like`, its kv_rows)."""
    tokens, heads, width = shape
    t, at = _tensors.empty(like, 0, tokens, heads, width)
    return t, _pack_rows(at, heads * width, width, heads, _ROW_TYPES[like.dtype])


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

    ``scales``: those of a float8_e4m3fn cache's pages, as kv_append_scaled leaves them.  ``pages`` (int32
    [tokens][H or 1][budget], dense rows) and ``counts`` (int32 [tokens]): each new token attends over the first
    ``counts`` of its ``pages`` alone, which are places in its sequence's table, as kv_keep chooses them from kv_score's
    scores.  Neither goes with ``weights``, and with either all rows are as with ``full_weights``.
    """
    device = cache.struct.device
    layout = cache.layout
    qr, q_shape = _rows(q, "q", layout.head_dim, device)
    tokens, q_heads, _ = q_shape
    if weights is not None and max_len is None and isinstance(weights, torch.Tensor) and weights.dim() == 3:
        max_len = weights.shape[2]
    batch, B, max_q, most = _batch(layout.block_size, device, tables, lens, starts, tokens, max_q, max_len)
    if k_scale != 1.0 or v_scale != 1.0:
        k_scale, v_scale = _factor(k_scale, "k_scale"), _factor(v_scale, "v_scale")
    else:
        k_scale = v_scale = 1.0
    slopes_at = prior_at = weights_at = weights_seq = weights_head = 0
    if slopes is not None:
        _floats(slopes, "slopes", device, (q_heads,))
        slopes_at = slopes.data_ptr()
    if weights is not None:
        _weights(weights, "weights", device, (B, layout.num_kv_heads))
        if weights.shape[2] < most:
            raise ValueError(f"weights of {weights.shape[2]} tokens for sequences of up to {most}")
        weights_at, weights_seq, weights_head = weights.data_ptr(), weights.stride(0), weights.stride(1)
        if prior is not None:
            _weights(prior, "prior", device)
            if prior.shape != weights.shape or prior.stride() != weights.stride():
                raise TypeError("prior must have the shape and strides of weights")
            prior_at = prior.data_ptr()
    elif prior is not None:
        raise ValueError("prior without weights")
    window = _int32(window, "window") if window else 0
    options = (_cache_dtype(cache, dtype, q), window, 0.0 if scale is None else _factor(scale, "scale"),
               _factor(softcap, "softcap") if softcap else 0.0, k_scale, v_scale, slopes_at, prior_at, weights_at,
               weights_seq, weights_head, 1 if full_weights else 0, 0)
    by = chosen = None
    budget = -1
    if scales is not None:
        by = _pack_scales(*_page_scales(scales, cache, device))
    if pages is not None:
        chosen, budget = _page_list(pages, counts, tokens, device)
    elif counts is not None:
        raise ValueError("counts without pages")
    if out is not None and (out is q or out.dtype != q.dtype or out.shape != q_shape):
        raise TypeError("out must have the type and shape of q, and be another tensor")
    heads = (tokens, q_heads)
    if lse is not None:
        _floats(lse, "lse", device, heads)
    key = (layout.num_kv_heads, layout.head_dim, layout.elem_bytes, layout.block_size, B, max_q, tokens, most, window,
           weights is None, q_heads, budget, by is None)
    need = _attend_bytes.get(key)
    at, plain = ctypes.byref(cache.struct), by is None and chosen is None
    if plain:
        batch, options = ctypes.byref(KvBatch.from_buffer_copy(batch)), ctypes.byref(KvAttendOptions(*options))
    else:
        options = _pack_attend(*options)
    if need is None:
        need = _lib.kv_attend_workspace(at, batch, options, qr) if plain else \
            _lib.kv_attend_pages_workspace(at, batch, options, by, chosen, qr)
        if need < 0:
            _raise(need)
        if len(_attend_bytes) >= 4096:
            _attend_bytes.clear()
        _attend_bytes[key] = need
    handle, here = _call_stream(stream)
    workspace = None
    with here:
        if out is None:
            out, outr = _new_rows(q, q_shape)
        else:
            outr, _ = _rows(out, "out", layout.head_dim, device)
        if lse is None:
            lse, lse_at = _tensors.empty(q, 1, tokens, q_heads)
        else:
            lse_at = lse.data_ptr()
        if need:
            space, workspace = _tensors.empty(q, 3, need)
    layer = _int32(layer, "layer")
    if plain:
        _raise(_lib.kv_attend(at, layer, batch, options, qr, outr, lse_at, workspace, need, handle))
    else:
        _raise(_lib.kv_attend_pages(at, layer, batch, options, by, chosen, qr, outr, lse_at, workspace, need, handle))
    if stream is not None:
        _used(stream, q, tables, lens, starts, slopes, weights, prior, out, lse, scales, pages, counts)
    return out, lse


_attend_bytes = {}  # workspaces' bytes by the numbers that they depend on


def kv_attend_pages(cache: Cache, layer: int, q, tables, lens, starts=None, *, scales=None, pages=None, counts=None,
                    **options):
    """kv_attend with ``scales`` of pages, or over chosen ``pages``, or both."""
    if scales is None and pages is None:
        raise ValueError("neither scales nor pages")
    return kv_attend(cache, layer, q, tables, lens, starts, scales=scales, pages=pages, counts=counts, **options)


def kv_bounds(cache: Cache, layer: int, bounds: Cache, tables, lens, starts=None, *, max_q=None, max_len=None,
              dtype=None, stream=None) -> None:
    """For the pages of layer ``layer`` that new tokens lie in: the lowest and the highest stored K of every column over
    the page's tokens, into the same block of ``bounds``, a cache of the same heads, head_dim and element size with one
    token a block (lowest as K, highest as V).  Without ``starts`` each sequence has one new token; for a restored
    prefix, name as many rows as it has tokens.

    ``dtype``: the cache's, which 2-byte elements alone do not say."""
    device = cache.struct.device
    layout = cache.layout
    if starts is None:
        tokens = tables.shape[0] if isinstance(tables, torch.Tensor) and tables.dim() else 0
    else:
        # (How many rows there are only the device knows: as many as sequences may have tokens.)
        tokens = 2**31 - 1
        max_q = tokens if max_q is None else max_q
    batch = _batch(layout.block_size, device, tables, lens, starts, tokens, max_q, max_len)[0]
    if dtype is None:
        if layout.elem_bytes != 1:
            raise TypeError("dtype is needed: bfloat16 or float16")
        dtype = torch.float8_e4m3fn
    handle, _ = _call_stream(stream)
    _raise(_lib.kv_bounds(ctypes.byref(cache.struct), _int32(layer, "layer"), batch, _cache_dtype(cache, dtype, None),
                          ctypes.byref(bounds.struct), handle))
    if stream is not None:
        _used(stream, tables, lens, starts)


def kv_score(bounds: Cache, layer: int, q, tables, lens, starts=None, *, block_size: int, max_q=None, max_len=None,
             dtype=None, scale: float = 1.0, scales=None, out=None, counts=None, stream=None):
    """What no token of a page can exceed in scale * (q . k): for each new token, KV head and page up to the token's own
    the largest over the head's queries ``q`` ([tokens][query heads][D]) of q's positive part times the page's highest K
    and its negative part times the lowest, from kv_bounds's ``bounds`` of pages of ``block_size`` tokens.

    Returns (scores float32 [tokens][H][pages], counts int32 [tokens]: pages up to the token's own), which are kv_keep's
    weights and lens.  ``out`` and ``counts`` are made if not given; scores of pages beyond ``counts``, and rows of no
    sequence, are left as they were (in made ones, scores hold anything, and counts 0 with ``starts``)."""
    device = bounds.struct.device
    layout = bounds.layout
    qr, (tokens, _, _) = _rows(q, "q", layout.head_dim, device)
    block_size = _int32(block_size, "block_size")
    if block_size < 1:
        raise ValueError(f"block_size must be positive (got {block_size})")
    batch, _, _, most = _batch(block_size, device, tables, lens, starts, tokens, max_q, max_len)
    heads = layout.num_kv_heads
    pages = -(-max(most, 0) // block_size)
    handle, here = _call_stream(stream)
    with here:
        if out is None:
            out, out_at = _tensors.empty(q, 1, tokens, heads, pages)
            token, head = heads * pages, pages
        else:
            _weights(out, "out", device, (tokens, heads))
            if out.shape[2] < pages:
                raise ValueError(f"out of {out.shape[2]} pages for sequences of up to {pages}")
            out_at, (token, head, _) = out.data_ptr(), out.stride()
        if counts is None:
            counts, counts_at = (_tensors.empty if starts is None else _tensors.zeros)(q, 2, tokens)
        else:
            counts_at = _dense_ints(counts, "counts", 1, device, tokens)
    by = None if scales is None else KvPageScales(*_page_scales(scales, bounds, device))
    options = _pack_score(_cache_dtype(bounds, dtype, q), block_size, _factor(scale, "scale"), 0,
                          0 if by is None else ctypes.addressof(by), token, head)
    _raise(_lib.kv_score(ctypes.byref(bounds.struct), _int32(layer, "layer"), batch, options, qr, out_at, counts_at,
                         handle))
    if stream is not None:
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
    B = _ints(tables, "tables", 2, device)[0][0]
    _dense_ints(keep, "keep", 3, device, B)
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
