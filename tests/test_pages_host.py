"""Rotation, scaled pages and chosen pages on the CPU: what they refuse before any HIP call, and their references."""
import ctypes
import math

import numpy as np
import pytest
import torch

import pages_reference as pref
from test_attend_host import LAYOUT, SOME, _batch, _cache, _each, _rows

EMPTY = dict(num_seqs=0, num_queries=0, block_tables=None, lens=None)


def _scales(attend, heads, **changes):
    fields = dict(data=SOME, block_stride=2 * heads, kv_stride=heads)
    fields.update(changes)
    return attend.KvPageScales(**fields)


BAD_SCALES = (dict(data=None), dict(kv_stride=1), dict(block_stride=3), dict(block_stride=2, kv_stride=2),
              dict(kv_stride=-2), dict(block_stride=-4))


def _fp8(kvx, **changes):
    return _cache(kvx, kvx.make_layout(2, 2, 64, 1, 16, 16), **changes)


def test_append_scaled_refusals():
    from paper_2609_15021_amd import attend, kvx

    def call(cache, layer, batch, k=None, v=None, scales=None):
        heads = cache.layout.num_kv_heads
        k, v = k or _rows(attend, heads), v or _rows(attend, heads)
        scales = scales or _scales(attend, heads)
        return kvx._lib.kv_append_scaled(ctypes.byref(cache), layer, ctypes.byref(batch), ctypes.byref(k),
                                         ctypes.byref(v), ctypes.byref(scales), None)

    good, batch = _fp8(kvx), _batch(attend)
    assert call(_cache(kvx, kvx.make_layout(*LAYOUT)), 0, batch) == kvx.KV_EINVAL  # 2-byte elements
    assert call(good, 2, batch) == kvx.KV_EINVAL
    assert call(good, 0, _batch(attend, max_len=65)) == kvx.KV_EINVAL
    for changes in BAD_SCALES:
        assert call(good, 0, batch, scales=_scales(attend, 2, **changes)) == kvx.KV_EINVAL, changes
    for changes, status in ((dict(data=None), -1), (dict(data=SOME + 8), -4), (dict(heads=3), -1), (dict(dtype=3), -1)):
        assert call(good, 0, batch, k=_rows(attend, 2, **changes)) == status, changes
        assert call(good, 0, batch, v=_rows(attend, 2, **changes)) == status, changes
    assert call(good, 0, batch, k=_rows(attend, 2, dtype=attend.KV_DTYPE_F16)) == kvx.KV_EINVAL  # unlike v
    assert call(good, 0, _batch(attend, **EMPTY)) == kvx.KV_OK
    k = _rows(attend, 2)
    args = (ctypes.byref(good), 0, ctypes.byref(batch), ctypes.byref(k), ctypes.byref(k))
    assert kvx._lib.kv_append_scaled(*args, None, None) == kvx.KV_EINVAL


def test_rotate_refusals():
    from paper_2609_15021_amd import attend, kvx

    def call(cache, layer, batch, q=None, out=None, k=None, v=None, scales=None, **options):
        heads = cache.layout.num_kv_heads
        q = q or _rows(attend, 4 * heads)
        out = out or _rows(attend, 4 * heads)
        k, v = k or _rows(attend, heads), v or _rows(attend, heads)
        fields = dict(cache_dtype=attend.KV_DTYPE_BF16 if cache.layout.elem_bytes == 2 else attend.KV_DTYPE_E4M3,
                      rotary_dim=64, freqs=SOME, weight_dtype=attend.KV_DTYPE_F32)
        fields.update(options)
        o = attend.KvRotateOptions(**fields)
        if scales:
            o.scales = ctypes.pointer(scales)
        return kvx._lib.kv_rotate(ctypes.byref(cache), layer, ctypes.byref(batch), ctypes.byref(o), ctypes.byref(q),
                                  ctypes.byref(out), ctypes.byref(k), ctypes.byref(v), None)

    _each(call, kvx, attend)
    good, batch = _cache(kvx, kvx.make_layout(*LAYOUT)), _batch(attend)
    for options in (dict(rotary_dim=63), dict(rotary_dim=-2), dict(rotary_dim=66), dict(interleaved=2), dict(freqs=None),
                    dict(reserved=1), dict(eps=-1.0), dict(eps=math.nan), dict(weight_offset=math.inf),
                    dict(magnitude=-1.0), dict(magnitude=math.inf), dict(k_scale=0.5), dict(cache_dtype=0),
                    dict(cache_dtype=attend.KV_DTYPE_E4M3), dict(q_weight=SOME, weight_dtype=attend.KV_DTYPE_F16),
                    dict(k_weight=SOME, weight_dtype=0), dict(scales=_scales(attend, 2))):
        assert call(good, 0, batch, **options) == kvx.KV_EINVAL, options
    fp8 = _fp8(kvx)
    assert call(fp8, 0, batch, k_scale=-1.0) == kvx.KV_EINVAL
    assert call(fp8, 0, batch, k_scale=0.5, scales=_scales(attend, 2)) == kvx.KV_EINVAL
    for changes in BAD_SCALES:
        assert call(fp8, 0, batch, scales=_scales(attend, 2, **changes)) == kvx.KV_EINVAL, changes
    # Too many tokens for a launch: refused as a whole, rotated queries too.
    tiny = _cache(kvx, kvx.make_layout(1, 2, 64, 1, 1, 1))
    many = _batch(attend, num_queries=1 << 24, max_queries=1 << 24, max_len=1 << 24, table_len=1 << 24,
                  table_stride=1 << 24, starts=SOME)
    assert call(tiny, 0, many, scales=_scales(attend, 2)) == kvx.KV_EUNSUPPORTED
    for name in ("q", "out", "k", "v"):
        heads = 8 if name in ("q", "out") else 2
        for changes, status in ((dict(data=None), -1), (dict(data=SOME + 8), -4), (dict(heads=heads + 1), -1),
                                (dict(token_stride=132), -4), (dict(dtype=attend.KV_DTYPE_F16), -1)):
            assert call(good, 0, batch, **{name: _rows(attend, heads, **changes)}) == status, (name, changes)
    for changes in (dict(token_stride=8), dict(head_stride=0)):
        assert call(good, 0, batch, out=_rows(attend, 8, **changes)) == kvx.KV_EINVAL, changes
    assert call(good, 0, _batch(attend, **EMPTY)) == kvx.KV_OK
    rows = _rows(attend, 2)
    args = [ctypes.byref(rows)] * 4
    assert kvx._lib.kv_rotate(ctypes.byref(good), 0, ctypes.byref(batch), None, *args, None) == kvx.KV_EINVAL


def test_attend_pages_refusals():
    from paper_2609_15021_amd import attend, kvx

    def call(cache, layer, batch, q=None, scales=None, pages=None, neither=False, size=1 << 40, **options):
        heads = 2 * cache.layout.num_kv_heads
        q = q or _rows(attend, heads)
        fp8 = cache.layout.elem_bytes == 1
        fields = dict(cache_dtype=attend.KV_DTYPE_E4M3 if fp8 else attend.KV_DTYPE_BF16)
        fields.update(options)
        o = attend.KvAttendOptions(**fields)
        if not (scales or pages or neither):
            pages = _list()
        by = ctypes.byref(scales) if scales else None
        chosen = ctypes.byref(pages) if pages else None
        need = kvx._lib.kv_attend_pages_workspace(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(o), by, chosen,
                                                  ctypes.byref(q))
        got = kvx._lib.kv_attend_pages(ctypes.byref(cache), layer, ctypes.byref(batch), ctypes.byref(o), by, chosen,
                                       ctypes.byref(q), ctypes.byref(q), SOME, SOME, size, None)
        assert need in (got, 0) or need > 0 or layer != 0, (need, got)
        return got

    def _list(**changes):
        fields = dict(pages=SOME, counts=SOME, token_stride=8, head_stride=4, heads=2, budget=4)
        fields.update(changes)
        return attend.KvPageList(**fields)

    _each(call, kvx, attend)
    good, fp8, batch = _cache(kvx, kvx.make_layout(*LAYOUT)), _fp8(kvx), _batch(attend)
    assert call(good, 0, batch, neither=True) == kvx.KV_EINVAL
    assert call(good, 0, batch, scales=_scales(attend, 2)) == kvx.KV_EINVAL  # 2-byte elements
    for changes in BAD_SCALES:
        assert call(fp8, 0, batch, scales=_scales(attend, 2, **changes)) == kvx.KV_EINVAL, changes
    for options in (dict(k_scale=0.5), dict(v_scale=2.0)):
        assert call(fp8, 0, batch, scales=_scales(attend, 2), **options) == kvx.KV_EINVAL, options
    for changes, status in ((dict(heads=3), -1), (dict(budget=0), -1), (dict(token_stride=-1), -1), (dict(pages=None), -1),
                            (dict(counts=None), -1), (dict(head_stride=-1), -1), (dict(budget=2**31 // 16), -4)):
        assert call(good, 0, batch, pages=_list(**changes)) == status, changes
    weights = dict(weights_out=SOME, weights_seq_stride=128, weights_head_stride=64)
    assert call(good, 0, batch, **weights) == kvx.KV_EUNSUPPORTED
    assert call(good, 0, batch, size=15) == kvx.KV_EINVAL
    many = _batch(attend, num_queries=1 << 24, max_queries=1 << 24, starts=SOME)
    assert call(good, 0, many) == kvx.KV_EUNSUPPORTED
    assert call(good, 0, _batch(attend, **EMPTY), pages=_list(pages=None, counts=None)) == kvx.KV_OK


@pytest.mark.parametrize("fp8", [False, True])
def test_chosen_pages_of_many_sequences(fp8):
    """Lists know no sequence's bounds: max_queries may be all of a large batch's new tokens, as the binding has it by
    default, and only rows, parts and heads are limited, for the workspace as for the call."""
    from paper_2609_15021_amd import attend, kvx
    cache = _cache(kvx, kvx.make_layout(1, 8, 64, 1 if fp8 else 2, 16, 16))
    q = _rows(attend, 40, token_stride=2560)
    o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_E4M3 if fp8 else attend.KV_DTYPE_BF16)
    by = _scales(attend, 8) if fp8 else None

    def call(tokens, max_queries, q=q, cache=cache, seqs=2048):
        batch = _batch(attend, num_seqs=seqs, num_queries=tokens, max_queries=max_queries, starts=SOME)
        pages = attend.KvPageList(pages=SOME, counts=SOME, token_stride=32, head_stride=4, budget=4,
                                  heads=cache.layout.num_kv_heads)
        args = (ctypes.byref(o), ctypes.byref(by) if by else None, ctypes.byref(pages), ctypes.byref(q))
        need = kvx._lib.kv_attend_pages_workspace(ctypes.byref(cache), ctypes.byref(batch), *args)
        # (A workspace that is too small: what is not refused before comes to that.)
        got = kvx._lib.kv_attend_pages(ctypes.byref(cache), 0, ctypes.byref(batch), *args, ctypes.byref(q), SOME, SOME,
                                       0, None)
        assert got == (kvx.KV_EINVAL if need > 0 else need)
        return need

    assert call(8192, 8192) == call(8192, 4) > 0
    assert call(1 << 20, 1 << 20) == call(1 << 20, 512) > 0
    assert call((1 << 20) + 1, 4) == kvx.KV_EUNSUPPORTED
    # Rows beyond 32 bits in a sequence, which only tiles of a sequence's rows would have to count.
    one = _cache(kvx, kvx.make_layout(1, 1, 64, 1 if fp8 else 2, 16, 16))
    wide = _rows(attend, 16383, token_stride=1 << 20)
    by = _scales(attend, 1) if fp8 else None
    assert call(1 << 18, 1 << 18, wide, one, 1) > 0


def test_bounds_and_score_refusals():
    from paper_2609_15021_amd import attend, kvx
    ones = lambda *dims, **kw: _cache(kvx, kvx.make_layout(*dims, 1, 1), **kw)  # noqa: E731

    def bound(cache, layer, batch, bounds=None, dtype=attend.KV_DTYPE_BF16):
        lay = cache.layout
        bounds = bounds or ones(2, lay.num_kv_heads, lay.head_dim, lay.elem_bytes)
        return kvx._lib.kv_bounds(ctypes.byref(cache), layer, ctypes.byref(batch), dtype, ctypes.byref(bounds), None)

    _each(bound, kvx, attend)
    good, batch = _cache(kvx, kvx.make_layout(*LAYOUT)), _batch(attend)
    for dims, changes in (((2, 1, 64, 2), {}), ((2, 2, 128, 2), {}), ((2, 2, 64, 1), {}), ((2, 2, 64, 2), dict(num_blocks=63)),
                          ((1, 2, 64, 2), dict(align=8))):
        assert bound(good, 0, batch, bounds=ones(*dims, **changes)) < 0, (dims, changes)
    assert bound(good, 1, batch, bounds=ones(1, 2, 64, 2)) == kvx.KV_EINVAL  # no such layer
    assert bound(good, 0, batch, bounds=good) == kvx.KV_EINVAL               # 16 tokens a block
    assert bound(good, 0, batch, dtype=attend.KV_DTYPE_E4M3) == kvx.KV_EINVAL
    assert bound(good, 0, _batch(attend, **EMPTY)) == kvx.KV_OK
    assert kvx._lib.kv_bounds(ctypes.byref(good), 0, ctypes.byref(batch), 1, None, None) == kvx.KV_EINVAL

    def score(bounds, layer, batch, q=None, scales=None, scores=SOME, **options):
        q = q or _rows(attend, 2 * bounds.layout.num_kv_heads)
        fields = dict(cache_dtype=attend.KV_DTYPE_BF16, block_size=16, token_stride=8, head_stride=4)
        fields.update(options)
        o = attend.KvScoreOptions(**fields)
        if scales:
            o.scales = ctypes.pointer(scales)
        return kvx._lib.kv_score(ctypes.byref(bounds), layer, ctypes.byref(batch), ctypes.byref(o), ctypes.byref(q),
                                 scores, SOME, None)

    low_high = ones(2, 2, 64, 2)
    assert score(good, 0, batch) == kvx.KV_EINVAL  # not bounds
    assert score(low_high, 2, batch) == kvx.KV_EINVAL
    for options in (dict(block_size=0), dict(block_size=15), dict(cache_dtype=attend.KV_DTYPE_F16), dict(cache_dtype=3),
                    dict(scale=-1.0), dict(scale=math.nan), dict(reserved=1), dict(token_stride=3), dict(head_stride=3),
                    dict(token_stride=-8), dict(scores=None), dict(scales=_scales(attend, 2))):
        assert score(low_high, 0, batch, **options) == kvx.KV_EINVAL, options
    for changes, status in ((dict(data=None), -1), (dict(data=SOME + 8), -4), (dict(heads=3), -1)):
        assert score(low_high, 0, batch, q=_rows(attend, 4, **changes)) == status, changes
    fp8 = ones(2, 2, 64, 1)
    for changes in BAD_SCALES:
        assert score(fp8, 0, batch, scales=_scales(attend, 2, **changes), cache_dtype=3) == kvx.KV_EINVAL, changes
    long = _batch(attend, max_len=2**31 - 1024, table_len=2**31 - 1024, table_stride=2**31)
    assert score(low_high, 0, long, block_size=1, token_stride=2**40, head_stride=2**32) == kvx.KV_EUNSUPPORTED
    assert score(low_high, 0, _batch(attend, **EMPTY)) == kvx.KV_OK


@pytest.mark.parametrize("name,pack", [("KvRows", "rows"), ("KvBatch", "batch"), ("KvAttendOptions", "attend"),
                                       ("KvPageScales", "scales"), ("KvPageList", "list"), ("KvRotateOptions", "rotate"),
                                       ("KvScoreOptions", "score")])
def test_structures_as_bytes(name, pack):
    """What the binding packs is the structure, field by field."""
    from paper_2609_15021_amd import attend
    kind = getattr(attend, name)
    numbers = [i + 1 for i in range(len(kind._fields_))]
    data = getattr(attend, f"_pack_{pack}")(*numbers)
    assert len(data) == ctypes.sizeof(kind)
    x = kind.from_buffer_copy(data)
    for number, (field, kind_of) in zip(numbers, kind._fields_):
        got = getattr(x, field)
        assert (ctypes.cast(got, ctypes.c_void_p).value if isinstance(got, ctypes._Pointer) else got) == number, field


def test_tensors_answer_as_the_binding_does(monkeypatch):
    """The compiled module and the checks in Python give the same structures, for tensors of every kind of stride."""
    from paper_2609_15021_amd import _tensors, attend, kvx
    lay = kvx.make_layout(1, 2, 64, 1, 16, 16)

    class Fake:
        layout, struct = lay, _cache(kvx, lay)

    wide = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    meta = torch.zeros(4, 9, dtype=torch.int32)
    scales, counts = torch.zeros(70, 2, 16, dtype=torch.uint8)[..., :2], torch.zeros(3, dtype=torch.int32)
    freqs, weight = torch.ones(32, dtype=torch.float64), torch.ones(64)
    half, short = wide[:1].half(), weight.bfloat16()
    pages = torch.zeros(3, 4000, dtype=torch.int32)
    calls = [lambda: attend._rows(wide, "x", 64, -1), lambda: attend._rows(wide[:, 2:5], "x", 64, -1),
             lambda: attend._rows(half, "x", 64, -1), lambda: attend._rows(wide.transpose(0, 1), "x", 64, -1),
             lambda: attend._batch(16, -1, meta[:3], counts, None, 3, None, None),
             lambda: attend._batch(16, -1, meta[:3, :5], counts, meta[0, :4], 7, 5, 33),
             lambda: attend._batch(16, -1, meta[:3], counts, meta[0, :4], 7, 2**70, -2**70),
             lambda: attend._batch(2**20, -1, pages, counts, None, 3, 9, 2**40),
             lambda: attend._page_scales(scales, Fake, -1),
             lambda: attend._page_scales(scales.view(torch.float8_e8m0fnu), Fake, -1),
             lambda: attend._page_list(meta[:3].view(3, 3, 3), counts, 3, -1),
             lambda: attend._dense_ints(counts, "x", 1, -1, 3),
             lambda: attend._rotate_arguments(torch.bfloat16, 64, 3, -1, freqs, counts, weight, weight),
             lambda: attend._rotate_arguments(torch.bfloat16, 64, 3, -1, None, None, short, None)]
    fast = [call() for call in calls]
    for name in ("rows", "batch", "scales", "lists", "ints", "rotation"):
        monkeypatch.setattr(_tensors, name, lambda *args: None)
    for a, call in zip(fast, calls):
        b = call()
        assert (tuple(a) if isinstance(a, (tuple, list)) else a) == (tuple(b) if isinstance(b, (tuple, list)) else b)


def test_exponents():
    """The smallest power of two that brings a page to 448: on both sides of every border."""
    for e in (1, 2, 90, 127, 200):
        top = 448.0 * 2.0**(e - 127)
        assert pref.exponent(top) == e and pref.exponent(np.nextafter(top, np.inf)) == e + 1
    assert pref.exponent(0.0) == 1


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_products(interleaved):
    """What a rotation is for: products of rotated rows depend on the difference of their positions alone."""
    gen = np.random.default_rng(0)
    q, k = gen.standard_normal((2, 24))
    freqs = 10000.0 ** (-np.arange(8) / 8)
    at = lambda x, p: pref.rotated(x, p, freqs, interleaved=interleaved)[0]  # noqa: E731
    assert np.isclose(at(q, 100) @ at(k, 60), at(q, 45) @ at(k, 5), atol=1e-10)
    assert not np.isclose(at(q, 100) @ at(k, 60), at(q, 100) @ at(k, 61), atol=1e-3)


def test_binding_refusals():
    """What the binding refuses by itself: tensors on the CPU, of other types and shapes."""
    from paper_2609_15021_amd import attend, kvx
    lay = kvx.make_layout(1, 2, 64, 1, 16, 16)

    class Fake:
        layout, struct = lay, _cache(kvx, lay)

    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    tables, lens = torch.zeros(1, 4, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        attend.kv_rotate(Fake, 0, q, q[:, :2], q[:, :2], tables, lens)
    with pytest.raises(ValueError):
        attend.kv_attend_pages(Fake, 0, q, tables, lens)
    with pytest.raises(ValueError):
        attend.kv_append(Fake, 0, q, q, tables, lens, scales=tables, k_scale=0.5)
    for scales in (torch.zeros(64, 2, 2), torch.zeros(64, 2, dtype=torch.uint8), None):
        with pytest.raises(TypeError):
            attend._page_scales(scales, Fake, -1)
    for shape in ((63, 2, 2), (64, 2, 3), (64, 1, 2)):
        with pytest.raises(ValueError):
            attend._page_scales(torch.zeros(shape, dtype=torch.uint8), Fake, -1)
    with pytest.raises(TypeError):
        attend._page_scales(torch.zeros(64, 2, 4, dtype=torch.uint8)[..., ::2], Fake, -1)
    _, block, kv = attend._page_scales(torch.zeros(64, 2, 16, dtype=torch.float8_e8m0fnu)[..., :2], Fake, -1)
    assert (block, kv) == (32, 16)
