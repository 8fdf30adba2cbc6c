"""The operators on a paged cache on the CPU: exports, and what they refuse before any HIP call."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import attend_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "kvx_attend.h")
SOME = 0x7F0000000000  # an address that is never read: refused calls end before any


def _declared():
    return sorted(set(re.findall(r"^KV_API\s+[^;(]*?\b(kv_\w+)\s*\(", open(HEADER).read(), flags=re.M)))


def test_exports():
    from paper_2609_15021_amd import attend, kvx
    assert set(attend.EXPORTS) == set(_declared())
    out = subprocess.run(["nm", "-D", "--defined-only", kvx.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = {ln.split()[-1] for ln in out.splitlines() if " T " in ln}
    assert set(attend.EXPORTS) <= exported
    for name in attend.EXPORTS:
        assert callable(getattr(attend, name, None)) or name.endswith("_workspace")


def test_header_compiles_as_plain_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "kvx_attend.h"\nint main(void){kv_batch b={0};kv_attend_options o={0};(void)b;(void)o;'
                   'return (int)sizeof(kv_rows)-32;}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-c", "-o",
                    str(tmp_path / "t.o")], check=True)


def _cache(kvx, layout, num_blocks=64, stride=0, order=0, reserved=0, align=0):
    ptrs = (ctypes.c_void_p * layout.num_layers)(*[SOME + (1 << 32) * l + align for l in range(layout.num_layers)])
    c = kvx.KvCache(layout, num_blocks, 0, order, reserved, ctypes.cast(ptrs, ctypes.POINTER(ctypes.c_void_p)), stride)
    c._keep = ptrs
    return c


def _batch(attend, **changes):
    fields = dict(num_seqs=2, max_queries=1, num_queries=2, max_len=64, table_len=4, reserved=0, table_stride=4,
                  block_tables=SOME, lens=SOME, starts=None)
    fields.update(changes)
    return attend.KvBatch(**fields)


def _rows(attend, count, **changes):
    fields = dict(data=SOME, token_stride=count * 64, head_stride=64, heads=count, dtype=attend.KV_DTYPE_BF16)
    fields.update(changes)
    return attend.KvRows(**fields)


LAYOUT = (2, 2, 64, 2, 16, 16)
BAD_CACHES = [("layout", (2, 2, 64, 4, 16, 16), {}, -1), ("layer", LAYOUT, dict(layer=2), -1),
              ("layer", LAYOUT, dict(layer=-1), -1), ("blocks", LAYOUT, dict(num_blocks=0), -1),
              ("order", LAYOUT, dict(order=2), -1), ("reserved", LAYOUT, dict(reserved=1), -1),
              ("stride", LAYOUT, dict(stride=4096), -1), ("stride", LAYOUT, dict(stride=8200), -4),
              ("pointer", LAYOUT, dict(align=8), -4), ("D", (1, 2, 264, 2, 16, 16), {}, -4),
              ("D", (1, 2, 12, 2, 16, 16), {}, -4)]
BAD_BATCHES = [(dict(num_seqs=-1), -1), (dict(max_queries=0), -1), (dict(num_queries=-1), -1), (dict(max_len=65), -1),
               (dict(max_len=-1), -1), (dict(table_stride=3), -1), (dict(block_tables=None), -1), (dict(lens=None), -1),
               (dict(reserved=1), -1), (dict(num_queries=1), -1), (dict(num_seqs=65536, num_queries=65536), -4)]


def _each(call, kvx, attend):
    """call(cache, layer, batch) for every cache and batch that must be refused."""
    good = _cache(kvx, kvx.make_layout(*LAYOUT))
    for what, dims, changes, status in BAD_CACHES:
        changes = dict(changes)
        layer = changes.pop("layer", 0)
        got = call(_cache(kvx, kvx.make_layout(*dims), **changes), layer, _batch(attend))
        assert got == status, (what, dims, changes, got, kvx.kv_last_error())
    for changes, status in BAD_BATCHES:
        assert call(good, 0, _batch(attend, **changes)) == status, (changes, kvx.kv_last_error())


def test_append_refusals():
    from paper_2609_15021_amd import attend, kvx

    def call(cache, layer, batch, k=None, v=None, dtype=attend.KV_DTYPE_BF16, ks=1.0, vs=1.0):
        heads = cache.layout.num_kv_heads
        k, v = k or _rows(attend, heads), v or _rows(attend, heads)
        return kvx._lib.kv_append(ctypes.byref(cache), layer, ctypes.byref(batch), ctypes.byref(k), ctypes.byref(v),
                                  dtype, ks, vs, None)

    _each(call, kvx, attend)
    good, batch = _cache(kvx, kvx.make_layout(*LAYOUT)), _batch(attend)
    for changes, status in ((dict(data=None), -1), (dict(data=SOME + 8), -4), (dict(token_stride=132), -4),
                            (dict(head_stride=-64), -1), (dict(heads=3), -1), (dict(dtype=attend.KV_DTYPE_E4M3), -1),
                            (dict(dtype=attend.KV_DTYPE_F16), -1)):
        rows = _rows(attend, 2, **changes)
        assert call(good, 0, batch, k=rows) == status, changes
        assert call(good, 0, batch, v=rows) == status, changes
    assert call(good, 0, batch, dtype=attend.KV_DTYPE_E4M3) == kvx.KV_EINVAL  # 2-byte elements
    assert call(good, 0, batch, dtype=0) == kvx.KV_EINVAL
    assert call(good, 0, batch, ks=0.5) == kvx.KV_EINVAL                      # a scale, but not quantised
    fp8 = _cache(kvx, kvx.make_layout(1, 2, 64, 1, 16, 16))
    assert call(fp8, 0, batch, dtype=attend.KV_DTYPE_BF16) == kvx.KV_EINVAL
    for scale in (-1.0, math.nan):
        assert call(fp8, 0, batch, dtype=attend.KV_DTYPE_E4M3, ks=scale) == kvx.KV_EINVAL
    # Nothing to do is no error, whatever the pointers.
    empty = _batch(attend, num_seqs=0, num_queries=0, block_tables=None, lens=None)
    assert call(good, 0, empty, k=_rows(attend, 2, data=None), v=_rows(attend, 2, data=None)) == kvx.KV_OK
    assert kvx._lib.kv_append(None, 0, None, None, None, 1, 1.0, 1.0, None) == kvx.KV_EINVAL


def test_attend_refusals():
    from paper_2609_15021_amd import attend, kvx

    def call(cache, layer, batch, q=None, out=None, lse=SOME, space=SOME, size=1 << 40, workspace_only=False,
             **options):
        heads = 2 * cache.layout.num_kv_heads
        q, out = q or _rows(attend, heads), out or _rows(attend, heads)
        o = attend.KvAttendOptions(**dict(dict(cache_dtype=attend.KV_DTYPE_BF16), **options))
        if workspace_only:
            return kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(o),
                                                ctypes.byref(q))
        return kvx._lib.kv_attend(ctypes.byref(cache), layer, ctypes.byref(batch), ctypes.byref(o), ctypes.byref(q),
                                  ctypes.byref(out), lse, space, size, None)

    _each(call, kvx, attend)
    good, batch = _cache(kvx, kvx.make_layout(*LAYOUT)), _batch(attend)
    for changes, status in ((dict(data=None), -1), (dict(data=SOME + 8), -4), (dict(token_stride=132), -4),
                            (dict(heads=3), -1), (dict(dtype=attend.KV_DTYPE_F16), -1), (dict(dtype=7), -1)):
        rows = _rows(attend, 4, **changes)
        assert call(good, 0, batch, q=rows) == status, changes
        assert call(good, 0, batch, out=rows) == status, changes
    for options in (dict(window=-1), dict(scale=-1.0), dict(scale=math.inf), dict(softcap=math.nan),
                    dict(softcap=-2.0), dict(k_scale=2.0), dict(v_scale=0.5), dict(cache_dtype=0),
                    dict(cache_dtype=attend.KV_DTYPE_E4M3), dict(weights_in=SOME),
                    dict(weights_out=SOME, weights_seq_stride=128, weights_head_stride=63),
                    dict(weights_out=SOME, weights_seq_stride=63, weights_head_stride=64),
                    dict(weights_out=SOME, weights_seq_stride=-128, weights_head_stride=64)):
        assert call(good, 0, batch, **options) == kvx.KV_EINVAL, options
        assert call(good, 0, batch, workspace_only=True, **options) == kvx.KV_EINVAL, options
    for options in (dict(scale=1e-38), dict(scale=1e37), dict(scale=1e-30, softcap=1e10)):
        assert call(good, 0, batch, **options) == kvx.KV_EUNSUPPORTED, options
    for changes in (dict(max_queries=2**30, num_queries=2**30), dict(max_queries=1 << 20, num_queries=1 << 20, num_seqs=500)):
        many = _batch(attend, starts=SOME, **changes)
        assert call(good, 0, many) == kvx.KV_EUNSUPPORTED, changes
    need = call(good, 0, batch, workspace_only=True)
    assert need >= 0
    if need:
        assert call(good, 0, batch, size=need - 1) == kvx.KV_EINVAL
        assert call(good, 0, batch, space=None) == kvx.KV_EINVAL
        assert call(good, 0, batch, space=SOME + 4) == kvx.KV_EUNSUPPORTED
    assert call(good, 0, _batch(attend, num_seqs=0, num_queries=0)) == kvx.KV_OK
    assert kvx._lib.kv_attend(None, 0, None, None, None, None, None, None, 0, None) == kvx.KV_EINVAL
    assert kvx._lib.kv_attend_workspace(None, None, None, None) == kvx.KV_EINVAL


def test_attend_workspace_follows_the_batch():
    """More work never needs less workspace, and its size is a size."""
    from paper_2609_15021_amd import attend, kvx
    cache = _cache(kvx, kvx.make_layout(1, 8, 128, 2, 16, 16), num_blocks=1 << 20)
    o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16)
    for seqs, queries, length in ((1, 1, 1), (1, 1, 131077), (64, 1, 8192), (1, 2085, 34853), (7, 37, 131072),
                                  (65535, 1, 16), (1, 1, 2**31 - 1024), (3, 100000, 200000)):
        tokens = seqs * queries
        b = _batch(attend, num_seqs=seqs, max_queries=queries, num_queries=tokens, max_len=length,
                   table_len=-(-length // 16), table_stride=-(-length // 16), starts=SOME)
        q = _rows(attend, 40, token_stride=40 * 128, head_stride=128)
        need = kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(o), ctypes.byref(q))
        assert 0 <= need < 1 << 36, (seqs, queries, length, need)


def test_keep_and_compact_refusals():
    from paper_2609_15021_amd import attend, kvx

    def keep(weights=SOME, lens=SOME, seqs=2, heads=2, max_len=64, budget=16, sinks=2, recent=4, out=SOME, kept=SOME,
             space=SOME, size=1 << 30):
        return kvx._lib.kv_keep(weights, 128, 64, lens, seqs, heads, max_len, budget, sinks, recent, out, kept, SOME,
                                space, size, None)

    for changes in (dict(weights=None), dict(lens=None), dict(out=None), dict(kept=None), dict(seqs=-1), dict(heads=0),
                    dict(max_len=-1), dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=13)):
        assert keep(**changes) == kvx.KV_EINVAL, changes
    assert keep(seqs=65536) == kvx.KV_EUNSUPPORTED
    assert keep(max_len=2**31 - 1) == kvx.KV_EUNSUPPORTED
    need = kvx._lib.kv_keep_workspace(2, 2, 100000, 16)
    assert need > 0 and kvx._lib.kv_keep_workspace(2, 2, 100000, 100000) == 0
    assert keep(max_len=100000, size=need - 1) == keep(max_len=100000, space=None) == kvx.KV_EINVAL
    assert keep(max_len=100000, space=SOME + 2) == kvx.KV_EUNSUPPORTED
    assert kvx._lib.kv_keep_workspace(2, 2, 64, 0) == kvx.KV_EINVAL
    assert keep(seqs=0, lens=None) == kvx.KV_OK

    def compact(cache, layer=0, seqs=2, src=SOME, stride=4, length=4, idx=SOME, heads=2, budget=16, kept=SOME, dst=SOME,
                dst_stride=1, dst_len=1):
        return kvx._lib.kv_compact(ctypes.byref(cache), layer, seqs, src, stride, length, idx, heads, budget, kept, dst,
                                   dst_stride, dst_len, None)

    for what, dims, changes, status in BAD_CACHES:
        if what in ("D", "layout") and dims[2] != 12:
            continue  # any element size and row length moves
        changes = dict(changes)
        layer = changes.pop("layer", 0)
        assert compact(_cache(kvx, kvx.make_layout(*dims), **changes), layer) == status, (what, dims, changes)
    good = _cache(kvx, kvx.make_layout(*LAYOUT))
    for changes in (dict(seqs=-1), dict(heads=3), dict(budget=17), dict(budget=0), dict(stride=3), dict(dst_stride=0),
                    dict(src=None), dict(idx=None), dict(kept=None), dict(dst=None)):
        assert compact(good, **changes) == kvx.KV_EINVAL, changes
    assert compact(good, seqs=65536) == kvx.KV_EUNSUPPORTED
    assert compact(good, seqs=0, src=None) == kvx.KV_OK
    assert kvx._lib.kv_compact(None, 0, 1, None, 0, 0, None, 1, 1, None, None, 0, 0, None) == kvx.KV_EINVAL


def test_binding_refuses_before_any_library_call(monkeypatch):
    """Shapes and types that contradict each other end in the binding (host tensors stand in for any wrong one)."""
    from paper_2609_15021_amd import attend, kvx

    class NoLibrary:
        def __getattr__(self, name):
            raise AssertionError(f"library call {name} made for a refused request")

    cache = object.__new__(kvx.Cache)
    cache.layout = kvx.make_layout(*LAYOUT)
    cache.struct = _cache(kvx, cache.layout)
    monkeypatch.setattr(attend, "_lib", NoLibrary())
    rows = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    ints = torch.zeros(2, 4, dtype=torch.int32)
    for call in (lambda: attend.kv_append(cache, 0, rows, rows, ints, ints[:, 0]),
                 lambda: attend.kv_attend(cache, 0, rows, ints, ints[:, 0]),
                 lambda: attend.kv_keep(torch.zeros(2, 2, 8), ints[:, 0], 4),
                 lambda: attend.kv_compact(cache, 0, ints, ints[None], ints[:, 0], ints)):
        with pytest.raises(TypeError, match="device tensor"):
            call()


def test_reference_attend_against_a_softmax():
    """The 64-bit form the GPU tests compare with, against torch's softmax on a batch without options."""
    c = ref.Case(2, 3, 16, 4, [9, 1, 0, 6], [2, 1, 0, 8], seed=3)
    out, lse, weights, *_ = ref.attend(c)
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            p = n - c.new[b] + i
            row = int(c.starts[b]) + i
            if p < 0:
                assert not out[row].any() and np.isinf(lse[row]).all()
                continue
            for head in range(6):
                s = torch.tensor(c.k[b][:p + 1, head // 3]) @ c.q[row, head].double() / 4.0
                want = torch.softmax(s, 0) @ torch.tensor(c.v[b][:p + 1, head // 3])
                np.testing.assert_allclose(out[row, head], want.numpy(), rtol=1e-12)
                np.testing.assert_allclose(lse[row, head], torch.logsumexp(s, 0).item(), rtol=1e-12)
    # Every row that sees a token gives away a weight of 1 per query head.
    rows = [sum(1 for i in range(q) if n - q + i >= 0) for n, q in zip(c.lens, c.new)]
    np.testing.assert_allclose(weights.sum((1, 2)), [6 * r for r in rows], rtol=1e-12)


def test_reference_keep():
    w = np.array([[[5, 1, np.nan, 1, 7, -np.inf, 1, 0.0, -0.0, 9]]], dtype=np.float32)
    for budget, sinks, recent, want in ((4, 0, 0, [0, 1, 4, 9]), (5, 0, 0, [0, 1, 3, 4, 9]), (3, 1, 1, [0, 4, 9]),
                                        (8, 0, 1, [0, 1, 3, 4, 6, 7, 8, 9]), (9, 0, 0, [0, 1, 3, 4, 5, 6, 7, 8, 9]),
                                        (2, 1, 1, [0, 9]), (10, 0, 0, list(range(10)))):
        got, kept, kw = ref.keep(w, [10], budget, sinks, recent)
        assert got[0, 0].tolist() == want and kept.tolist() == [min(10, budget)]
