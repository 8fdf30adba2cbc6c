"""Edges of the operators on the paged cache on the CPU: workspaces, and what is refused before any HIP call."""
import ctypes
import math

import pytest
import torch

from test_attend_host import SOME, _batch, _cache, _rows


def test_workspace_of_scores_is_bounded():
    """Received weights of few new tokens come from stored scores, up to a GiB of them; wider bounds need no more."""
    from paper_2609_15021_amd import attend, kvx
    cache = _cache(kvx, kvx.make_layout(1, 8, 128, 2, 16, 16), num_blocks=1 << 20)
    q = _rows(attend, 64, token_stride=64 * 128, head_stride=128)

    def need(seqs, length, weights):
        b = _batch(attend, num_seqs=seqs, num_queries=seqs, max_len=length, table_len=-(-length // 16),
                   table_stride=-(-length // 16))
        o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16, weights_out=SOME if weights else None,
                                   weights_seq_stride=8 * length, weights_head_stride=length)
        return kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(o), ctypes.byref(q))

    for seqs, length in ((1, 100), (48, 8192), (32, 131072), (33, 131072), (256, 131072), (65535, 4096),
                         (1, 2**31 - 1024)):
        without, score_bytes = need(seqs, length, False), seqs * 8 * 8 * -(-length // 32) * 32 * 4
        extra = need(seqs, length, True) - without
        assert without >= 0 and extra == (score_bytes if score_bytes <= 1 << 30 else 0), (seqs, length, extra)


@pytest.mark.parametrize("which", ["ks", "vs"])
def test_append_refuses_infinite_scales(which):
    from paper_2609_15021_amd import attend, kvx
    cache, batch, rows = _cache(kvx, kvx.make_layout(1, 2, 64, 1, 16, 16)), _batch(attend), _rows(attend, 2)
    for scale in (math.inf, -math.inf):
        scales = dict(dict(ks=1.0, vs=1.0), **{which: scale})
        assert kvx._lib.kv_append(ctypes.byref(cache), 0, ctypes.byref(batch), ctypes.byref(rows), ctypes.byref(rows),
                                  attend.KV_DTYPE_E4M3, scales["ks"], scales["vs"], None) == kvx.KV_EINVAL


def test_strides_that_lead_nowhere():
    """A single token's or head's stride may be anything; over two it has to be a multiple of 16 bytes."""
    from paper_2609_15021_amd import attend, kvx
    cache = _cache(kvx, kvx.make_layout(1, 1, 64, 2, 16, 16))
    o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16)
    for tokens, heads, changes, fine in ((1, 1, dict(token_stride=129, head_stride=3), True),
                                         (1, 2, dict(token_stride=129), True), (2, 1, dict(head_stride=1), True),
                                         (1, 2, dict(head_stride=129), False), (2, 1, dict(token_stride=129), False)):
        b, q = _batch(attend, num_seqs=tokens, num_queries=tokens), _rows(attend, heads, **changes)
        need = kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(o), ctypes.byref(q))
        assert need >= 0 if fine else need == kvx.KV_EUNSUPPORTED, (tokens, heads, changes)


class _Answers:
    """Stands in for the library: every call succeeds, and the last one's arguments are kept."""

    name = args = None

    def __getattr__(self, name):
        def call(*args):
            self.name, self.args = name, args
            return 0
        return call


@pytest.fixture
def host_cache(monkeypatch):
    """(cache handle, library) for the binding's own work on host tensors."""
    from paper_2609_15021_amd import attend, kvx
    cache = object.__new__(kvx.Cache)
    cache.layout = kvx.make_layout(2, 2, 64, 1, 16, 16)
    cache.struct = _cache(kvx, cache.layout)
    cache.struct.device = -1  # where host tensors are
    lib = _Answers()
    monkeypatch.setattr(attend, "_lib", lib)
    monkeypatch.setattr(attend, "_call_stream", lambda stream: (None, attend._HERE))
    monkeypatch.setattr(attend, "_attend_bytes", {})
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    return cache, lib


def test_binding_takes_single_entries_with_any_stride(host_cache):
    """A batch of one cut from wider tensors: lengths, a table of one page, rows of one token, weights of one."""
    from paper_2609_15021_amd import attend
    cache, lib = host_cache
    meta = torch.zeros(1, 7, dtype=torch.int32)
    wide = torch.zeros(1, 3, 129, dtype=torch.bfloat16)
    q, k = wide[:, :2, :64], wide[:, 1:, :64]
    lens, table = meta[:, 3], meta[:, 1:2]
    assert lens.stride() == (7,)
    attend.kv_append(cache, 0, k, k, table.T.T, lens)
    assert lib.name == "kv_append"
    attend.kv_attend(cache, 0, q, torch.zeros(9, 1, dtype=torch.int32).T[:, :1], lens)
    assert lib.name == "kv_attend"
    attend.kv_keep(torch.zeros(1, 2, 5)[:, :, ::5], lens, 4)
    assert lib.name == "kv_keep"
    attend.kv_compact(cache, 0, table, torch.zeros(1, 1, 1, dtype=torch.int32), lens, table)
    assert lib.name == "kv_compact"
    two = torch.zeros(2, 7, dtype=torch.int32)
    with pytest.raises(TypeError, match="dense last dimension"):
        attend.kv_keep(torch.zeros(2, 2, 5), two[:, 3], 4)


def test_attend_refuses_rows_of_out_that_overlap():
    """Rows of q may be one and the same (a stride of 0), rows of out not."""
    from paper_2609_15021_amd import attend, kvx
    cache, batch = _cache(kvx, kvx.make_layout(1, 2, 64, 2, 16, 16)), _batch(attend)
    o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16)
    for changes in (dict(token_stride=0), dict(head_stride=0), dict(token_stride=56), dict(head_stride=32)):
        q, out = _rows(attend, 4, **changes), _rows(attend, 4)
        assert kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(o),
                                            ctypes.byref(q)) >= 0
        assert kvx._lib.kv_attend(ctypes.byref(cache), 0, ctypes.byref(batch), ctypes.byref(o), ctypes.byref(out),
                                  ctypes.byref(q), SOME, SOME, 1 << 40, None) == kvx.KV_EINVAL, changes
        assert b"rows of out" in kvx._lib.kv_last_error()
    nothing, rows = _batch(attend, num_seqs=0), _rows(attend, 4, token_stride=0, head_stride=0)
    assert kvx._lib.kv_attend(ctypes.byref(cache), 0, ctypes.byref(nothing), ctypes.byref(o), ctypes.byref(rows),
                              ctypes.byref(rows), None, SOME, 1 << 40, None) == kvx.KV_OK


def test_binding_refuses_factors_that_the_library_takes_for_defaults(host_cache):
    """0, and what is 0 in 32 bits, would be the default of the C ABI: 1 / sqrt(D), no cap, a scale of 1."""
    from paper_2609_15021_amd import attend
    cache, lib = host_cache
    rows, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    tables, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for options in (dict(scale=0.0), dict(scale=1e-50), dict(scale=-0.0), dict(softcap=1e-50), dict(softcap=-1e-60),
                    dict(k_scale=0.0), dict(v_scale=0), dict(k_scale=1e-46), dict(v_scale=-1e-46)):
        (name, value), = options.items()
        with pytest.raises(ValueError, match=name):
            attend.kv_attend(cache, 0, rows, tables, lens, **options)
        if name[1:] == "_scale":
            with pytest.raises(ValueError, match=name):
                attend.kv_append(cache, 0, kv, kv, tables, lens, **options)
    assert lib.name is None
    attend.kv_attend(cache, 0, rows, tables, lens, scale=0.25, softcap=0, k_scale=2, v_scale=1e-30)
    options = lib.args[3]._obj
    assert (options.scale, options.softcap, options.k_scale) == (0.25, 0.0, 2.0) and 0 < options.v_scale < 2e-30


def test_binding_refuses_numbers_beyond_32_bits(host_cache):
    """A window of 2^32 + 5 is none of 5 tokens, and layer 2^32 is not layer 0."""
    from paper_2609_15021_amd import attend
    cache, lib = host_cache
    rows, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    tables, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    weights, keep = torch.zeros(2, 2, 64), torch.zeros(2, 2, 4, dtype=torch.int32)
    calls = [lambda: attend.kv_append(cache, 2**32, kv, kv, tables, lens),
             lambda: attend.kv_attend(cache, 2**32 + 1, rows, tables, lens),
             lambda: attend.kv_attend(cache, 0, rows, tables, lens, window=2**32 + 5),
             lambda: attend.kv_attend(cache, 0, rows[:1].expand(2**32 + 2, 4, 64), tables, lens,
                                      torch.zeros(3, dtype=torch.int32)),
             lambda: attend.kv_keep(weights, lens, 2**32 + 4), lambda: attend.kv_keep(weights, lens, 4, sinks=2**32),
             lambda: attend.kv_keep(weights, lens, 4, recent=-2**33),
             lambda: attend.kv_compact(cache, -2**32, tables, keep, lens, tables)]
    for call in calls:
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert lib.name in (None, "kv_attend_workspace")  # which enqueues nothing
    attend.kv_attend(cache, 0, rows, tables, lens, max_len=2**40)
    assert lib.args[2]._obj.max_len == 64
    attend.kv_attend(cache, 0, rows, tables, lens, max_len=-2**32)
    assert lib.args[2]._obj.max_len == -1


def test_binding_refuses_what_requires_a_gradient(host_cache):
    """The operators have no backward pass: an output without one must not stand for it silently."""
    from paper_2609_15021_amd import attend
    cache, lib = host_cache
    q, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    leaf_q, leaf_kv = q.clone().requires_grad_(), kv.clone().requires_grad_()
    tables, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    weights, slopes = torch.zeros(2, 2, 64), torch.zeros(4)
    leaf_w, leaf_s = weights.clone().requires_grad_(), slopes.clone().requires_grad_()
    calls = [lambda: attend.kv_append(cache, 0, leaf_kv, kv, tables, lens),
             lambda: attend.kv_append(cache, 0, kv, leaf_kv * 2, tables, lens),
             lambda: attend.kv_attend(cache, 0, leaf_q, tables, lens),
             lambda: attend.kv_attend(cache, 0, q, tables, lens, out=leaf_q.clone()),
             lambda: attend.kv_attend(cache, 0, q, tables, lens, slopes=leaf_s),
             lambda: attend.kv_attend(cache, 0, q, tables, lens, weights=weights, prior=leaf_w + 1),
             lambda: attend.kv_keep(leaf_w, lens, 4)]
    for call in calls:
        with pytest.raises(RuntimeError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    attend.kv_attend(cache, 0, leaf_q.detach(), tables, lens, slopes=leaf_s.detach())


def test_full_weights_is_a_choice_of_two(host_cache):
    from paper_2609_15021_amd import attend, kvx
    cache, batch, rows = _cache(kvx, kvx.make_layout(1, 2, 64, 2, 16, 16)), _batch(attend), _rows(attend, 4)
    for fields, fine in ((dict(full_weights=1), True), (dict(full_weights=2), False), (dict(full_weights=-1), False),
                         (dict(reserved=1), False)):
        o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16, **fields)
        need = kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(o), ctypes.byref(rows))
        assert need >= 0 if fine else need == kvx.KV_EINVAL, fields
    handle, lib = host_cache
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    tables, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for full in (False, True):
        attend.kv_attend(handle, 0, q, tables, lens, full_weights=full)
        assert lib.args[3]._obj.full_weights == full


def test_tables_without_entries_need_no_address():
    """Sequences of no tokens: a table of no entries has no address in torch."""
    from paper_2609_15021_amd import attend, kvx
    cache, rows = _cache(kvx, kvx.make_layout(1, 2, 64, 2, 16, 16)), _rows(attend, 4)
    o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16)
    for fields, fine in ((dict(table_len=0, table_stride=0, max_len=0, block_tables=None), True),
                         (dict(table_len=1, table_stride=1, max_len=0, block_tables=None), False),
                         (dict(table_len=0, table_stride=0, max_len=0, block_tables=None, lens=None), False)):
        batch = _batch(attend, **fields)
        need = kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(o), ctypes.byref(rows))
        assert need >= 0 if fine else need == kvx.KV_EINVAL, fields


def test_workspace_of_the_widest_bounds():
    """Scores for everything that a call may name would take 2^67 bytes: more than a size holds, and none are kept."""
    from paper_2609_15021_amd import attend, kvx
    H, most = 16383, 2**31 - 1024
    cache = _cache(kvx, kvx.make_layout(1, H, 8, 2, 1, 1))
    q = _rows(attend, H, token_stride=H * 8, head_stride=8)
    need = []
    for weights_out in (None, SOME):
        b = _batch(attend, num_seqs=65535, max_queries=16, num_queries=16 * 65535, max_len=most, table_len=most,
                   table_stride=most, starts=SOME)
        o = attend.KvAttendOptions(cache_dtype=attend.KV_DTYPE_BF16, weights_out=weights_out,
                                   weights_seq_stride=most * H, weights_head_stride=most)
        need.append(kvx._lib.kv_attend_workspace(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(o),
                                                 ctypes.byref(q)))
    assert need[0] == need[1] > 0
