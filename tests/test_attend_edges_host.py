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
