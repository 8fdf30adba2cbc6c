"""Edges of the operators on the paged cache on the CPU: workspaces, and what is refused before any HIP call."""
import ctypes

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
