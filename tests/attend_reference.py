"""Plain 64-bit forms of the operators on a paged cache, and batches to try them on.

Everything here is host code written from the definitions in ``include/kvx_attend.h``: one sequence, one row, one head at
a time.  Slots of the cache that hold no token, and pages that no table names, hold NaN.
"""
from __future__ import annotations

import math

import numpy as np
import torch

DEV = torch.device("cuda:0")
HALF_STEP = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}


class Case:
    """A batch of sequences in a paged cache of one layer.  ``lens`` and ``new``: tokens and new tokens of each."""

    def __init__(self, H, G, D, BS, lens, new, *, nhd=False, dtype=torch.bfloat16, fp8=False, seed=0, stride_pad=0,
                 spread=1.5, pad_entry=2**30):
        self.H, self.G, self.D, self.BS, self.nhd, self.dtype, self.fp8 = H, G, D, BS, nhd, dtype, fp8
        self.lens, self.new = list(lens), list(new)
        self.B, self.T = len(self.lens), sum(self.new)
        self.k_scale, self.v_scale = (0.11, 0.07) if fp8 else (1.0, 1.0)
        gen = torch.Generator().manual_seed(seed)
        self.cache_dtype = torch.float8_e4m3fn if fp8 else dtype
        pages = [-(-n // BS) for n in self.lens]
        self.num_blocks = sum(pages) + 3
        order = torch.randperm(self.num_blocks, generator=gen).tolist()
        width = max(1, max(pages, default=0)) + 1
        self.tables = torch.full((self.B, width), pad_entry, dtype=torch.int32)
        self.starts = torch.tensor([0] + list(np.cumsum(self.new)), dtype=torch.int32)
        row = BS * H * D
        elems = 2 * row + stride_pad  # elements between blocks
        flat = torch.full((self.num_blocks, elems), math.nan).to(self.cache_dtype)
        shape = (2, BS, H, D) if nhd else (2, H, BS, D)
        at = 0
        self.k, self.v = [], []  # float64 [n][H][D], as stored (without the scales)
        for b, n in enumerate(self.lens):
            kv = torch.randn(2, n, H, D, generator=gen) * (8.0 if fp8 else 1.0)
            kv[0] *= spread
            kv = kv.to(self.cache_dtype)
            self.k.append(kv[0].double().numpy())
            self.v.append(kv[1].double().numpy())
            for j in range(pages[b]):
                block = order[at]
                at += 1
                self.tables[b, j] = block
                some = kv[:, j * BS:(j + 1) * BS]
                cut = flat[block, :2 * row].view(shape).clone()
                target = cut.view(torch.uint8) if fp8 else cut
                source = (some if nhd else some.transpose(1, 2)).contiguous()
                source = source.view(torch.uint8) if fp8 else source
                if nhd:
                    target[:, :some.shape[1]] = source
                else:
                    target[:, :, :some.shape[1]] = source
                (flat.view(torch.uint8) if fp8 else flat)[block, :2 * row] = target.reshape(-1)
        self.free = order[at:]
        self.flat, self.shape, self.elems = flat, shape, elems
        qkv = torch.randn(self.T, H * G + 2 * H, D, generator=gen).to(dtype)
        self.qkv = qkv
        self.q, self.new_k, self.new_v = qkv.split([H * G, H, H], dim=1)

    def device(self):
        """(kvx.Cache, its tensor, q, k, v views of one device tensor, tables, lens, starts)."""
        from paper_2609_15021_amd import kvx
        t = self.flat.to(DEV)
        layout = kvx.make_layout(1, self.H, self.D, t.element_size(), self.BS, self.BS)
        cache = kvx.Cache([t], layout, self.num_blocks, block_stride_bytes=self.elems * t.element_size(),
                          block_order=kvx.KV_BLOCK_NHD if self.nhd else kvx.KV_BLOCK_HND)
        q, k, v = self.qkv.to(DEV).split([self.H * self.G, self.H, self.H], dim=1)
        return (cache, t, q, k, v, self.tables.to(DEV), torch.tensor(self.lens, dtype=torch.int32).to(DEV),
                self.starts.to(DEV))

    def rows_of(self, flat, b, n):
        """[2][n][H][D] rows of sequence b's first n tokens in a copy of the cache (as stored values, float64)."""
        out = np.zeros((2, n, self.H, self.D))
        for t in range(n):
            page = flat[int(self.tables[b, t // self.BS]), :2 * self.BS * self.H * self.D].view(self.shape)
            x = page[:, t % self.BS] if self.nhd else page[:, :, t % self.BS]
            out[:, t] = x.double().numpy()
        return out


def attend(c: Case, *, scale=None, softcap=0.0, window=0, slopes=None, hidden_pages=()):
    """(out, lse, weights [B][H][longest], bounds of all three) in 64 bits.  ``hidden_pages``: (b, page) pairs whose
    tokens take part in nothing.

    The bounds count what a kernel with 32-bit sums and its weights exp(s - m) rounded to the rows' type may be off:
    a score by its D products' additions, each rounded (to 2^-23 of the sum of their magnitudes), and by a few roundings
    of its own size; the sums by one rounding per 16 tokens and a tree; the output by half a step of its type.
    """
    scale = 1.0 / math.sqrt(c.D) if scale is None else scale
    Hq, longest = c.H * c.G, max(c.lens, default=0)
    out, lse = np.zeros((c.T, Hq, c.D)), np.full((c.T, Hq), -np.inf)
    out_off, lse_off = np.zeros_like(out), np.zeros_like(lse)
    weights, weights_off = np.zeros((c.B, c.H, longest)), np.zeros((c.B, c.H, longest))
    half = HALF_STEP[c.dtype]
    q = c.q.double().numpy()
    for b, n in enumerate(c.lens):
        k, v = c.k[b] * c.k_scale, c.v[b] * c.v_scale
        t = np.arange(n)
        shown = np.ones(n, dtype=bool)
        for hb, page in hidden_pages:
            if hb == b:
                shown[page * c.BS:(page + 1) * c.BS] = False
        for i in range(c.new[b]):
            p, row = n - c.new[b] + i, int(c.starts[b]) + i
            seen = (t <= p) & shown
            if window:
                seen &= p - t < window
            if not seen.any():
                continue
            for head in range(Hq):
                h = head // c.G
                kk, vv, far = k[seen, h], v[seen, h], (p - t)[seen]
                s = scale * (kk @ q[row, head])
                off = scale * (np.abs(kk) @ np.abs(q[row, head])) * c.D * 2.0**-23 + np.abs(s) * 2.0**-22
                if softcap:
                    s = softcap * np.tanh(s / softcap)
                    off = off + softcap * 2.0**-22
                if slopes is not None:
                    s = s - slopes[head] * far
                    off = off + (np.abs(slopes[head] * far) + np.abs(s)) * 2.0**-23
                m = s.max()
                e = np.exp(s - m)
                total = e.sum()
                w = e / total
                lse[row, head] = m + np.log(total)
                out[row, head] = w @ vv
                # An error of a score is that share of its weight; s - m is rounded, and so is exp.
                off = off + (np.abs(s) + abs(m)) * 2.0**-23 + 2.0**-21
                far_off = float(w @ off)
                sums = (seen.sum() / 16 + 64) * 2.0**-23
                lse_off[row, head] = far_off + sums + (1 + abs(lse[row, head])) * 2.0**-22
                magnitude = w @ np.abs(vv)
                out_off[row, head] = (half * np.abs(out[row, head]) + half * magnitude + sums * magnitude +
                                      (w * off) @ np.abs(vv) + far_off * magnitude + 2.0**-25)
                got = np.zeros(n)
                got[seen] = w
                weights[b, h, :n] += got
                got[seen] = w * (off + lse_off[row, head])
                weights_off[b, h, :n] += got
        if n:
            weights_off[b, :, :n] += weights[b, :, :n] * (c.new[b] * c.G + 2) * 2.0**-24 + 2.0**-40
    return out, lse, weights, out_off, lse_off, weights_off


def check(got, want, off, what):
    """|got - want| <= off everywhere, infinities equal."""
    got = np.asarray(got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = got == want
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= off)
    if bad.any():
        at = tuple(int(x[0]) for x in np.nonzero(bad))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} are off; first at {at}: got {got[at]}, want "
                             f"{want[at]}, allowed {off[at]}")


def keep(weights, lens, budget, sinks, recent):
    """(keep, kept_lens, kept_weights) by sorting; weights [B][H][L] float32 numpy."""
    B, H, _ = weights.shape
    out = np.full((B, H, budget), -1, dtype=np.int32)
    kept_weights = np.zeros((B, H, budget), dtype=np.float32)
    for b, n in enumerate(lens):
        for h in range(H):
            if n <= budget:
                chosen = list(range(n))
            else:
                middle = range(sinks, n - recent)
                w = weights[b, h]
                ranked = sorted(middle, key=lambda t: (math.isnan(w[t]), 0.0 if math.isnan(w[t]) else -float(w[t]), t))
                chosen = sorted(list(range(sinks)) + ranked[:budget - sinks - recent] + list(range(n - recent, n)))
            out[b, h, :len(chosen)] = chosen
            kept_weights[b, h, :len(chosen)] = weights[b, h, chosen]
    return out, np.minimum(lens, budget).astype(np.int32), kept_weights
