"""Plain 64-bit forms of rotation, scaled pages, bounds of pages and attention over chosen pages, and batches with scales.

Host code from the definitions in ``include/kvx_attend.h``, one row and head at a time, beside ``attend_reference.py``,
whose batches these are: slots without a token and pages without an owner hold NaN, and unused scales are no scale.
"""
from __future__ import annotations

import math

import numpy as np
import torch

import attend_reference as ref

E4M3 = torch.float8_e4m3fn


class ScaledCase(ref.Case):
    """A batch in e4m3 pages with scales of 2^-7 to 2^-2; 255, which is no scale, where no page has an owner."""

    def __init__(self, *args, exponents=(120, 126), **kw):
        super().__init__(*args, fp8=True, **kw)
        gen = torch.Generator().manual_seed(kw.get("seed", 0) + 1)
        self.k_scale = self.v_scale = 1.0
        self.scales = torch.full((self.num_blocks, 2, self.H), 255, dtype=torch.uint8)
        for b, n in enumerate(self.lens):
            for j in range(-(-n // self.BS)):
                self.scales[int(self.tables[b, j])] = torch.randint(*exponents, (2, self.H), generator=gen).to(torch.uint8)
            page = self.tables[b, torch.arange(n) // self.BS].long()
            by = torch.pow(2.0, self.scales[page].double() - 127).numpy()  # [n][2][H]
            self.k[b], self.v[b] = self.k[b] * by[:, 0, :, None], self.v[b] * by[:, 1, :, None]


def choose(c, budget, heads, seed, *, also_first=True):
    """(pages [tokens][heads][budget], counts) at random, in any order, each new token's own page among them; entries
    beyond a count are no page."""
    gen = np.random.default_rng(seed)
    pages = np.full((c.T, heads, budget), 2**30, dtype=np.int32)
    counts = np.zeros(c.T, dtype=np.int32)
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            row, own = int(c.starts[b]) + i, max(n - c.new[b] + i, 0) // c.BS
            counts[row] = min(own + 1, budget)
            for h in range(heads):
                some = gen.permutation(own)[:counts[row] - 1]
                pages[row, h, :counts[row]] = gen.permutation(np.append(some, own))
    return torch.from_numpy(pages), torch.from_numpy(counts)


def attend_chosen(c, pages, counts, *, scale=None, softcap=0.0, window=0, slopes=None):
    """(out, lse, bounds of both) of attention over chosen pages; the bounds as attend_reference.attend's, but for weights
    as two numbers of their type, whose rounding (2^-16 of a weight) takes the place of half a step."""
    scale = 1.0 / math.sqrt(c.D) if scale is None else scale
    Hq = c.H * c.G
    out, lse = np.zeros((c.T, Hq, c.D)), np.full((c.T, Hq), -np.inf)
    out_off, lse_off = np.zeros_like(out), np.zeros_like(lse)
    half = ref.HALF_STEP[c.dtype]
    q = c.q.double().numpy()
    for b, n in enumerate(c.lens):
        k, v = c.k[b] * c.k_scale, c.v[b] * c.v_scale
        for i in range(c.new[b]):
            p, row = n - c.new[b] + i, int(c.starts[b]) + i
            for head in range(Hq):
                h = head // c.G
                chosen = pages[row, h if pages.shape[1] > 1 else 0, :int(counts[row])].tolist()
                t = np.array([j * c.BS + s for j in chosen for s in range(c.BS)], dtype=np.int64)
                t = t[(t <= p) & (t >= 0)]
                if window:
                    t = t[p - t < window]
                if not t.size:
                    continue
                kk, vv, far = k[t, h], v[t, h], p - t
                s = scale * (kk @ q[row, head])
                off = scale * (np.abs(kk) @ np.abs(q[row, head])) * c.D * 2.0**-23 + np.abs(s) * 2.0**-21
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
                off = off + (np.abs(s) + abs(m)) * 2.0**-23 + 2.0**-21
                far_off = float(w @ off)
                sums = (t.size / 16 + 64) * 2.0**-23
                lse_off[row, head] = far_off + sums + (1 + abs(lse[row, head])) * 2.0**-22
                magnitude = w @ np.abs(vv)
                out_off[row, head] = (half * np.abs(out[row, head]) + (2.0**-15 + sums) * magnitude +
                                      (w * off) @ np.abs(vv) + far_off * magnitude + 2.0**-25)
    return out, lse, out_off, lse_off


def rotated(x, position, freqs, *, weight=None, eps=0.0, offset=0.0, interleaved=False, magnitude=1.0):
    """(rows, bounds without the last rounding) of x [..., D] (float64), normed and rotated by one position.

    Bounds: a norm's sum of D squares is off by 13 roundings in a row (8 in a lane, 5 between lanes), half of which its
    root keeps, and the mean, eps, root, quotient and two products by one each: under 2^-20 in all; a cosine by 2^-21 (two
    units of the last place of one in 32 bits, its argument, and magnitude) and by the angle's error, 2^-52 of the
    angle in turns twice; the two products and their sum by 2^-22 of what goes into them.
    """
    D, half = x.shape[-1], len(freqs)
    y = x.astype(np.float64)
    norm = 0.0
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * (offset + weight)
        norm = 2.0**-20
    out, off = y.copy(), norm * np.abs(y)
    angle = position * np.asarray(freqs, dtype=np.float64)
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    i = np.arange(half)
    left, right = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = y[..., left], y[..., right]
    out[..., left], out[..., right] = a * c - b * s, b * c + a * s
    share = magnitude * (norm + 2.0**-21 + 2.0**-22 + np.abs(angle) * 2.0**-51)
    off[..., left] = off[..., right] = (np.abs(a) + np.abs(b)) * share
    assert D >= 2 * half
    return out, off


def exponent(most):
    """The exponent byte of the smallest power of two that most <= 448 * 2^(e - 127) holds for."""
    e = 1
    while e < 254 and most > 448.0 * 2.0**(e - 127):
        e += 1
    return e


def append_scaled(c, flat, scales, k, v):
    """The cache (a copy of `flat`, e4m3) and scales after kv_append_scaled of rows k, v [tokens][H][D]."""
    flat, scales = flat.clone(), scales.clone()
    for b, n in enumerate(c.lens):
        first = n - c.new[b]
        for page in range(max(first, 0) // c.BS, -(-n // c.BS)) if n and c.new[b] else ():
            t0, t1 = max(first, page * c.BS, 0), min(n, (page + 1) * c.BS)
            block, old = int(c.tables[b, page]), t0 - page * c.BS
            for kv, rows in ((0, k), (1, v)):
                x = rows[int(c.starts[b]) + t0 - first:int(c.starts[b]) + t1 - first].double()
                for h in range(c.H):
                    y = x[:, h]
                    finite = y[torch.isfinite(y)].abs()
                    before = int(scales[block, kv, h]) if old else 0
                    e = max(exponent(float(finite.max()) if finite.numel() else 0.0), before)
                    slot = flat[block, :2 * c.BS * c.H * c.D].view(c.shape)
                    held = slot[kv, :, h] if c.nhd else slot[kv, h]
                    if old and e > before:
                        held.view(torch.uint8)[:old] = (held[:old].double() * 2.0**(before - e)).to(E4M3).view(torch.uint8)
                    stored = (y * 2.0**(127 - e)).clamp(-448.0, 448.0).to(E4M3)
                    held.view(torch.uint8)[old:old + t1 - t0] = stored.view(torch.uint8)
                    scales[block, kv, h] = e
    return flat, scales


def bounds(c, flat):
    """[blocks][2][H][D] lowest and highest K of the pages that new tokens lie in (float64, NaN elsewhere)."""
    out = np.full((c.num_blocks, 2, c.H, c.D), np.nan)
    for b, n in enumerate(c.lens):
        for page in range(max(n - c.new[b], 0) // c.BS, -(-n // c.BS)) if n and c.new[b] else ():
            block = int(c.tables[b, page])
            slot = flat[block, :2 * c.BS * c.H * c.D].view(c.shape)[0].double().numpy()
            x = (slot if c.nhd else slot.transpose(1, 0, 2))[:min(c.BS, n - page * c.BS)]  # [rows][H][D]
            none = np.isnan(x).all(0)
            low, high = np.where(np.isnan(x), np.inf, x).min(0), np.where(np.isnan(x), -np.inf, x).max(0)
            out[block, 0], out[block, 1] = np.where(none, 0.0, low), np.where(none, 0.0, high)
    return out


def scores(c, low_high, factors=None, scale=1.0):
    """(scores [tokens][H][pages], their bounds, counts); low_high [blocks][2][H][D], factors [blocks][H]."""
    width = c.tables.shape[1]
    out = np.full((c.T, c.H, width), np.nan)
    off = np.zeros_like(out)
    counts = np.zeros(c.T, dtype=np.int32)
    q = c.q.double().numpy()
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            p, row = n - c.new[b] + i, int(c.starts[b]) + i
            counts[row] = p // c.BS + 1 if p >= 0 else 0
            for j in range(counts[row]):
                block = int(c.tables[b, j])
                for h in range(c.H):
                    x = q[row, h * c.G:(h + 1) * c.G]
                    by = scale * (1.0 if factors is None else factors[block, h])
                    low, high = low_high[block, 0, h], low_high[block, 1, h]
                    out[row, h, j] = by * np.maximum(x * low, x * high).sum(-1).max()
                    # 2 D products, exact, and as many additions in 32 bits.
                    sums = (np.maximum(x, 0) * np.abs(high) + np.abs(np.minimum(x, 0) * low)).sum(-1).max()
                    off[row, h, j] = by * sums * (2 * c.D + 4) * 2.0**-23
    return out, off, counts
