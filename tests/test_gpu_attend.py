"""The operators on a paged cache on the GPU, against their 64-bit forms (tests/attend_reference.py).

In every cache, slots without a token and pages without an owner hold NaN, and the unused entries of a block table are no
block at all: a kernel that let either in would show it.
"""
import itertools

import numpy as np
import pytest
import torch

import attend_reference as ref
from paper_2609_15021_amd import attend, kvx

pytestmark = pytest.mark.gpu
DEV = ref.DEV
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def no_faults():
    attend.kv_attend_async_error(clear=True)
    yield
    torch.cuda.synchronize()
    assert attend.kv_attend_async_error(clear=True) == 0


def run(c, options=None, weights=None, **kw):
    """kv_attend on a Case, checked against the reference; returns its outputs on the host."""
    options = dict(options or {})
    cache, _, q, _, _, tables, lens, starts = c.device()
    plain = dict(options)
    if plain.get("slopes") is not None:
        options["slopes"] = torch.tensor(plain["slopes"], dtype=torch.float32, device=DEV)
        plain["slopes"] = options["slopes"].double().cpu().numpy()
    want = ref.attend(c, **plain)
    longest = max(c.lens)
    w = prior = None
    if weights:
        prior = torch.rand(c.B, c.H, longest + 3, generator=torch.Generator().manual_seed(5)).to(DEV)
        w = prior if weights == "in_place" else torch.full_like(prior, -7.0)
        before = prior.clone()
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, k_scale=c.k_scale, v_scale=c.v_scale, weights=w,
                                prior=prior, **options, **kw)
    torch.cuda.synchronize()
    ref.check(lse, want[1], want[4], "lse")
    ref.check(out, want[0], want[3], "out")
    if weights:
        for b, n in enumerate(c.lens):
            expected = before[b, :, :n].double().cpu().numpy() + want[2][b, :, :n]
            ref.check(w[b, :, :n], expected, want[5][b, :, :n] + np.abs(expected) * 2.0**-24, "weights")
            left = before if weights == "in_place" else torch.full_like(before, -7.0)
            assert torch.equal(w[b, :, n:], left[b, :, n:])
    return out.cpu(), lse.cpu(), None if w is None else w.cpu()


# One new token per sequence: lengths around every size that a kernel may cut at, and odd ones.
LENS = [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 500, 1000, 1025]


@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,dtype", [
    (2, 1, 64, 16, False, False, BF16), (1, 5, 128, 16, False, False, BF16), (2, 8, 128, 32, True, False, F16),
    (2, 6, 256, 32, True, True, BF16), (1, 16, 64, 8, False, True, F16), (3, 4, 80, 24, True, False, BF16),
    (1, 17, 96, 16, False, False, F16), (2, 3, 192, 7, False, False, BF16), (1, 2, 16, 1, False, True, BF16),
    (1, 33, 128, 64, True, True, F16), (5, 2, 8, 3, False, False, F16), (1, 64, 256, 16, False, False, BF16),
    (2, 7, 112, 16, True, True, BF16), (1, 1, 248, 16, False, False, F16)])
def test_one_new_token(H, G, D, BS, nhd, fp8, dtype):
    c = ref.Case(H, G, D, BS, LENS, [1] * len(LENS), nhd=nhd, fp8=fp8, dtype=dtype, seed=D + G)
    run(c)


@pytest.mark.parametrize("weights", ["fresh", "in_place"])
@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,dtype", [(2, 5, 128, 16, False, False, BF16), (1, 6, 256, 32, True, True, BF16),
                                                    (2, 1, 64, 5, False, False, F16), (1, 20, 96, 16, True, False, BF16)])
def test_one_new_token_weights(H, G, D, BS, nhd, fp8, dtype, weights):
    c = ref.Case(H, G, D, BS, [1, 33, 64, 1000, 257], [1] * 5, nhd=nhd, fp8=fp8, dtype=dtype, seed=D + G)
    run(c, weights=weights)


OPTIONS = [dict(softcap=5.0), dict(window=1), dict(window=37), dict(window=100000), dict(slopes=True),
           dict(softcap=2.0, window=50, slopes=True, scale=0.3), dict(scale=2.0)]


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("H,G,D,fp8,new", [(2, 4, 64, False, [1, 1, 1, 1]), (1, 6, 128, True, [1, 3, 70, 2]),
                                            (2, 2, 128, False, [1, 200, 17, 64])])
def test_options(H, G, D, fp8, new, options):
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = [2.0**-(1 + i % 7) for i in range(H * G)]
    c = ref.Case(H, G, D, 16, [300, 200, 129, 64], new, fp8=fp8, seed=11)
    run(c, options, weights="fresh")


# Several new tokens: rows of a head group around the sizes of a tile, all of a sequence, and mixed with single ones.
@pytest.mark.parametrize("lens,new", [([40, 300, 7], [2, 3, 7]), ([70, 129], [70, 129]), ([600, 31], [33, 31]),
                                      ([1, 1000, 64, 90], [1, 1, 64, 2]), ([513], [256]), ([260, 255, 800], [130, 129, 5])])
@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,dtype", [
    (1, 1, 64, 16, False, False, BF16), (2, 5, 128, 16, False, False, BF16), (1, 6, 256, 32, True, True, BF16),
    (1, 3, 80, 24, True, False, F16), (2, 2, 192, 7, False, True, F16), (1, 16, 96, 1, False, False, BF16),
    (1, 20, 8, 16, True, False, F16)])
def test_several_new_tokens(H, G, D, BS, nhd, fp8, dtype, lens, new):
    c = ref.Case(H, G, D, BS, lens, new, nhd=nhd, fp8=fp8, dtype=dtype, seed=7 * D + G)
    run(c, weights="fresh")


@pytest.mark.parametrize("lens,new,window", [([3000], [70], 0), ([1300, 4100], [66, 90], 0), ([4100, 700], [129, 65], 300),
                                             ([2500, 100, 900], [3, 100, 1], 0)])
@pytest.mark.parametrize("H,G,D,fp8,dtype", [(1, 1, 128, False, BF16), (2, 2, 64, False, F16), (1, 3, 256, True, BF16),
                                              (1, 2, 200, False, BF16)])
def test_long_sequences_in_parts(H, G, D, fp8, dtype, lens, new, window):
    """Few rows over many tokens: they are split, and joined."""
    c = ref.Case(H, G, D, 16, lens, new, fp8=fp8, dtype=dtype, seed=D + G)
    run(c, dict(window=window), weights="fresh")


@pytest.mark.parametrize("softcap", [0.5, 64.0, 65.0, 3000.0])
def test_caps(softcap):
    """Small and large caps, where scores are far below and far above them."""
    for new in ([1, 1], [90, 70]):
        c = ref.Case(2, 2, 64, 16, [200, 100], new, seed=21, spread=6.0)
        run(c, dict(softcap=softcap, scale=1.0), weights="fresh")


def test_many_sequences():
    """Hundreds of sequences, long ones among short ones, and more than are shared out in parts."""
    gen = np.random.default_rng(3)
    lens = [int(n) for n in gen.integers(0, 60, 150)]
    lens[7], lens[70], lens[149] = 3000, 1500, 700
    c = ref.Case(2, 2, 64, 16, lens, [1 if n % 5 else 0 for n in lens], seed=22)
    run(c, weights="fresh")
    lens = [int(n) for n in gen.integers(0, 12, 1100)]
    lens[1000] = 400
    run(ref.Case(1, 2, 16, 4, lens, [1 + n % 2 for n in lens], seed=23))


@pytest.mark.parametrize("options", [{}, dict(softcap=5.0, window=90), dict(softcap=100.0)])
@pytest.mark.parametrize("fp8", [False, True])
def test_weights_of_many_tiles(fp8, options):
    """Received weights where the tokens alone fill the chip (2,280 tiles of 32), and of few tiles with many rows."""
    lens = [600] + [1 + 37 * i % 400 for i in range(29)]
    c = ref.Case(4, 5, 64, 16, lens, [min(n, 4 + i % 3) for i, n in enumerate(lens)], fp8=fp8, seed=61)
    run(c, options, weights="fresh")
    c = ref.Case(1, 5, 96, 16, [333, 40], [300, 7], fp8=fp8, seed=62)
    run(c, options, weights="in_place")


def test_weights_at_any_element():
    """Rows of weights that start at odd elements, of odd lengths."""
    for new in ([1, 1, 1], [30, 70, 1]):
        c = ref.Case(2, 3, 64, 16, [37, 90, 258], new, seed=24)
        cache, _, q, _, _, tables, lens, starts = c.device()
        wide = torch.rand(3, 2, 2, 263, device=DEV)
        before = wide.clone()
        view = wide[:, 1, :, 1:260]
        attend.kv_attend(cache, 0, q, tables, lens, starts, weights=view, prior=view, max_len=258)
        want = ref.attend(c)
        for b, n in enumerate(c.lens):
            expected = before[b, 1, :, 1:1 + n].double().cpu().numpy() + want[2][b, :, :n]
            ref.check(view[b, :, :n], expected, want[5][b, :, :n] + np.abs(expected) * 2.0**-24, "weights")
            assert torch.equal(wide[b, 1, :, 1 + n:], before[b, 1, :, 1 + n:])
        assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[..., 0], before[..., 0])


def test_rows_without_tokens():
    """Empty sequences, sequences without new tokens, and rows that would lie before token 0: 0 and -infinity."""
    for lens, new in (([0, 5, 0, 3], [1, 1, 0, 6]), ([0], [4]), ([2, 100], [130, 0]), ([0, 0], [0, 0]), ([3], [0])):
        c = ref.Case(2, 3, 64, 16, lens, new, seed=2)
        if max(lens):
            out, lse, _ = run(c, weights="fresh")
        else:
            cache, _, q, _, _, tables, ln, starts = c.device()
            out, lse = attend.kv_attend(cache, 0, q, tables, ln, starts)
        for b, (n, count) in enumerate(zip(lens, new)):
            empty = slice(int(c.starts[b]), int(c.starts[b]) + max(0, count - n))
            assert not out[empty].any() and torch.isinf(lse[empty]).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_no_starts_and_no_sequences(fp8):
    c = ref.Case(2, 4, 128, 16, [5, 40, 700], [1, 1, 1], fp8=fp8, seed=4)
    cache, _, q, k, v, tables, lens, starts = c.device()
    scales = dict(k_scale=c.k_scale, v_scale=c.v_scale)
    a = attend.kv_attend(cache, 0, q, tables, lens, starts, **scales)
    b = attend.kv_attend(cache, 0, q, tables, lens, **scales)
    tight = attend.kv_attend(cache, 0, q, tables, lens, max_len=700, **scales)
    want = ref.attend(c)
    for out, lse in (a, b, tight):
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")
    none = attend.kv_attend(cache, 0, q[:0], tables[:0], lens[:0], **scales)
    assert none[0].shape == (0, 8, 128) and none[1].shape == (0, 8)
    attend.kv_append(cache, 0, k[:0], v[:0], tables[:0], lens[:0], **scales)
    assert attend.kv_keep(torch.zeros(0, 2, 8, device=DEV), lens[:0], 4)[0].shape == (0, 2, 4)


def test_extreme_values():
    """Scores far apart and far from 0: no overflow, and the largest takes everything."""
    for dtype, fp8 in ((BF16, False), (F16, False), (BF16, True)):
        c = ref.Case(2, 4, 64, 16, [100, 1, 333], [1, 1, 60], dtype=dtype, fp8=fp8, seed=9)
        run(c, dict(scale=40.0), weights="fresh")
        run(c, dict(scale=1e-20), weights="fresh")


def test_many_small_weights():
    """One heavy token and thousands of light ones: what they add up to is not lost (float16 too)."""
    for dtype in (BF16, F16):
        n = 3000
        c = ref.Case(1, 2, 64, 16, [n], [1], dtype=dtype, seed=1)
        # The first token's key is along the query, the others' are 0: their weights are all exp(-12).
        cache, t, q, _, _, tables, lens, starts = c.device()
        block = t.view(c.num_blocks, 2, 1, 16, 64)
        block[:, 0] = 0
        block[int(c.tables[0, 0]), 0, 0, 0, 0] = 12.0
        block[:, 1] = 1.0
        block[int(c.tables[0, 0]), 1, 0, 0] = 0.0
        q[:] = 0
        q[:, :, 0] = 8.0  # score 12 for the first, 0 for the others
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts)
        rest = (n - 1) * np.exp(-12.0)
        want = rest / (1 + rest)
        assert abs(out.double() - want).max() <= want * 2 * ref.HALF_STEP[dtype] + want * n / 16 * 2.0**-23
        assert abs(lse.double() - (12 + np.log1p(rest))).max() <= 2.0**-18


def test_strides_and_rows_behind_the_last():
    """Views as q, out with strides of its own, weights inside a wider tensor; rows behind the last sequence stay."""
    c = ref.Case(2, 4, 128, 16, [50, 200], [3, 20], seed=6)
    cache, _, _, _, _, tables, lens, starts = c.device()
    extra = 5
    wide = torch.zeros(c.T + extra, 13, 2, 128, dtype=BF16, device=DEV)
    q = wide[:, 2:10, 1]
    q[:c.T] = c.q.to(DEV)
    out = torch.full((c.T + extra, 2, 8, 128), 9.0, dtype=BF16, device=DEV)
    lse = torch.full((c.T + extra, 8), 9.0, device=DEV)
    weights = torch.full((2, 5, 2, 300), 9.0, device=DEV)
    view = weights[:, 3]
    attend.kv_attend(cache, 0, q, tables, lens, starts, out=out[:, 1], lse=lse, weights=view, max_len=250)
    want = ref.attend(c)
    ref.check(out[:c.T, 1], want[0], want[3], "out")
    ref.check(lse[:c.T], want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(view[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")
        assert (view[b, :, n:] == 9).all()
    assert (out[c.T:] == 9).all() and (out[:, 0] == 9).all() and (lse[c.T:] == 9).all()
    for i in (0, 1, 2, 4):
        assert (weights[:, i] == 9).all()


@pytest.mark.parametrize("new", [[1, 1, 1], [2, 100, 30]])
def test_bad_pages_and_lengths(new):
    """A block id outside the cache is reported and its tokens take part in nothing; a sequence whose length or rows
    are out of bounds is left out; the others are as without them."""
    c = ref.Case(2, 4, 128, 16, [60, 300, 100], new, seed=8)
    c.tables[1, 3] = c.num_blocks
    c.tables[1, 0] = -1
    cache, _, q, k, v, tables, lens, starts = c.device()
    weights = torch.full((3, 2, 300), 3.0, device=DEV)
    prior = torch.zeros_like(weights)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, weights=weights, prior=prior)
    want = ref.attend(c, hidden_pages=[(1, 0), (1, 3)])
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")
    assert attend.kv_attend_async_error(clear=True) == kvx.KV_ASYNC_BAD_BLOCK
    good = ref.attend(c, hidden_pages=[(1, 0), (1, 3)])
    for wrong_lens, wrong_starts in (([60, -1, 100], None), ([60, 301, 100], None),
                                     (None, [0, new[0], c.T + 1, c.T + 1]), (None, [0, new[0], -1, c.T])):
        out = torch.full((c.T, 8, 128), 5.0, dtype=BF16, device=DEV)
        ln = lens if wrong_lens is None else torch.tensor(wrong_lens, dtype=torch.int32, device=DEV)
        st = starts if wrong_starts is None else torch.tensor(wrong_starts, dtype=torch.int32, device=DEV)
        weights.fill_(3.0)
        attend.kv_attend(cache, 0, q, tables, ln, st, max_len=300, out=out, weights=weights)
        assert attend.kv_attend_async_error(clear=True) & attend.KV_ASYNC_BAD_BATCH
        first = slice(0, new[0])
        ref.check(out[first], good[0][first], good[3][first], "out")
        if wrong_lens:
            assert (out[new[0]:new[0] + new[1]] == 5).all() and (weights[1] == 3).all()
            last = slice(new[0] + new[1], c.T)
            ref.check(out[last], good[0][last], good[3][last], "out")


def test_hidden_pages_are_not_looked_up():
    """Pages that a window hides from every new token may be gone: their entries in the table are not read."""
    for new in (1, 5, 100):
        c = ref.Case(1, 4, 64, 16, [500], [new], seed=12)
        first = max(0, 500 - new + 1 - 64) // 16
        c.tables[0, :first] = -5
        c.tables[0, -(-500 // 16):] = -5
        run(c, dict(window=64), weights="fresh")


@pytest.mark.parametrize("nhd", [False, True])
def test_cache_beyond_32_bits(nhd):
    """Pages more than 4 GiB apart."""
    BS, H, D = 16, 2, 128
    block = 2 * BS * H * D
    stride = 96 << 20  # elements: 192 MiB between blocks
    num = 40           # 7.5 GiB
    t = torch.empty(num * stride, dtype=BF16, device=DEV)
    pages = t.view(num, stride)[:, :block]
    c = ref.Case(H, 4, D, BS, [33 * 16 + 5], [1], nhd=nhd, seed=3)
    for j in range(34):
        pages[(j * 7 + 3) % num] = c.flat[int(c.tables[0, j]), :block].to(DEV)
    tables = torch.tensor([[(j * 7 + 3) % num for j in range(34)]], dtype=torch.int32, device=DEV)
    layout = kvx.make_layout(1, H, D, 2, BS, BS)
    cache = kvx.Cache([t], layout, num, block_stride_bytes=stride * 2,
                      block_order=kvx.KV_BLOCK_NHD if nhd else kvx.KV_BLOCK_HND)
    lens = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    want = ref.attend(c)
    for queries in (1, 40):
        if queries > 1:
            c2 = ref.Case(H, 4, D, BS, [33 * 16 + 5], [queries], nhd=nhd, seed=3)
            c2.k, c2.v = c.k, c.v
            want, q = ref.attend(c2), c2.q.to(DEV)
            starts = c2.starts.to(DEV)
        else:
            q, starts = c.q.to(DEV), None
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts)
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")
    # The last token again, and out to a fresh page at the far end.
    attend.kv_append(cache, 0, c.new_k.to(DEV), c.new_v.to(DEV), tables, lens)
    keep = torch.tensor([[[0, 7, 33 * 16 + 4]]], dtype=torch.int32, device=DEV)
    spare = next(i for i in range(num - 1, 0, -1) if i not in tables[0].tolist())
    attend.kv_compact(cache, 0, tables, keep, torch.tensor([3], dtype=torch.int32, device=DEV),
                      torch.tensor([[spare]], dtype=torch.int32, device=DEV))
    got = pages[spare].view(c.shape).cpu()
    got = got if nhd else got.transpose(1, 2)
    for j, token in enumerate((0, 7)):
        np.testing.assert_array_equal(got[0, j].double().numpy(), c.k[0][token])
        np.testing.assert_array_equal(got[1, j].double().numpy(), c.v[0][token])
    assert torch.equal(got[0, 2], c.new_k[0]) and torch.equal(got[1, 2], c.new_v[0])


def test_repeatable():
    """The same bits on every run."""
    for new in ([1, 1, 1], [100, 17, 3]):
        c = ref.Case(2, 5, 128, 16, [3000, 17, 900], new, seed=14)
        cache, _, q, _, _, tables, lens, starts = c.device()
        weights = torch.zeros(3, 2, 3000, device=DEV)
        first = [t.clone() for t in attend.kv_attend(cache, 0, q, tables, lens, starts, weights=weights)] + [weights.clone()]
        for _ in range(20):
            got = (*attend.kv_attend(cache, 0, q, tables, lens, starts, weights=weights), weights)
            for x, y in zip(first, got):
                assert torch.equal(x, y)


# ---- kv_append ----------------------------------------------------------------------------


@pytest.mark.parametrize("H,D,BS,nhd,fp8,dtype", list(itertools.chain(
    [(2, 64, 16, False, False, BF16), (3, 80, 7, True, False, F16), (1, 8, 1, False, False, BF16)],
    [(4, 256, 32, True, True, BF16), (2, 16, 5, False, True, F16)])))
def test_append(H, D, BS, nhd, fp8, dtype):
    """Rows land in their slots, rounded once; rows before token 0 and all other bytes of the cache stay."""
    c = ref.Case(H, 2, D, BS, [1, 40, 0, 100, 3, 64], [1, 17, 0, 100, 5, 1], nhd=nhd, fp8=fp8, dtype=dtype, seed=D,
                 stride_pad=16)
    cache, t, _, k, v, tables, lens, starts = c.device()
    k.mul_(3000.0 if fp8 else 1.0)  # beyond e4m3's range too
    v[0, 0, 0] = float("nan")
    before = t.clone()
    attend.kv_append(cache, 0, k, v, tables, lens, starts, k_scale=c.k_scale, v_scale=c.v_scale)
    want = before.cpu().view(torch.uint8 if fp8 else torch.int16).clone()
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            p, row = n - c.new[b] + i, int(c.starts[b]) + i
            if p < 0:
                continue
            page = want[int(c.tables[b, p // BS]), :2 * BS * H * D].view(c.shape)
            for kv, (rows, scale) in enumerate(((k, c.k_scale), (v, c.v_scale))):
                x = rows[row].cpu()
                if fp8:
                    x = (x.float() / np.float32(scale)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                else:
                    x = x.view(torch.int16)
                (page[kv, p % BS] if nhd else page[kv, :, p % BS]).copy_(x)
    got = t.cpu().view(want.dtype)
    if fp8:  # e4m3 has a NaN of each sign: 0x7f and 0xff
        got, want = (torch.where(x & 0x7f == 0x7f, 0x7f, x) for x in (got, want))
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_append_rounds_every_value(dtype):
    """All 65,536 values of a 2-byte type as e4m3, at scales that are exact and that are not."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).view(32, 8, 256)
    layout = kvx.make_layout(1, 8, 256, 1, 32, 32)
    t = torch.zeros(2, 2 * 32 * 8 * 256, dtype=torch.uint8, device=DEV)
    cache = kvx.Cache([t], layout, 2, block_order=kvx.KV_BLOCK_NHD)
    rows = every.to(DEV)
    tables = torch.tensor([[1]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([32], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 32], dtype=torch.int32, device=DEV)
    for k_scale, v_scale in ((1.0, 0.25), (0.037, 3.0e-5)):
        attend.kv_append(cache, 0, rows, rows, tables, lens, starts, k_scale=k_scale, v_scale=v_scale)
        got = t[1].cpu().view(2, 32, 8, 256)
        for kv, scale in enumerate((k_scale, v_scale)):
            x = every.float() / np.float32(scale)
            want = x.clamp(-448, 448).to(torch.float8_e4m3fn)
            nan = torch.isnan(x)
            assert torch.equal(got[kv][~nan], want.view(torch.uint8)[~nan])
            assert torch.isnan(got[kv].view(torch.float8_e4m3fn).float()[nan]).all()


# ---- kv_keep and kv_compact -----------------------------------------------------------------


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 4, 16), (64, 0, 64), (64, 32, 32),
                                                 (1000, 4, 100), (1000, 0, 0), (5000, 0, 1)])
def test_keep(budget, sinks, recent):
    """Ties by the thousand, zeros of both signs, infinities and NaN; lengths around the budget, 0 and 1."""
    gen = torch.Generator().manual_seed(budget + sinks)
    lens = [0, 1, 2, budget - 1, budget, budget + 1, 2 * budget + 1, 4097, 5003]
    L, H = 5100, 3
    lens = [min(n, L) for n in lens]
    w = torch.randn(len(lens), H, L, generator=gen)
    w[:, 1] = (w[:, 1] * 2).round() / 2          # few values
    w[:, 2] = torch.where(w[:, 2] > 1, w[:, 2], torch.zeros(()))
    w[:, 2, ::3] *= -0.0
    w[0::2, 1, 5::97] = float("nan")
    w[:, 0, 3::501] = float("inf")
    w[:, 0, 7::401] = float("-inf")
    device = w.to(DEV)
    got = attend.kv_keep(device, torch.tensor(lens, dtype=torch.int32, device=DEV), budget, sinks=sinks, recent=recent)
    want = ref.keep(w.numpy(), lens, budget, sinks, recent)
    assert torch.equal(got[0].cpu(), torch.from_numpy(want[0]))
    assert got[1].cpu().tolist() == want[1].tolist()
    assert np.array_equal(got[2].cpu().numpy(), want[2], equal_nan=True)


@pytest.mark.parametrize("budget", [1, 4096, 40000, 131000])
def test_keep_long(budget):
    """Rows of 131,077 tokens, one choice for all heads, in a strided view; and weights that are all alike."""
    L = 131077
    w = torch.rand(2, 3, L, generator=torch.Generator().manual_seed(1))
    w[1] = 0.5
    device = w.to(DEV)[:, 1:2]
    lens = torch.tensor([L, L - 5], dtype=torch.int32, device=DEV)
    keep, kept, kw = attend.kv_keep(device, lens, budget, sinks=budget // 8, recent=budget // 4)
    for b, n in enumerate((L, L - 5)):
        want = ref.keep(w[b:b + 1, 1:2, :].numpy(), [n], budget, budget // 8, budget // 4)
        assert torch.equal(keep[b:b + 1].cpu(), torch.from_numpy(want[0]))
        assert np.array_equal(kw[b:b + 1].cpu().numpy(), want[2])
    assert kept.cpu().tolist() == [budget, budget]


@pytest.mark.parametrize("seqs,heads,longest", [(65, 2, 9001), (1, 2, 17000), (128, 1, 8193)])
def test_keep_many_rows_and_pieces(seqs, heads, longest):
    """Rows that no longer fit one workgroup's registers: many of them, and few, with lengths around the pieces' edges."""
    gen = torch.Generator().manual_seed(longest)
    w = (torch.rand(seqs, heads, longest, generator=gen) * 50).round() / 50  # every value many times
    edges = [longest, 8192, 8193, 4096, 4097, 1, 0, 3, 700, 699]
    lens = [edges[i % len(edges)] for i in range(seqs)]
    got = attend.kv_keep(w.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), 700, sinks=3, recent=200)
    want = ref.keep(w.numpy(), lens, 700, 3, 200)
    assert torch.equal(got[0].cpu(), torch.from_numpy(want[0])) and got[1].cpu().tolist() == want[1].tolist()
    assert np.array_equal(got[2].cpu().numpy(), want[2])


@pytest.mark.parametrize("budget,sinks,recent", [(9000, 9000, 0), (9000, 0, 9000), (9000, 100, 8900), (9000, 8999, 0),
                                                 (9000, 8192, 100), (16384, 1, 8192)])
def test_keep_pieces(budget, sinks, recent):
    """Rows cut into pieces: nothing left to choose, first and last tokens that end at or inside a piece, NaN, infinities
    and ties in all of them, and lengths that leave pieces without a token."""
    L, H = 40000, 2
    lens = [40000, 32768, 16385, 9001, 9000, 0]
    w = torch.randn(len(lens), H, L, generator=torch.Generator().manual_seed(sinks))
    w[:, 1] = w[:, 1].round()
    w[1::2, :, ::7] = float("nan")
    w[:, :, 3::5001] = float("inf")
    w[:, :, 5::4001] = float("-inf")
    got = attend.kv_keep(w.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), budget, sinks=sinks, recent=recent)
    want = ref.keep(w.numpy(), lens, budget, sinks, recent)
    assert torch.equal(got[0].cpu(), torch.from_numpy(want[0])) and got[1].cpu().tolist() == want[1].tolist()
    assert np.array_equal(got[2].cpu().numpy(), want[2], equal_nan=True)


def test_keep_refuses_lengths_on_the_device():
    w = torch.rand(3, 1, 50, device=DEV)
    keep, kept, _ = attend.kv_keep(w, torch.tensor([51, 20, -1], dtype=torch.int32, device=DEV), 8)
    assert attend.kv_attend_async_error(clear=True) == attend.KV_ASYNC_BAD_BATCH
    want = ref.keep(w[1:2].cpu().numpy(), [20], 8, 0, 0)
    assert torch.equal(keep[1:2].cpu(), torch.from_numpy(want[0])) and int(kept[1]) == 8


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("H,D,E,BS,nhd", [(2, 64, 2, 16, False), (3, 80, 1, 7, True), (1, 4, 4, 1, False),
                                          (4, 256, 1, 32, True), (2, 128, 4, 24, False)])
def test_compact(H, D, E, BS, nhd, shared):
    gen = torch.Generator().manual_seed(D)
    lens, budget, num = [70, 5, 33, 0], 40, 500
    shape = (num, 2, BS, H, D * E) if nhd else (num, 2, H, BS, D * E)
    t = torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8)
    order = torch.randperm(num, generator=gen, dtype=torch.int32)
    width, fresh = -(-70 // BS), -(-budget // BS)
    tables = order[:4 * width].view(4, width)
    dst = order[4 * width:4 * width + 4 * fresh].view(4, fresh).clone()
    heads = 1 if shared else H
    keep = torch.full((4, heads, budget), -1, dtype=torch.int32)
    kept = [min(n, budget) - (1 if n > 1 else 0) for n in lens]
    for b, n in enumerate(lens):
        for h in range(heads):
            keep[b, h, :kept[b]] = torch.randperm(max(n, 1), generator=gen)[:kept[b]].sort().values.int()
        dst[b, -(-kept[b] // BS):] = -1  # unused entries are not read
    keep[0, 0, 1] = keep[0, 0, 0]        # a token named twice is read twice
    device = t.to(DEV)
    cache = kvx.Cache([device], kvx.make_layout(1, H, D, E, BS, BS), num,
                      block_order=kvx.KV_BLOCK_NHD if nhd else kvx.KV_BLOCK_HND)
    attend.kv_compact(cache, 0, tables.to(DEV), keep.to(DEV), torch.tensor(kept, dtype=torch.int32, device=DEV),
                      dst.to(DEV))
    want = t.clone()
    for b in range(4):
        for h in range(H):
            for j in range(kept[b]):
                token = int(keep[b, 0 if shared else h, j])
                src, to = int(tables[b, token // BS]), int(dst[b, j // BS])
                for kv in (0, 1):
                    if nhd:
                        want[to, kv, j % BS, h] = t[src, kv, token % BS, h]
                    else:
                        want[to, kv, h, j % BS] = t[src, kv, h, token % BS]
    assert torch.equal(device.cpu(), want)


def test_compact_reports_what_it_cannot_move():
    t = torch.randint(0, 256, (8, 2, 1, 16, 64), dtype=torch.uint8, device=DEV)
    before = t.clone()
    cache = kvx.Cache([t], kvx.make_layout(1, 1, 64, 1, 16, 16), 8)
    ints = dict(dtype=torch.int32, device=DEV)
    tables, dst = torch.tensor([[0, 99], [1, 2]], **ints), torch.tensor([[4], [5]], **ints)
    keep = torch.tensor([[[3, 20, 32, -1]], [[0, 1, 2, 3]]], **ints)
    attend.kv_compact(cache, 0, tables, keep, torch.tensor([4, 5], **ints), dst)
    assert attend.kv_attend_async_error(clear=True) == kvx.KV_ASYNC_BAD_BLOCK | attend.KV_ASYNC_BAD_BATCH
    before[4, :, :, 0] = before[0, :, :, 3]  # token 20 has no page, 32 and -1 are none, sequence 1 keeps too many
    assert torch.equal(t, before)


# ---- Streams, graphs, and all of them together --------------------------------------------------


def test_other_stream():
    """Everything on a stream that is not the current one, with temporaries that end before the work does."""
    c = ref.Case(2, 4, 128, 16, [300, 40], [1, 1], seed=15)
    want = ref.attend(c)
    s = torch.cuda.Stream()
    for handle in (s, s.cuda_stream):
        cache, _, q, k, v, tables, lens, starts = c.device()
        torch.cuda.synchronize()
        results = []
        for _ in range(8):
            if isinstance(handle, torch.cuda.Stream):
                results.append(attend.kv_attend(cache, 0, q.clone(), tables, lens, stream=handle))
            else:
                results.append(attend.kv_attend(cache, 0, q, tables, lens, stream=handle))
            if isinstance(handle, torch.cuda.Stream):
                s.wait_stream(torch.cuda.current_stream())
        torch.empty(1 << 20, device=DEV).fill_(1.0)
        s.synchronize()
        for out, lse in results[1:]:
            ref.check(out, want[0], want[3], "out")
            ref.check(lse, want[1], want[4], "lse")


def test_captured_step():
    """A decoding step captured once and replayed while the sequences grow, beside eager calls of the same kind."""
    lens0, steps = [30, 500, 1], 6
    c = ref.Case(2, 4, 128, 16, [n + steps for n in lens0], [1, 1, 1], seed=16)
    cache, t, _, _, _, tables, _, _ = c.device()
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.zeros(3, h, 128, dtype=BF16, device=DEV) for h in (8, 2, 2))
    lens = torch.tensor(lens0, dtype=torch.int32, device=DEV)
    weights = torch.zeros(3, 2, 512, device=DEV)

    def step():
        attend.kv_append(cache, 0, k, v, tables, lens, max_len=512)
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, max_len=512, weights=weights, prior=weights)
        return out, lse, *attend.kv_keep(weights, lens, 32, sinks=2, recent=8)

    lens += 1
    step()  # the library's first use of the device
    lens -= 1
    weights.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(other):
        second = attend.kv_attend(cache, 0, q, tables, lens, max_len=512)
    eager_weights = torch.zeros_like(weights)
    for i in range(steps):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen).to(BF16))
        lens += 1
        graph.replay()
        other.replay()
        got = [x.clone() for x in captured]
        torch.cuda.synchronize()
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, max_len=512, weights=eager_weights, prior=eager_weights)
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1]) and torch.equal(weights, eager_weights)
        assert torch.equal(second[0], out) and torch.equal(second[1], lse)
        for x, y in zip(attend.kv_keep(eager_weights, lens, 32, sinks=2, recent=8), got[2:]):
            assert torch.equal(x, y)
        # And against the definition, with the cache as it now is.
        now = ref.Case(2, 4, 128, 16, lens.tolist(), [1, 1, 1], seed=16)
        now.tables = c.tables
        flat = t.cpu()
        rows = [now.rows_of(flat, b, n) for b, n in enumerate(now.lens)]
        now.k, now.v, now.q = [r[0] for r in rows], [r[1] for r in rows], q.cpu()
        for b, n in enumerate(now.lens):
            assert np.array_equal(rows[b][0][n - 1], k[b].double().cpu().numpy())
        want = ref.attend(now)
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")


@pytest.mark.parametrize("fp8,nhd", [(False, False), (True, True)])
def test_restore_extend_decode_evict_publish(fp8, nhd):
    """As a replica uses them: a stored prefix is loaded into a fresh cache, the prompt's tail is appended and attends
    behind it, tokens are decoded with their weights accumulated, the cache is cut to a budget, decoding goes on, and
    what is kept is stored and loaded again."""
    H, G, D, BS, prefix, tail, budget = 2, 4, 128, 16, 512, 45, 200
    size, dtype = (1, torch.float8_e4m3fn) if fp8 else (2, BF16)
    scales = dict(k_scale=0.11, v_scale=0.07) if fp8 else {}
    c = ref.Case(H, G, D, BS, [prefix], [1], fp8=fp8, nhd=nhd, seed=17)
    source, _, _, _, _, table, _, _ = c.device()
    layout = kvx.make_layout(1, H, D, size, BS, 256)
    source = kvx.Cache([source._keep[0]], layout, c.num_blocks, block_order=source.struct.block_order)
    pool = kvx.kv_pool_create(layout, 4, "staged")
    kvx.kv_store(source, table[0].contiguous(), prefix, pool, [0, 1])
    num = 128
    t = torch.full((num, 2 * BS * H * D), float("nan"), device=DEV).to(dtype)
    cache = kvx.Cache([t], layout, num, block_order=source.struct.block_order)
    order = torch.randperm(num, generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(DEV)
    table = order[:64].contiguous()
    kvx.kv_load(cache, table, prefix, pool, [0, 1])
    tables = table.view(1, -1)
    gen = torch.Generator().manual_seed(2)

    def rows(n, heads):
        return torch.randn(n, heads, D, generator=gen).to(BF16).to(DEV)

    n = prefix
    ints = dict(dtype=torch.int32, device=DEV)
    weights = torch.zeros(1, H, 1024, device=DEV)

    def new_tokens(count):
        """Append `count` tokens and let them attend; both checked against the cache's contents."""
        nonlocal n
        n += count
        q, k, v = rows(count, H * G), rows(count, H), rows(count, H)
        lens, starts = torch.tensor([n], **ints), torch.tensor([0, count], **ints)
        attend.kv_append(cache, 0, k, v, tables, lens, starts, **scales)
        before = weights.clone()
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, max_len=1024, weights=weights, prior=weights,
                                    **scales)
        now = ref.Case(H, G, D, BS, [n], [count], fp8=fp8, nhd=nhd)
        now.k_scale, now.v_scale = scales.get("k_scale", 1.0), scales.get("v_scale", 1.0)
        now.tables = tables.cpu()
        held = now.rows_of(t.cpu(), 0, n)
        assert not np.isnan(held).any()
        now.k, now.v, now.q = [held[0]], [held[1]], q.cpu()
        want = ref.attend(now)
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")
        ref.check(weights[0, :, :n], before[0, :, :n].double().cpu().numpy() + want[2][0],
                  want[5][0] + 2.0**-23 * np.abs(want[2][0] + 1), "weights")
        return held

    first = new_tokens(tail)
    np.testing.assert_array_equal(first[0][:prefix], c.k[0])  # the restored prefix
    for _ in range(3):
        held = new_tokens(1)
    keep, kept, kept_weights = attend.kv_keep(weights, torch.tensor([n], **ints), budget, sinks=4, recent=32, max_len=n)
    want = ref.keep(weights[:, :, :n].cpu().numpy(), [n], budget, 4, 32)
    assert torch.equal(keep.cpu(), torch.from_numpy(want[0]))
    fresh = order[64:64 + -(-(budget + 16) // BS)].contiguous().view(1, -1)
    attend.kv_compact(cache, 0, tables, keep, kept, fresh)
    n, tables = int(kept), fresh
    weights = torch.zeros_like(weights)
    weights[:, :, :budget] = kept_weights
    now = ref.Case(H, G, D, BS, [n], [1], fp8=fp8, nhd=nhd)
    now.tables = tables.cpu()
    moved = now.rows_of(t.cpu(), 0, n)
    for h in range(H):
        np.testing.assert_array_equal(moved[:, :, h], held[:, keep[0, h].cpu().numpy(), h])
    for _ in range(2):
        held = new_tokens(1)
    # Publish what is kept, and take it into another cache.
    kvx.kv_store(cache, tables[0].contiguous(), n, pool, [2])
    t2 = torch.full((num, 2 * BS * H * D), float("nan"), device=DEV).to(dtype)
    other = kvx.Cache([t2], layout, num, block_order=source.struct.block_order)
    back = order[100:100 + -(-n // BS)].contiguous()
    kvx.kv_load(other, back, n, pool, [2])
    torch.cuda.synchronize()
    now = ref.Case(H, G, D, BS, [n], [1], fp8=fp8, nhd=nhd)
    now.tables = back.view(1, -1).cpu()
    np.testing.assert_array_equal(now.rows_of(t2.cpu(), 0, n), held)
