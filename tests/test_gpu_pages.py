"""Rotation, scaled pages, bounds and scores of pages, and attention over chosen pages on the GPU, against their 64-bit
forms (tests/pages_reference.py).

As in test_gpu_attend.py, slots without a token and pages without an owner hold NaN, unused entries of tables and lists are no
block and no page, and unused scales are no scale.
"""
import contextlib

import numpy as np
import pytest
import torch

import attend_reference as ref
import pages_reference as pref
from paper_2609_15021_amd import attend, kvx

pytestmark = pytest.mark.gpu
DEV = ref.DEV
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def no_faults():
    attend.kv_attend_async_error(clear=True)
    yield
    torch.cuda.synchronize()
    assert attend.kv_attend_async_error(clear=True) == 0


@contextlib.contextmanager
def fault(bit):
    """The device reports this one fault."""
    yield
    torch.cuda.synchronize()
    assert attend.kv_attend_async_error(clear=True) == bit


def same_bytes(got, want, what):
    """(NaN stays NaN: of e4m3's two, 0x7f and 0xff, either.)"""
    nan = got.dtype == E4M3
    got, want = got.cpu().contiguous().view(torch.uint8), want.contiguous().view(torch.uint8)
    if nan:
        got, want = (torch.where(x == 0xff, 0x7f, x) for x in (got, want))
    bad = (got != want).nonzero()
    assert not len(bad), f"{what}: {len(bad)} bytes differ, first at {bad[0].tolist()}"


LENS = [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 500, 1000, 1025]


# ---- Rotation -----------------------------------------------------------------------------


def run_rotate(c, *, rotary=None, norm="both", interleaved=False, positions=None, magnitude=1.0, offset=0.0,
               weight_dtype=torch.float32, in_place=False, scales=None, base=10000.0, **kw):
    D, half = c.D, (c.D if rotary is None else rotary) // 2
    cache, flat, q, k, v, tables, lens, starts = c.device()
    gen = torch.Generator().manual_seed(9)
    weights = (1 + 0.2 * torch.randn(2, D, generator=gen)).to(weight_dtype)
    qw, kw_ = (w if on else None for w, on in zip(weights, (norm in ("both", "q"), norm in ("both", "k"))))
    freqs = base ** (-np.arange(half) / max(half, 1))
    options = dict(freqs=torch.tensor(freqs, dtype=torch.float64).to(DEV) if half else None, magnitude=magnitude,
                   positions=None if positions is None else torch.tensor(positions, dtype=torch.int32).to(DEV),
                   q_weight=None if qw is None else qw.to(DEV), k_weight=None if kw_ is None else kw_.to(DEV), eps=1e-5,
                   weight_offset=offset, interleaved=interleaved, k_scale=0.5 if c.fp8 and scales is None else 1.0,
                   v_scale=0.25 if c.fp8 and scales is None else 1.0)
    by = None if scales is None else scales.to(DEV)
    got = attend.kv_rotate(cache, 0, q, k, v, tables, lens, starts, scales=by, out=q if in_place else None, **options,
                           **kw)
    torch.cuda.synchronize()
    assert (got.data_ptr() == q.data_ptr()) == in_place
    out, out_off = np.zeros((c.T, c.H * c.G, D)), np.zeros((c.T, c.H * c.G, D))
    kk, kk_off = np.zeros((c.T, c.H, D)), np.zeros((c.T, c.H, D))
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            row = int(c.starts[b]) + i
            p = n - c.new[b] + i if positions is None else positions[row]
            more = dict(eps=1e-5, offset=offset, interleaved=interleaved, magnitude=magnitude)
            out[row], out_off[row] = pref.rotated(c.q[row].double().numpy(), p, freqs,
                                                  weight=None if qw is None else qw.double().numpy(), **more)
            kk[row], kk_off[row] = pref.rotated(c.new_k[row].double().numpy(), p, freqs,
                                                weight=None if kw_ is None else kw_.double().numpy(), **more)
    half_step = ref.HALF_STEP[c.dtype]
    ref.check(got, out, out_off + half_step * (np.abs(out) + out_off) + 2.0**-25, "q")
    # The cache: K within a rounding, V as it is, everything else untouched.
    after = flat.cpu()
    want = c.flat.clone()
    written = torch.zeros(c.flat.shape, dtype=torch.bool)
    for b, n in enumerate(c.lens):
        for i in range(c.new[b]):
            t, row = n - c.new[b] + i, int(c.starts[b]) + i
            if t < 0:
                continue
            block, slot = int(c.tables[b, t // c.BS]), t % c.BS
            flat_rows = 2 * c.BS * c.H * c.D
            at = lambda x, kv: (x[block, :flat_rows].view(c.shape)[kv, slot] if c.nhd  # noqa: E731
                                else x[block, :flat_rows].view(c.shape)[kv, :, slot])
            at(written, 0)[:] = True
            at(written, 1)[:] = True
            stored_k, stored_v = at(after, 0).double().numpy(), at(after, 1)
            if not c.fp8:
                ref.check(stored_k, kk[row], kk_off[row] + half_step * (np.abs(kk[row]) + kk_off[row]) + 2.0**-25, "k")
                same_bytes(stored_v, c.new_v[row], "v")
            elif scales is None:
                wide, off = np.clip(kk[row] / 0.5, -448, 448), kk_off[row] / 0.5
                ref.check(stored_k, wide, off + 2.0**-4 * (np.abs(wide) + off) + 2.0**-10, "k")
                want_v = (c.new_v[row].float() / 0.25).clamp(-448, 448).to(E4M3)
                same_bytes(stored_v, want_v, "v")
            else:
                factor = torch.pow(2.0, by[block].double() - 127).cpu().numpy()[:, :, None]
                off = kk_off[row] * (1 + 2.0**-4) + 2.0**-4 * np.abs(kk[row]) + 2.0**-10 * factor[0]
                ref.check(stored_k * factor[0], kk[row], off, "k")
                want_v = (c.new_v[row].double() / torch.from_numpy(factor[1])).clamp(-448, 448).to(E4M3)
                same_bytes(stored_v, want_v, "v")
    if scales is None:
        keep = ~written
        assert torch.equal(after.view(torch.uint8 if c.fp8 else torch.int16)[keep],
                           want.view(torch.uint8 if c.fp8 else torch.int16)[keep])
    else:
        # Scales and older rows are exact.
        wanted, wanted_scales = pref.append_scaled(c, c.flat, scales, torch.from_numpy(kk), c.new_v)
        assert torch.equal(by.cpu(), wanted_scales)  # (no page's largest K is next to a border here)
        untouched = ~written
        same = after.view(torch.uint8) == wanted.view(torch.uint8)
        assert bool(same[untouched].all())
    return got


@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,dtype", [
    (2, 1, 64, 16, False, False, BF16), (1, 5, 128, 16, False, False, BF16), (2, 6, 256, 32, True, True, BF16),
    (1, 16, 64, 8, False, True, F16), (3, 4, 80, 24, True, False, BF16), (1, 17, 96, 16, False, False, F16),
    (2, 3, 192, 7, False, False, BF16), (1, 2, 16, 1, False, True, F16), (5, 2, 8, 3, False, False, F16),
    (1, 1, 248, 16, False, False, F16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_one_new_token(H, G, D, BS, nhd, fp8, dtype, interleaved):
    c = ref.Case(H, G, D, BS, LENS, [1] * len(LENS), nhd=nhd, fp8=fp8, dtype=dtype, seed=D + G)
    run_rotate(c, interleaved=interleaved)


@pytest.mark.parametrize("rotary", [2, 20, 32, 48, 64, 0])
@pytest.mark.parametrize("norm", ["both", "q", "k", "none"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_columns(rotary, norm, interleaved):
    """Parts of a row, pairs that lie in other lanes' columns, and norms of one operand alone."""
    c = ref.Case(2, 3, 64, 16, [5, 40], [3, 20], seed=rotary)
    run_rotate(c, rotary=rotary, norm=norm, interleaved=interleaved)


@pytest.mark.parametrize("lens,new", [([40, 300, 7], [2, 3, 7]), ([600, 31, 0, 9], [533, 31, 0, 1]), ([1100], [1100]),
                                      ([3, 5], [6, 5])])
@pytest.mark.parametrize("fp8", [False, True])
def test_rotate_many(lens, new, fp8):
    """Tails, whole prompts, and rows that would lie before token 0, which have no slot."""
    c = ref.Case(2, 2, 128, 16, lens, new, fp8=fp8, nhd=fp8, seed=3)
    run_rotate(c, magnitude=1.25, offset=1.0, weight_dtype=BF16)


@pytest.mark.parametrize("rotary", [20, 32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_keeps_infinities_in_place(rotary, interleaved):
    """Without a norm an infinity or NaN reaches its own column and its partner's, and no other."""
    c = ref.Case(1, 1, 64, 16, [9], [1], seed=1)
    cache, _, _, _, _, tables, lens, _ = c.device()
    freqs = torch.full((rotary // 2,), 0.1, dtype=torch.float64, device=DEV)
    for column in (0, 7, rotary - 1, rotary, rotary + 1, 63):
        q = torch.ones(1, 1, 64, dtype=BF16, device=DEV)
        q[0, 0, column] = float("inf") if column % 2 else float("nan")
        half = rotary // 2
        partner = column ^ 1 if interleaved else column + half if column < half else column - half
        hit = {column, partner} if column < rotary else {column}
        got = attend.kv_rotate(cache, 0, q, q, q, tables, lens, freqs=freqs, interleaved=interleaved)
        assert set((~torch.isfinite(got[0, 0])).nonzero().view(-1).tolist()) == hit


@pytest.mark.parametrize("in_place", [False, True])
def test_rotate_far_positions(in_place):
    """Positions of their own, up to the largest."""
    c = ref.Case(1, 4, 64, 16, [50, 8], [6, 2], seed=5)
    run_rotate(c, positions=[0, 131071, 10**6, 2**31 - 1, 77, 2**24 + 1, -5, -2**31], in_place=in_place)


@pytest.mark.parametrize("lens,new", [([40, 300, 7], [2, 3, 7]), ([260], [129]), ([5, 17, 64], [1, 1, 1])])
@pytest.mark.parametrize("H,G,D,BS,nhd,rotary,interleaved", [(2, 2, 64, 16, False, 64, False), (1, 3, 128, 8, True, 20, False),
                                                             (2, 1, 256, 64, True, 128, True), (1, 2, 80, 24, False, 0, False)])
def test_rotate_into_scaled_pages(lens, new, H, G, D, BS, nhd, rotary, interleaved):
    c = pref.ScaledCase(H, G, D, BS, lens, new, nhd=nhd, seed=D)
    run_rotate(c, rotary=rotary, interleaved=interleaved, scales=c.scales)


# ---- Rows into scaled pages ---------------------------------------------------------------


def run_append(c, k, v):
    cache, flat, _, _, _, tables, lens, starts = c.device()
    by = c.scales.to(DEV)
    want, want_scales = pref.append_scaled(c, c.flat, c.scales, k, v)
    attend.kv_append(cache, 0, k.to(DEV), v.to(DEV), tables, lens, starts, scales=by)
    torch.cuda.synchronize()
    assert torch.equal(by.cpu(), want_scales)
    same_bytes(flat, want, "cache")
    return flat, by


@pytest.mark.parametrize("lens,new", [(LENS, [1] * len(LENS)), ([40, 300, 7, 0, 64], [2, 3, 7, 0, 64]), ([700], [533]),
                                      ([3, 5], [6, 5]), ([70, 65], [1, 33])])
@pytest.mark.parametrize("H,G,D,BS,nhd,dtype", [(2, 1, 64, 16, False, BF16), (4, 1, 256, 32, True, BF16),
                                                (1, 1, 128, 200, False, F16), (3, 1, 80, 7, True, BF16),
                                                (1, 1, 16, 1, False, F16), (2, 1, 256, 300, False, BF16)])
def test_append_scaled(H, G, D, BS, nhd, dtype, lens, new):
    c = pref.ScaledCase(H, G, D, BS, lens, new, nhd=nhd, dtype=dtype, seed=D + BS)
    gen = torch.Generator().manual_seed(1)
    # Magnitudes over eight decades, by row: scales grow, stay and fall to a fresh page's own.
    size = 10.0 ** (torch.rand(c.T, 1, 1, generator=gen) * 8 - 5)
    run_append(c, (c.new_k.float() * size).clamp(-6e4, 6e4).to(dtype), (c.new_v.float() * size).clamp(-6e4, 6e4).to(dtype))


def test_append_scaled_edges():
    """Rows of zeros, the largest and smallest numbers, exact borders, infinities and NaN."""
    c = pref.ScaledCase(1, 1, 16, 4, [12, 5, 9, 4, 30], [4, 1, 5, 4, 8], seed=2)
    k, v = torch.zeros(c.T, 1, 16, dtype=BF16), torch.zeros(c.T, 1, 16, dtype=BF16)
    k[4, 0, 3], k[5, 0, 0], k[6, 0, 1] = 448.0, 450.0, -448.0 * 2.0**-20
    k[10, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1.0])
    k[11, 0, 0] = 3.3e38
    k[14:22, 0, 5] = torch.tensor([2.0**-130, 1e-38, 1e-30, 0.0, 7.0, -7.0, 7.03125, float("inf")])
    v[0:4, 0, 0] = float("nan")
    run_append(c, k, v)


def test_append_step_by_step():
    """A page filled a token at a time holds what filling it at once would, but for what its older rows lost."""
    c = pref.ScaledCase(2, 1, 64, 16, [16], [16], seed=4)
    gen = torch.Generator().manual_seed(3)
    rows = (torch.randn(16, 2, 64, generator=gen) * torch.exp2(torch.arange(16) / 2).view(-1, 1, 1)).to(BF16)
    at_once, by = run_append(c, rows, rows)
    cache, flat, _, _, _, tables, _, _ = c.device()
    scales = c.scales.to(DEV)
    for n in range(1, 17):
        lens = torch.tensor([n], dtype=torch.int32, device=DEV)
        attend.kv_append_scaled(cache, 0, rows[n - 1:n].to(DEV), rows[n - 1:n].to(DEV), tables, lens, scales)
    torch.cuda.synchronize()
    assert torch.equal(scales.cpu(), by.cpu())
    block = int(c.tables[0, 0])
    x, y = flat[block].float().cpu(), at_once[block].float().cpu()
    # Values that were rounded in e4m3's normal numbers only are the same; others are within a step of the smallest,
    # 2^-9, and halves of it that each growth adds: under 2^-8.
    assert bool(((x == y) | ((x - y).abs() <= 2.0**-8)).all())


# ---- Attention over scaled pages ----------------------------------------------------------


def run_scaled(c, options=None, **kw):
    options = dict(options or {})
    cache, _, q, _, _, tables, lens, starts = c.device()
    plain = dict(options)
    if plain.get("slopes") is not None:
        options["slopes"] = torch.tensor(plain["slopes"], dtype=torch.float32, device=DEV)
        plain["slopes"] = options["slopes"].double().cpu().numpy()
    want = ref.attend(c, **plain)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, scales=c.scales.to(DEV), **options, **kw)
    torch.cuda.synchronize()
    ref.check(lse, want[1], want[4], "lse")
    ref.check(out, want[0], want[3], "out")
    return out, lse


@pytest.mark.parametrize("lens,new", [(LENS, [1] * len(LENS)), ([40, 300, 7], [2, 3, 7]), ([70, 129], [70, 129]),
                                      ([1, 1000, 64, 90], [1, 1, 64, 2]), ([513, 0], [256, 0]), ([260, 255, 800], [130, 129, 5])])
@pytest.mark.parametrize("H,G,D,BS,nhd,dtype", [(2, 1, 64, 16, False, BF16), (1, 5, 128, 16, False, F16),
                                                (1, 6, 256, 32, True, BF16), (1, 3, 80, 24, True, F16),
                                                (2, 2, 192, 7, False, BF16), (1, 20, 16, 1, False, F16),
                                                (1, 4, 256, 12, False, F16)])
def test_attend_scaled(H, G, D, BS, nhd, dtype, lens, new):
    run_scaled(pref.ScaledCase(H, G, D, BS, lens, new, nhd=nhd, dtype=dtype, seed=7 * D + G))


@pytest.mark.parametrize("lens,new", [([40, 300, 70], [2, 67, 70]), ([70, 129], [70, 129]), ([513, 0], [256, 0]),
                                      ([260, 255, 800], [130, 129, 5])])
@pytest.mark.parametrize("H,G,D,BS,nhd,dtype", [(2, 1, 64, 16, False, BF16), (1, 5, 128, 16, False, F16),
                                                (1, 6, 256, 32, True, BF16), (1, 3, 80, 24, True, F16),
                                                (2, 2, 192, 7, False, BF16), (1, 20, 16, 1, False, F16),
                                                (1, 4, 256, 12, False, F16)])
def test_attend_scaled_within_wide_bounds(H, G, D, BS, nhd, dtype, lens, new):
    """The host's bounds leave room for far longer sequences, which would need many tiles."""
    c = pref.ScaledCase(H, G, D, BS, lens, new, nhd=nhd, dtype=dtype, seed=7 * D + G)
    wide = torch.full((len(lens), 100000 // BS), -1, dtype=torch.int32)
    wide[:, :c.tables.shape[1]] = c.tables
    c.tables = wide
    run_scaled(c)


@pytest.mark.parametrize("H,G,D,BS,dtype", [(8, 5, 64, 16, BF16), (6, 8, 128, 7, F16), (4, 6, 256, 32, BF16)])
def test_attend_scaled_short_prompts(H, G, D, BS, dtype):
    """Whole prompts beside single tokens, rows before token 0, and sequences without rows, of few tokens each."""
    lens = [130, 1, 64, 200, 3, 0, 90, 250]
    run_scaled(pref.ScaledCase(H, G, D, BS, lens, [130, 1, 2, 67, 5, 0, 0, 250], dtype=dtype, seed=H))


OPTIONS = [dict(softcap=5.0), dict(softcap=100.0), dict(window=1), dict(window=37), dict(slopes=True),
           dict(softcap=2.0, window=50, slopes=True, scale=0.3)]


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [1, 200, 17, 64]])
def test_attend_scaled_options(new, dtype, options):
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = [2.0**-(1 + i % 7) for i in range(8)]
    c = pref.ScaledCase(2, 4, 128, 16, [300, 200, 129, 64], new, dtype=dtype, seed=11)
    run_scaled(c, options)
    run_scaled(c, options, full_weights=True)


@pytest.mark.parametrize("options", [dict(softcap=5.0), dict(window=600), dict(window=570, slopes=True, softcap=20.0)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_scaled_options_of_longer_tails(dtype, options):
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = [2.0**-(1 + i % 7) for i in range(16)]
    c = pref.ScaledCase(4, 4, 64, 16, [900, 700, 64], [1, 200, 17], dtype=dtype, seed=24)
    run_scaled(c, options)


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_scaled_options_of_many_rows(dtype, options):
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = [2.0**-(1 + i % 7) for i in range(16)]
    c = pref.ScaledCase(4, 4, 128, 16, [300, 200, 129, 64], [1, 200, 17, 64], dtype=dtype, seed=23)
    run_scaled(c, options)
    run_scaled(c, options, full_weights=True)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("exponents", [(80, 82), (127, 133), (100, 134)])
def test_attend_scaled_sizes(dtype, exponents):
    """Scales far from float16's range, alike and mixed: V's show in the output as they are."""
    for new in ([1, 1], [150, 70]):
        c = pref.ScaledCase(1, 2, 64, 16, [400, 200], new, dtype=dtype, exponents=exponents, seed=12)
        # K's scales stay near 1, so that scores are scores.
        for b, n in enumerate(c.lens):
            page = c.tables[b, torch.arange(n) // c.BS].long()
            c.k[b] = c.k[b] * torch.pow(2.0, 123 - c.scales[page, 0].double()).numpy()[..., None]
        c.scales[:, 0] = torch.where(c.scales[:, 0] == 255, 255, 123).to(torch.uint8)
        want = ref.attend(c)
        cache, _, q, _, _, tables, lens, starts = c.device()
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, scales=c.scales.to(DEV))
        ref.check(lse, want[1], want[4], "lse")
        # float16's own range is the output's: what is beyond it is infinite, what is below rounds to its smallest.
        ok = np.abs(want[0]) < (6.5e4 if dtype == F16 else 1e38)
        off = want[3] + 2.0**-25
        ref.check(np.where(ok, out.double().cpu().numpy(), 0), np.where(ok, want[0], 0), off, "out")


@pytest.mark.parametrize("H,G,D,BS,dtype", [(2, 4, 64, 16, BF16), (4, 3, 128, 32, BF16), (2, 3, 256, 7, BF16),
                                            (2, 4, 64, 16, F16)])
@pytest.mark.parametrize("options", [dict(), dict(softcap=5.0, window=700)])
def test_attend_scaled_tails_round_their_output_alone(H, G, D, BS, dtype, options):
    """Longer tails' weights meet V as two numbers too, whatever the host's bounds: the bounds here are attend_chosen's,
    which leave no room for a weight rounded to the rows' type."""
    c = pref.ScaledCase(H, G, D, BS, [1100, 90], [330, 2], dtype=dtype, seed=D + G)
    every = torch.arange(-(-1100 // BS), dtype=torch.int32).expand(c.T, 1, -1)
    want = pref.attend_chosen(c, every, torch.full((c.T,), every.shape[2]), **options)
    cache, _, q, _, _, tables, lens, starts = c.device()
    for bounds in (dict(max_len=1100, max_q=330), dict()):
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, scales=c.scales.to(DEV), **options, **bounds)
        torch.cuda.synchronize()
        ref.check(lse, want[1], want[3], "lse")
        ref.check(out, want[0], want[2], "out")


@pytest.mark.parametrize("H,G,D,BS,dtype", [(4, 3, 128, 16, BF16), (2, 6, 256, 32, F16), (3, 4, 64, 7, BF16)])
def test_attend_scaled_single_tokens_beside_tails(H, G, D, BS, dtype):
    """Few rows over many tokens, in parts, where the batch has tails."""
    c = pref.ScaledCase(H, G, D, BS, [2000, 64, 1999, 5, 40, 700], [1, 30, 100, 1, 0, 2], dtype=dtype, seed=H)
    run_scaled(c)
    run_scaled(c, dict(window=300, softcap=20.0))


def test_attend_scaled_long():
    """Few rows over many tokens, split and joined, and many sequences."""
    run_scaled(pref.ScaledCase(1, 3, 128, 16, [5000, 3000], [1, 70], seed=13))
    gen = np.random.default_rng(3)
    lens = [int(n) for n in gen.integers(0, 60, 150)]
    lens[7], lens[70] = 3000, 1500
    run_scaled(pref.ScaledCase(2, 2, 64, 16, lens, [1 if n % 5 else 0 for n in lens], seed=22))


# ---- Bounds and scores --------------------------------------------------------------------


def bounds_cache(c, fill):
    t = torch.full((c.num_blocks, 2, c.H, 1, c.D), fill).to(c.cache_dtype).to(DEV)
    return kvx.Cache([t], kvx.make_layout(1, c.H, c.D, t.element_size(), 1, 1), c.num_blocks), t


@pytest.mark.parametrize("lens,new", [(LENS, [1] * len(LENS)), ([40, 300, 7, 0, 64], [2, 3, 7, 0, 64]), ([3, 5], [6, 5]),
                                      ([3000], [3000])])
@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,dtype", [
    (2, 1, 64, 16, False, False, BF16), (4, 1, 256, 32, True, True, BF16), (8, 1, 128, 16, False, False, F16),
    (3, 1, 80, 7, True, False, BF16), (1, 1, 16, 1, False, True, F16), (2, 1, 248, 300, False, False, BF16)])
def test_bounds(H, G, D, BS, nhd, fp8, dtype, lens, new):
    c = ref.Case(H, G, D, BS, lens, new, nhd=nhd, fp8=fp8, dtype=dtype, seed=D + BS)
    # A column without a number in one page, one with a NaN among others, infinities.
    slot = c.flat[int(c.tables[0, 0]), :2 * BS * H * D].view(c.shape)
    slot[0, ..., 3] = float("nan")
    last = c.flat[int(c.tables[1, 0] if c.B > 1 else c.tables[0, 1]), :2 * BS * H * D].view(c.shape)
    last[0, 0, 0, 1] = float("nan")
    if not fp8:
        last[0, 0, 0, 2] = float("inf")
    cache, _, _, _, _, tables, lens_d, starts = c.device()
    low_high, t = bounds_cache(c, 77.0)
    kw = {} if new.count(1) == len(new) else dict(starts=starts)
    attend.kv_bounds(cache, 0, low_high, tables, lens_d, max_len=max(lens), dtype=c.cache_dtype, **kw)
    torch.cuda.synchronize()
    want = pref.bounds(c, c.flat)
    got = t[:, :, :, 0].double().cpu().numpy()
    assert np.array_equal(got, np.where(np.isnan(want), 77.0 if not fp8 else float(torch.tensor(77.0).to(E4M3)), want))


def test_bounds_of_many_pages():
    """Enough pages that a wave has several at once."""
    c = ref.Case(8, 1, 64, 4, [6000, 3001], [6000, 3001], seed=31)
    cache, _, _, _, _, tables, lens, starts = c.device()
    low_high, t = bounds_cache(c, 0.0)
    attend.kv_bounds(cache, 0, low_high, tables, lens, starts, dtype=BF16)
    want = pref.bounds(c, c.flat)
    got = t[:, :, :, 0].double().cpu().numpy()
    assert np.array_equal(got, np.where(np.isnan(want), 0.0, want))


@pytest.mark.parametrize("lens,new", [(LENS, [1] * len(LENS)), ([40, 300, 7, 0], [2, 3, 7, 0]), ([3, 5], [6, 5]),
                                      ([2500, 100], [70, 33])])
@pytest.mark.parametrize("H,G,D,BS,scaled,dtype", [
    (2, 1, 64, 16, False, BF16), (1, 2, 128, 3, False, BF16), (1, 3, 80, 16, False, F16), (2, 5, 128, 16, True, BF16),
    (1, 8, 256, 32, True, F16), (1, 12, 256, 24, False, F16), (1, 17, 16, 8, True, BF16), (1, 40, 64, 16, False, BF16)])
def test_scores(H, G, D, BS, scaled, dtype, lens, new):
    kind = pref.ScaledCase if scaled else ref.Case
    c = kind(H, G, D, BS, lens, new, dtype=dtype, seed=D + G)
    gen = torch.Generator().manual_seed(8)
    some = torch.randn(c.num_blocks, H, D, 2, generator=gen).mul(8 if scaled else 1).to(c.cache_dtype).double()
    t = some.sort(-1).values.permute(0, 3, 1, 2).unsqueeze(3).contiguous()
    low_high = kvx.Cache([t.to(c.cache_dtype).to(DEV)],
                         kvx.make_layout(1, H, D, 1 if scaled else 2, 1, 1), c.num_blocks)
    _, _, q, _, _, tables, lens_d, starts = c.device()
    longest = max(lens)
    width = -(-longest // BS)
    out = torch.full((c.T, H, width + 3), -7.0, device=DEV)[:, :, :width]
    factors = torch.pow(2.0, c.scales[:, 0].double() - 127).numpy() if scaled else None
    want, off, counts = pref.scores(c, t[:, :, :, 0].numpy(), factors, 0.7)
    got, got_counts = attend.kv_score(low_high, 0, q, tables, lens_d, starts, block_size=BS, max_len=longest, out=out,
                                      scales=c.scales.to(DEV) if scaled else None, scale=0.7)
    torch.cuda.synchronize()
    assert got_counts.cpu().tolist() == counts.tolist()
    want, off = want[:, :, :width], off[:, :, :width]
    left = np.isnan(want)
    ref.check(got, np.where(left, -7.0, want), np.where(left, 0.0, off + np.abs(np.where(left, 0, want)) * 2.0**-21), "scores")


def test_scores_are_bounds():
    """No token of a page scores more than its page, and a page of one token as much as the token."""
    for BS in (1, 16):
        c = ref.Case(2, 3, 64, BS, [200], [5], seed=6)
        cache, _, q, _, _, tables, lens, starts = c.device()
        low_high, _ = bounds_cache(c, 0.0)
        all_rows = torch.tensor([0, 200], dtype=torch.int32, device=DEV)
        attend.kv_bounds(cache, 0, low_high, tables, lens, all_rows, dtype=BF16)
        got, counts = attend.kv_score(low_high, 0, q, tables, lens, starts, block_size=BS)
        s = np.einsum("ihgd,thd->ihgt", c.q.double().numpy().reshape(5, 2, 3, 64), c.k[0]).max(2)
        for i in range(5):
            p = 195 + i
            assert int(counts[i]) == p // BS + 1
            pages = got[i, :, :p // BS + 1].double().cpu().numpy()
            for j in range(p // BS + 1):
                best = s[i, :, j * BS:min(p + 1, (j + 1) * BS)].max(-1)
                assert (pages[:, j] >= best - 1e-4).all()
                if BS == 1:
                    assert np.allclose(pages[:, j], best, atol=1e-4)


@pytest.mark.parametrize("D,fp8,dtype", [(64, False, BF16), (64, False, F16), (80, True, BF16), (144, False, F16)])
def test_bounds_of_many_long_pages(D, fp8, dtype):
    """The same of pages of more rows than a lane has on their way, in every type, with numbers that are not finite."""
    c = ref.Case(8, 1, D, 20, [16500, 4507], [16500, 4507], fp8=fp8, dtype=dtype, seed=34)
    some = c.flat[int(c.tables[0, 1]), :2 * 20 * 8 * D].view(c.shape)
    some[0, 1, 3:19, 5] = float("nan")
    some[0, 2, :, 6] = float("nan")
    if not fp8:
        some[0, 0, 17, 1], some[0, 0, 9, 2] = float("inf"), -float("inf")
    cache, _, _, _, _, tables, lens, starts = c.device()
    low_high, t = bounds_cache(c, 0.0)
    attend.kv_bounds(cache, 0, low_high, tables, lens, starts, dtype=c.cache_dtype)
    want = pref.bounds(c, c.flat)
    got = t[:, :, :, 0].double().cpu().numpy()
    assert np.array_equal(got, np.where(np.isnan(want), 0.0, want))


# ---- Attention over chosen pages ----------------------------------------------------------


def run_chosen(c, budget, heads, options=None, seed=0, scaled=False):
    options = dict(options or {})
    pages, counts = pref.choose(c, budget, heads, seed)
    plain = dict(options)
    if plain.get("slopes") is not None:
        options["slopes"] = torch.tensor(plain["slopes"], dtype=torch.float32, device=DEV)
        plain["slopes"] = options["slopes"].double().cpu().numpy()
    want = pref.attend_chosen(c, pages, counts, **plain)
    cache, _, q, _, _, tables, lens, starts = c.device()
    if scaled:
        options["scales"] = c.scales.to(DEV)
    else:
        options.update(k_scale=c.k_scale, v_scale=c.v_scale)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, pages=pages.to(DEV), counts=counts.to(DEV), **options)
    torch.cuda.synchronize()
    ref.check(lse, want[1], want[3], "lse")
    ref.check(out, want[0], want[2], "out")


@pytest.mark.parametrize("lens,new", [(LENS, [1] * len(LENS)), ([40, 300, 7, 0], [2, 3, 7, 0]), ([3, 5], [6, 5]),
                                      ([2500, 100], [40, 33])])
@pytest.mark.parametrize("H,G,D,BS,nhd,fp8,scaled,dtype", [
    (2, 1, 64, 16, False, False, False, BF16), (1, 5, 128, 16, False, False, False, BF16),
    (2, 6, 256, 32, True, True, True, BF16), (1, 16, 64, 8, False, True, True, F16), (3, 4, 80, 24, True, False, False, F16),
    (1, 17, 96, 16, False, False, False, F16), (2, 3, 192, 7, False, False, False, BF16), (1, 2, 16, 1, False, True, False, F16),
    (1, 33, 128, 64, True, True, True, F16), (2, 7, 112, 12, True, True, False, BF16), (1, 1, 248, 16, False, False, False, F16),
    (1, 20, 64, 16, False, False, False, BF16)])
def test_attend_chosen(H, G, D, BS, nhd, fp8, scaled, dtype, lens, new):
    if scaled:
        c = pref.ScaledCase(H, G, D, BS, lens, new, nhd=nhd, dtype=dtype, seed=D + G)
    else:
        c = ref.Case(H, G, D, BS, lens, new, nhd=nhd, fp8=fp8, dtype=dtype, seed=D + G)
    for budget, heads in ((1, 1), (6, H), (60, 1)):
        run_chosen(c, budget, heads, seed=budget, scaled=scaled)


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("scaled,BS", [(False, 16), (True, 16), (True, 7)])
def test_attend_chosen_options(options, scaled, BS):
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = [2.0**-(1 + i % 7) for i in range(8)]
    kind = pref.ScaledCase if scaled else ref.Case
    c = kind(2, 4, 128, BS, [300, 200, 129, 64], [1, 5, 17, 3], seed=11)
    run_chosen(c, 5, 2, options, scaled=scaled)


def test_attend_chosen_long():
    """Lists that are cut into parts, and joined: a few, and more than eight."""
    c = ref.Case(1, 3, 128, 16, [6000, 900], [1, 1], seed=13)
    run_chosen(c, 300, 1)
    run_chosen(c, 20, 1)
    run_chosen(ref.Case(2, 5, 64, 16, [1500] * 9, [1] * 9, seed=14), 80, 2)


@pytest.mark.parametrize("H,G,D,BS,fp8,scaled,dtype", [(2, 3, 128, 16, False, False, BF16), (3, 1, 64, 8, False, False, F16),
                                                       (1, 2, 256, 16, False, False, BF16), (2, 2, 256, 32, True, True, F16),
                                                       (2, 17, 80, 7, False, False, BF16), (3, 2, 16, 16, True, False, BF16)])
def test_attend_chosen_by_many(H, G, D, BS, fp8, scaled, dtype):
    """So many rows that every wave has one for itself; rows before the first sequence's and behind the last's, bad ones."""
    if scaled:
        c = pref.ScaledCase(H, G, D, BS, [600, 0, 511, 3], [520, 0, 511, 1], dtype=dtype, seed=D)
    else:
        c = ref.Case(H, G, D, BS, [600, 0, 511, 3], [520, 0, 511, 1], fp8=fp8, dtype=dtype, seed=D)
    run_chosen(c, 3, H, scaled=scaled)
    run_chosen(c, 9, 1, dict(window=50, softcap=3.0, slopes=[2.0**-(1 + i % 7) for i in range(H * G)]), scaled=scaled)
    pages, counts = pref.choose(c, 2, 1, 0)
    counts[700], counts[701] = 3, -1
    want = pref.attend_chosen(c, pages, counts.clamp(0, 2))
    cache, _, q, _, _, tables, lens, starts = c.device()
    out, lse = torch.full((c.T + 2, H * G, D), 9.0, dtype=dtype, device=DEV), torch.full((c.T + 2, H * G), 9.0, device=DEV)
    wide = lambda x: torch.cat([x[:1], x, x[:1]])  # noqa: E731
    scales = dict(scales=c.scales.to(DEV)) if scaled else dict(k_scale=c.k_scale, v_scale=c.v_scale)
    with fault(attend.KV_ASYNC_BAD_BATCH):
        attend.kv_attend(cache, 0, wide(q), tables, lens, starts + 1, pages=wide(pages).to(DEV), counts=wide(counts).to(DEV),
                         out=out, lse=lse, **scales)
    for row in (0, 701, 702, c.T + 1):
        assert bool((out[row] == 9).all()) and bool((lse[row] == 9).all())
    keep = torch.ones(c.T, dtype=torch.bool)
    keep[700:702] = False
    ref.check(out[1:-1][keep.to(DEV)], want[0][keep], want[2][keep], "out")
    ref.check(lse[1:-1][keep.to(DEV)], want[1][keep], want[3][keep], "lse")


def test_attend_chosen_behind_the_last_row():
    """Sequences without new tokens, the last ones among them, where lists are joined: there is no row to look up."""
    c = ref.Case(2, 2, 64, 16, [900, 40, 700, 30, 20], [1, 0, 2, 0, 0], seed=18)
    run_chosen(c, 30, 2)
    run_chosen(c, 57, 1)


def test_attend_chosen_by_many_sequences():
    """More sequences than a wave looks at at once, without new tokens where it looks again, in a call whose bound of
    new tokens is the binding's default, all of them.  All pages, in order, are attention over everything."""
    gen = np.random.default_rng(5)
    new = [int(x) for x in gen.choice([0, 1, 1, 3], 2000)]
    for at in (0, 63, 64, 127, 128, 129, 1999):
        new[at] = 0
    new[65], new[1998] = 2, 1
    lens = [int(x) + n for x, n in zip(gen.integers(1, 30, 2000), new)]
    c = ref.Case(8, 16, 16, 16, lens, new, seed=33)
    assert -(-c.T * 16 // 128) * 8 * 2000 > 1 << 22  # (as tiles, too many for a launch)
    cache, _, q, _, _, tables, lens_d, starts = c.device()
    want, want_lse = attend.kv_attend(cache, 0, q, tables, lens_d, starts, max_q=3)
    seq = np.repeat(np.arange(2000), new)
    pages = torch.arange(3, dtype=torch.int32, device=DEV).expand(c.T, 1, 3)
    counts = torch.tensor([-(-lens[b] // 16) for b in seq], dtype=torch.int32, device=DEV)
    tight = attend.kv_attend(cache, 0, q, tables, lens_d, starts, pages=pages, counts=counts, max_q=3)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens_d, starts, pages=pages, counts=counts)
    assert torch.equal(out, tight[0]) and torch.equal(lse, tight[1])
    # Both outputs are within half a step of the same numbers, and what is beside their last rounding.
    assert (lse - want_lse).abs().max() < 2.0**-17
    assert ((out.float() - want.float()).abs() <= want.float().abs() * 2.0**-7 * 1.01 + 2.0**-13).all()


def test_attend_chosen_more_than_there_is():
    """Lists with far more room than a sequence has pages, and lists that name its few pages many times over."""
    for n in (60, 700):
        c = ref.Case(1, 2, 64, 16, [n, n - 9], [1, 1], seed=n)
        run_chosen(c, 400, 1)
        pages = torch.arange(400, dtype=torch.int32).remainder(3).view(1, 1, 400).expand(2, 1, 400).contiguous()
        counts = torch.tensor([400, 399], dtype=torch.int32)
        cache, _, q, _, _, tables, lens, _ = c.device()
        want = pref.attend_chosen(c, pages, counts)
        for max_len in (None, n):
            out, lse = attend.kv_attend(cache, 0, q, tables, lens, pages=pages.to(DEV), counts=counts.to(DEV),
                                        max_len=max_len)
            ref.check(lse, want[1], want[3], "lse")
            ref.check(out, want[0], want[2], "out")


def test_attend_all_pages_chosen():
    """All pages, in order, are attention over everything."""
    c = ref.Case(2, 4, 128, 16, [333, 50], [1, 1], seed=15)
    cache, _, q, _, _, tables, lens, _ = c.device()
    want, want_lse = attend.kv_attend(cache, 0, q, tables, lens)
    every = torch.arange(21, dtype=torch.int32, device=DEV).expand(2, 1, 21)
    counts = torch.tensor([21, 4], dtype=torch.int32, device=DEV)
    out, lse = attend.kv_attend_pages(cache, 0, q, tables, lens, pages=every, counts=counts)
    assert (lse - want_lse).abs().max() < 2.0**-18
    assert (out.float() - want.float()).abs().max() <= want.float().abs().max() * 2.0**-7


def test_attend_chosen_lists_as_they_come():
    """Pages behind the token, none at all, the same twice, windows that hide whole pages."""
    c = ref.Case(2, 2, 64, 16, [100, 100, 100, 100], [1] * 4, seed=16)
    pages = torch.tensor([[[6, 0, 6]], [[5, 1, 2]], [[0, 3, 1]], [[2, 2, 2]]], dtype=torch.int32)
    counts = torch.tensor([2, 0, 3, 3], dtype=torch.int32)
    cache, _, q, _, _, tables, lens, _ = c.device()
    want = pref.attend_chosen(c, pages, counts)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, pages=pages.to(DEV), counts=counts.to(DEV))
    ref.check(lse, want[1], want[3], "lse")
    ref.check(out, want[0], want[2], "out")
    assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, pages=pages.to(DEV), counts=counts.to(DEV), window=10)
    want = pref.attend_chosen(c, pages, counts, window=10)
    ref.check(lse, want[1], want[3], "lse")
    ref.check(out, want[0], want[2], "out")
    # A page behind the query's own holds no token that it sees.
    early = torch.tensor([20, 20, 20, 20], dtype=torch.int32, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q, tables, early, pages=pages.to(DEV), counts=counts.to(DEV))
    assert bool((out[3] == 0).all()) and bool(torch.isneginf(lse[3]).all())
    assert bool(torch.isfinite(lse[0]).all())


def test_attend_chosen_before_the_window():
    """A page that lies before the window may be given away: its block and its scales are not looked at."""
    c = pref.ScaledCase(2, 3, 64, 16, [100, 90], [1, 2], seed=19)
    pages = torch.tensor([0, 5, 6, 1, 4], dtype=torch.int32).expand(3, 1, 5).contiguous()
    counts = torch.tensor([5, 5, 4], dtype=torch.int32)
    cache, _, q, _, _, tables, lens, starts = c.device()
    by = c.scales.to(DEV)
    want = pref.attend_chosen(c, pages, counts, window=20)
    gone = tables.clone()
    gone[0, :4], gone[1, :4] = -1, 1 << 30
    other = by.clone()
    other.view(torch.uint8)[tables[0, :4].long()] = 255
    for table, scales in ((tables, by), (gone, by), (tables, other)):
        out, lse = attend.kv_attend(cache, 0, q, table, lens, starts, pages=pages.to(DEV), counts=counts.to(DEV),
                                    window=20, scales=scales)
        ref.check(lse, want[1], want[3], "lse")
        ref.check(out, want[0], want[2], "out")


@pytest.mark.parametrize("k_scale,v_scale", [(1.0, 0.37), (3.3, 2.0**-70), (1e-30, 3e30), (2.0**-10, 7e-4)])
def test_rotate_stores_what_append_does(k_scale, v_scale):
    """Without norms and a rotation an e4m3 cache holds the same bytes after either, whatever the scales."""
    c = ref.Case(2, 2, 64, 16, [300, 17], [290, 3], fp8=True, seed=22)
    _, flat, q, k, v, tables, lens, starts = c.device()
    k, v = ((x.double() * s).clamp(-3e38, 3e38).to(BF16) for x, s in ((k, k_scale), (v, v_scale)))
    k[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), 0.0, -0.0], dtype=BF16)
    caches = []
    for f in (attend.kv_append, lambda cache, layer, *x, **kw: attend.kv_rotate(cache, layer, q, *x, **kw)):
        cache, flat, *_ = c.device()
        f(cache, 0, k, v, tables, lens, starts, k_scale=k_scale, v_scale=v_scale)
        torch.cuda.synchronize()
        caches.append(flat.cpu())
    same_bytes(caches[0], caches[1], "cache")


def test_rotate_many_in_place():
    """Queries that are overwritten, while a workgroup has the next ones on their way."""
    c = ref.Case(2, 5, 64, 16, [700, 90], [650, 33], seed=21)
    run_rotate(c, rotary=20, in_place=True)
    run_rotate(c, in_place=True)


# ---- Bad numbers on the device, streams, graphs -------------------------------------------


def test_bad_numbers():
    c = ref.Case(2, 2, 64, 16, [100, 50, 60], [1, 1, 1], seed=17)
    cache, flat, q, k, v, tables, lens, _ = c.device()
    pages = torch.tensor([[[0, 1]], [[0, 9]], [[-3, 2]]], dtype=torch.int32, device=DEV)
    counts = torch.tensor([3, 2, 2], dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q.contiguous(), 5.0), torch.full((3, 4), 5.0, device=DEV)
    with fault(attend.KV_ASYNC_BAD_BATCH):  # row 0 is left out; pages 9 and -3 alone of the others
        attend.kv_attend(cache, 0, q, tables, lens, pages=pages, counts=counts, out=out, lse=lse)
    want = pref.attend_chosen(c, torch.tensor([[[0]], [[0]], [[2]]]), torch.tensor([0, 1, 1]))
    assert bool((out[0] == 5).all()) and bool((lse[0] == 5).all())
    ref.check(lse[1:], want[1][1:], want[3][1:], "lse")
    ref.check(out[1:], want[0][1:], want[2][1:], "out")
    # A block that is none takes part in nothing.
    bad = tables.clone()
    bad[0, 1] = c.num_blocks
    counts[0] = 2
    with fault(kvx.KV_ASYNC_BAD_BLOCK | attend.KV_ASYNC_BAD_BATCH):
        out, lse = attend.kv_attend(cache, 0, q, bad, lens, pages=pages, counts=counts)
    want = pref.attend_chosen(c, torch.tensor([[[0]], [[0]], [[2]]]), torch.tensor([1, 1, 1]))
    ref.check(out, want[0], want[2], "out")
    low_high, t = bounds_cache(c, 1.0)
    with fault(kvx.KV_ASYNC_BAD_BLOCK):
        scores, counts = attend.kv_score(low_high, 0, q, bad, lens, block_size=16)
    assert bool(torch.isneginf(scores[0, :, 1]).all()) and bool(torch.isfinite(scores[0, :, :1]).all())
    bad = tables.clone()
    bad[1, 3] = -1
    with fault(kvx.KV_ASYNC_BAD_BLOCK):
        attend.kv_bounds(cache, 0, low_high, bad, lens, dtype=BF16)
    before = flat.clone()
    freqs = torch.ones(32, dtype=torch.float64, device=DEV)
    with fault(kvx.KV_ASYNC_BAD_BLOCK):
        got = attend.kv_rotate(cache, 0, q, k, v, bad, lens, freqs=freqs)
    assert bool(torch.isfinite(got).all())
    changed = (flat.view(torch.int16) != before.view(torch.int16)).any(1).nonzero().view(-1).tolist()
    assert sorted(changed) == sorted([int(c.tables[0, 6]), int(c.tables[2, 3])])
    # Lengths beyond the bound: the sequence is left out of everything.
    before, marks = flat.clone(), torch.full_like(q.contiguous(), 3.0)
    with fault(attend.KV_ASYNC_BAD_BATCH):
        attend.kv_rotate(cache, 0, q, k, v, tables, lens, freqs=freqs, max_len=99, out=marks)
    assert bool((marks[0] == 3).all()) and not bool((marks[1] == 3).all())
    assert torch.equal(flat[int(c.tables[0, 6])].view(torch.int16), before[int(c.tables[0, 6])].view(torch.int16))
    scaled = pref.ScaledCase(2, 2, 64, 16, [100, 50], [1, 1], seed=18)
    cache, flat, q, k, v, tables, lens, _ = scaled.device()
    by, before = scaled.scales.to(DEV), flat.clone()
    with fault(attend.KV_ASYNC_BAD_BATCH):
        attend.kv_append(cache, 0, k, v, tables, lens, scales=by, max_len=40)
    assert torch.equal(by.cpu(), scaled.scales) and torch.equal(flat.view(torch.uint8), before.view(torch.uint8))


def test_rows_of_no_sequence():
    """Rows before the first start and behind the last are left as they were, by every call."""
    c = ref.Case(1, 2, 64, 16, [40, 20], [3, 2], seed=19)
    cache, _, q, k, v, tables, lens, starts = c.device()
    wide = lambda x: torch.cat([x[:1], x, x[:2]])  # noqa: E731
    q, k, v, starts = wide(q), wide(k), wide(v), starts + 1
    out = torch.full_like(q, 9.0)
    freqs = torch.ones(32, dtype=torch.float64, device=DEV)
    attend.kv_rotate(cache, 0, q, k, v, tables, lens, starts, freqs=freqs, out=out)
    assert bool((out[[0, 6, 7]] == 9).all()) and not bool((out[1:6] == 9).any(-1).any(-1).all())
    pages = torch.zeros(8, 1, 1, dtype=torch.int32, device=DEV)
    counts = torch.ones(8, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 9.0), torch.full((8, 2), 9.0, device=DEV)
    attend.kv_attend(cache, 0, q, tables, lens, starts, pages=pages, counts=counts, out=out, lse=lse)
    assert bool((out[[0, 6, 7]] == 9).all()) and bool((lse[[0, 6, 7]] == 9).all()) and not bool((lse[1:6] == 9).any())
    low_high, _ = bounds_cache(c, 1.0)
    counts = torch.full((8,), 9, dtype=torch.int32, device=DEV)
    scores = torch.full((8, 1, 4), 9.0, device=DEV)
    attend.kv_score(low_high, 0, q, tables, lens, starts, block_size=16, out=scores, counts=counts)
    assert counts.tolist() == [9, 3, 3, 3, 2, 2, 9, 9] and bool((scores[[0, 6, 7]] == 9).all())
    _, counts = attend.kv_score(low_high, 0, q, tables, lens, starts, block_size=16)
    assert counts.tolist() == [0, 3, 3, 3, 2, 2, 0, 0]


def test_empty_batches():
    c = pref.ScaledCase(2, 2, 64, 16, [40], [1], seed=20)
    cache, _, q, k, v, tables, lens, _ = c.device()
    by = c.scales.to(DEV)
    low_high, _ = bounds_cache(c, 1.0)
    for rows, starts in ((0, None), (0, torch.zeros(2, dtype=torch.int32, device=DEV))):
        B = 0 if starts is None else 1
        args = (tables[:B], lens[:B], starts)
        assert attend.kv_rotate(cache, 0, q[:0], k[:0], v[:0], *args, scales=by).shape == (0, 4, 64)
        attend.kv_append(cache, 0, k[:0], v[:0], *args, scales=by)
        attend.kv_bounds(cache, 0, low_high, *args)
        assert attend.kv_score(low_high, 0, q[:0], *args, block_size=16)[1].shape == (0,)
        pages, counts = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((0, 1, 2), (0,)))
        assert attend.kv_attend(cache, 0, q[:0], *args, scales=by, pages=pages, counts=counts)[0].shape == (0, 4, 64)
        assert attend.kv_attend(cache, 0, q[:0], *args, scales=by)[0].shape == (0, 4, 64)
    assert torch.equal(by.cpu(), c.scales)


class Step:
    """One layer's step on scaled pages: rotate and append, move the bounds, score, choose, attend."""

    def __init__(self, c, budget):
        self.cache, self.flat, self.q, self.k, self.v, self.tables, self.lens, self.starts = c.device()
        self.scales = c.scales.to(DEV)
        self.bounds, self.low_high = bounds_cache(c, 0.0)
        self.freqs = torch.tensor(10000.0 ** (-np.arange(c.D // 2) / (c.D // 2)), dtype=torch.float64).to(DEV)
        self.weight = torch.ones(c.D, device=DEV)
        self.budget, self.c = budget, c
        n = torch.tensor([0] + list(np.cumsum(c.lens)), dtype=torch.int32, device=DEV)
        attend.kv_bounds(self.cache, 0, self.bounds, self.tables, self.lens, n)

    def __call__(self, stream=None):
        batch = dict(tables=self.tables, lens=self.lens, starts=self.starts, stream=stream)
        q = attend.kv_rotate(self.cache, 0, self.q, self.k, self.v, freqs=self.freqs, q_weight=self.weight,
                             k_weight=self.weight, scales=self.scales, **batch)
        attend.kv_bounds(self.cache, 0, self.bounds, **batch)
        scores, counts = attend.kv_score(self.bounds, 0, q, block_size=self.c.BS, scales=self.scales, **batch)
        pages, kept, _ = attend.kv_keep(scores, counts, self.budget, sinks=1, recent=1, stream=stream)
        out, lse = attend.kv_attend(self.cache, 0, q, scales=self.scales, pages=pages, counts=kept, **batch)
        return q, scores, counts, pages, kept, out, lse


def check_step(c, step, got):
    """The choice is the best pages by the scores, and the output what the chosen pages give."""
    q, scores, counts, pages, kept, out, lse = (x.cpu() for x in got)
    want_keep, want_kept, _ = ref.keep(scores.numpy(), counts.numpy(), step.budget, 1, 1)
    assert np.array_equal(pages.numpy(), want_keep) and np.array_equal(kept.numpy(), want_kept)
    flat, by = step.flat.cpu(), torch.pow(2.0, step.scales.cpu().double() - 127).numpy()
    want_bounds = pref.bounds(c, flat)
    got_bounds = step.low_high[:, :, :, 0].double().cpu().numpy()
    assert np.array_equal(got_bounds[~np.isnan(want_bounds)], want_bounds[~np.isnan(want_bounds)])
    c.q = q
    want, off, _ = pref.scores(c, got_bounds, by[:, 0])
    width = scores.shape[2]
    seen = ~np.isnan(want[:, :, :width])
    assert (np.abs(scores.double().numpy() - want[:, :, :width])[seen] <=
            (off[:, :, :width] + np.abs(want[:, :, :width]) * 2.0**-21)[seen]).all()
    for b, n in enumerate(c.lens):
        rows = c.rows_of(flat, b, n)
        page = c.tables[b, torch.arange(n) // c.BS].long().numpy()
        c.k[b], c.v[b] = rows[0] * by[page, 0][..., None], rows[1] * by[page, 1][..., None]
    want = pref.attend_chosen(c, pages, kept)
    ref.check(lse, want[1], want[3], "lse")
    ref.check(out, want[0], want[2], "out")


@pytest.mark.parametrize("new", [[1, 1, 1], [4, 1, 20]])
def test_step(new):
    c = pref.ScaledCase(2, 3, 64, 16, [500, 30, 300], new, seed=24)
    step = Step(c, 6)
    check_step(c, step, step())


def test_step_on_a_restored_cache():
    """Pages, their scales and their bounds go through one pool each by the same block tables, into other blocks."""
    L, H, G, D, BS, C, n = 1, 4, 2, 64, 16, 64, 230
    c = pref.ScaledCase(H, G, D, BS, [n + 1], [1], seed=25)
    cache, flat, q, k, v, tables, lens, _ = c.device()
    # Scales padded to 16 bytes, so that they are a cache of one token a block.
    held = torch.zeros(c.num_blocks, 2, 16, dtype=torch.uint8, device=DEV)
    held[:, :, :H] = c.scales.to(DEV)
    low_high, t = bounds_cache(c, 0.0)
    attend.kv_bounds(cache, 0, low_high, tables, lens, torch.tensor([0, n], dtype=torch.int32, device=DEV))
    pages = -(-n // BS)
    other = 40
    new_blocks = torch.randperm(other, generator=torch.Generator().manual_seed(1))[:pages + 1].int().to(DEV)
    flat_b = torch.zeros(other, c.elems, dtype=E4M3, device=DEV)
    held_b = torch.zeros(other, 2, 16, dtype=torch.uint8, device=DEV)
    t_b = torch.zeros(other, 2, H, 1, D, dtype=E4M3, device=DEV)
    lay = kvx.make_layout(L, H, D, 1, BS, C)
    lay_s, lay_t = kvx.make_layout(L, 1, 16, 1, 1, C // BS), kvx.make_layout(L, H, D, 1, 1, C // BS)
    stream = torch.cuda.current_stream()
    ids = list(range(-(-n // C)))
    for a, b, layout, tokens in ((flat, flat_b, lay, n), (held, held_b, lay_s, pages), (t, t_b, lay_t, pages)):
        pool = kvx.kv_pool_create(layout, len(ids), "zero_copy")
        kvx.kv_store(kvx.Cache([a], layout, c.num_blocks), tables[0], tokens, pool, ids, stream)
        kvx.kv_load(kvx.Cache([b], layout, other), new_blocks, tokens, pool, ids, stream)
        torch.cuda.synchronize()
        assert kvx.kv_pool_async_error(pool) == 0
        kvx.kv_pool_destroy(pool)
    cache_b, bounds_b = kvx.Cache([flat_b], lay, other), kvx.Cache([t_b], lay_t, other)
    table_b = new_blocks.view(1, -1)
    freqs = torch.ones(D // 2, dtype=torch.float64, device=DEV)
    results = []
    for x, b, s, tab in ((cache, low_high, held, tables), (cache_b, bounds_b, held_b, table_b)):
        s = s[:, :, :H]
        got = attend.kv_rotate(x, 0, q, k, v, tab, lens, freqs=freqs, scales=s)
        attend.kv_bounds(x, 0, b, tab, lens)
        scores, counts = attend.kv_score(b, 0, got, tab, lens, block_size=BS, scales=s, max_len=n + 1)
        chosen, kept, _ = attend.kv_keep(scores, counts, 5, recent=1)
        results.append((scores, chosen) + attend.kv_attend(x, 0, got, tab, lens, scales=s, pages=chosen, counts=kept))
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_step_in_graphs():
    """Captured, and replayed with other numbers in the same arrays, with eager work between: every replay is what the
    eager calls give.  Two graphs have workspaces of their own."""
    cases = [pref.ScaledCase(2, 3, 64, 16, [3000, 30, 300], [1, 1, 1], seed=s) for s in (26, 27)]
    steps = [Step(c, 40) for c in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for step in steps:
            step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for step in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    for turn in range(3):
        for step in steps:
            step.q.copy_(torch.randn_like(step.q, dtype=torch.float32).to(step.q.dtype))
            step.lens.sub_(torch.tensor([turn * 100, 0, turn], dtype=torch.int32, device=DEV))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        replayed = [[x.clone() for x in out] for out in outs]
        for step, got in zip(steps, replayed):
            eager = step()
            torch.cuda.synchronize()
            for name, x, y in zip(("q", "scores", "counts", "pages", "kept", "out", "lse"), got, eager):
                if name == "scores":
                    seen = torch.arange(x.shape[2], device=DEV) < got[2].view(-1, 1, 1)
                    x, y = (z.masked_fill(~seen, 0) for z in (x, y))
                assert torch.equal(x, y), (turn, name)


def test_streams():
    """A call on a named stream, its tensors freed right behind it, while the current stream is busy with others."""
    c = pref.ScaledCase(2, 3, 64, 16, [500, 30, 300], [1, 1, 1], seed=28)
    step = Step(c, 6)
    want = [x.clone() for x in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = step(stream=s)
        for _ in range(20):
            torch.full((1 << 16,), -1, dtype=torch.int32, device=DEV)
        s.synchronize()
        for x, y, name in zip(got, want, ("q", "scores", "counts", "pages", "kept", "out", "lse")):
            if name != "scores":
                assert torch.equal(x, y), name


def test_same_bits():
    """The same call gives the same bits."""
    c = pref.ScaledCase(2, 3, 128, 16, [3000, 30, 300], [1, 1, 1], seed=29)
    step = Step(c, 100)
    first = step()
    for _ in range(3):
        again = step()
        assert torch.equal(first[5], again[5]) and torch.equal(first[6], again[6]) and torch.equal(first[0], again[0])


def test_strided_arguments():
    """Lists and scores that are views, heads a row apart, positions of any sign; odd strides that matter are refused."""
    c = ref.Case(2, 2, 64, 16, [100, 90], [1, 1], seed=30)
    cache, _, q, k, v, tables, lens, _ = c.device()
    pages, counts = pref.choose(c, 4, 2, 1)
    want = attend.kv_attend(cache, 0, q, tables, lens, pages=pages.to(DEV), counts=counts.to(DEV))
    wide = torch.full((2, 5, 9), 2**30, dtype=torch.int32, device=DEV)
    wide[:, 1::3, 2:6] = pages.to(DEV)
    got = attend.kv_attend(cache, 0, q, tables, lens, pages=wide[:, 1::3, 2:6], counts=counts.to(DEV))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(TypeError):
        attend.kv_attend(cache, 0, q, tables, lens, pages=wide[..., ::2], counts=counts.to(DEV))
    with pytest.raises(ValueError):
        attend.kv_attend(cache, 0, q, tables, lens, pages=wide)
    with pytest.raises(ValueError):
        attend.kv_attend(cache, 0, q, tables, lens, counts=counts.to(DEV))
    with pytest.raises(kvx.KvError):  # weights of what they do not go with
        attend.kv_attend(cache, 0, q, tables, lens, pages=wide[:, :2, :4], counts=counts.to(DEV),
                         weights=torch.zeros(2, 2, 112, device=DEV))
    with pytest.raises(RuntimeError):
        attend.kv_rotate(cache, 0, q.clone().requires_grad_(), k, v, tables, lens)
    with pytest.raises(TypeError):
        attend.kv_rotate(cache, 0, q, k, v, tables, lens, freqs=torch.ones(32, device=DEV))
    with pytest.raises(TypeError):
        attend.kv_rotate(cache, 0, q, k, v, tables, lens, q_weight=torch.ones(63, device=DEV))
    with pytest.raises(ValueError):
        attend.kv_rotate(cache, 0, q, k, v, tables, lens, magnitude=0.0)
    with pytest.raises(kvx.KvError):
        attend.kv_rotate(cache, 0, q, k, v, tables, lens, freqs=torch.ones(33, dtype=torch.float64, device=DEV))
    low_high, _ = bounds_cache(c, 1.0)
    with pytest.raises(TypeError):
        attend.kv_bounds(cache, 0, low_high, tables, lens)
    with pytest.raises(ValueError):
        attend.kv_score(low_high, 0, q, tables, lens, block_size=16, out=torch.zeros(2, 2, 3, device=DEV))
