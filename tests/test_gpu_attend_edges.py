"""Edges of the operators on the paged cache: bounds at the ends of 32 bits, plans that only large batches reach, and
streams that are not the current one.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import attend_reference as ref
from harness import gpu
from paper_2609_15021_amd import attend, kvx

pytestmark = pytest.mark.gpu
DEV = ref.DEV
BF16, F16 = torch.bfloat16, torch.float16
INTS = dict(dtype=torch.int32, device=DEV)


@pytest.fixture(autouse=True)
def no_faults():
    attend.kv_attend_async_error(clear=True)
    yield
    torch.cuda.synchronize()
    assert attend.kv_attend_async_error(clear=True) == 0


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 70, 70])
@pytest.mark.parametrize("new", [[70, 3], [5, 2], [1, 1]])
def test_windows_that_hide_nothing(window, new):
    """The widest windows are no window, for rows that would lie before token 0 too: outputs and received weights."""
    c = ref.Case(2, 3, 64, 16, [3, 40], new, seed=31)
    cache, _, q, _, _, tables, lens, starts = c.device()
    want = ref.attend(c)
    weights = torch.zeros(2, 2, 40, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, window=window, weights=weights)
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")


@pytest.mark.parametrize("new", [100, 1])
def test_longest_sequence(new):
    """A sequence of 2^31 - 1024 tokens, all pages but the last being one and the same: its last tokens, whose scores are
    90 above the others' (which weigh 2^31 exp(-90) or 2e-30 together), are all that counts."""
    BS, D = 4096, 8
    n = 2**31 - 1024
    pages = n // BS + 1
    gen = torch.Generator().manual_seed(32)
    t = torch.zeros(2, 2, 1, BS, D)
    t[0, 1] = 7.0
    t[1, 0, 0, :, 0] = 8.0
    t[1, 0, 0, :, 1] = torch.randn(BS, generator=gen)
    t[1, 1] = torch.randn(1, BS, D, generator=gen)
    t = t.to(BF16)
    q = torch.zeros(new, 1, D, dtype=BF16)
    q[:, 0, 0] = 32.0
    q[:, 0, 1] = torch.randn(new, generator=gen).to(BF16)
    cache = kvx.Cache([t.to(DEV)], kvx.make_layout(1, 1, D, 2, BS, BS), 2)
    tables = torch.zeros(1, pages, **INTS)
    tables[0, -1] = 1
    weights = torch.full((1, 1, n), 5.0, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q.to(DEV), tables, torch.tensor([n], **INTS), torch.tensor([0, new], **INTS),
                                weights=weights)
    got = np.zeros(BS)
    k, v = (t[1, i, 0].double().numpy() for i in (0, 1))
    for i in range(new):
        seen = n - new + i - (pages - 1) * BS + 1
        s = k[:seen] @ q[i, 0].double().numpy() / np.sqrt(D)
        w = np.exp(s - s.max())
        total = w.sum()
        w /= total
        # A score is off by 8 additions and its roundings, a weight by that and half a step, the sums by 16 tokens at a time.
        off = 2.0**-23 * (8 * np.abs(s).max() + 64 + seen / 16) * 4
        magnitude = w @ np.abs(v[:seen])
        want = w @ v[:seen]
        ref.check(out[i, 0], want, 2.0**-8 * (np.abs(want) + magnitude) + off * magnitude, "out")
        assert abs(float(lse[i, 0]) - (s.max() + np.log(total))) <= off + 2.0**-22 * 100
        got[:seen] += w
    # (A weight is off by its score's error and lse's, and by a rounding for each of the rows.)
    last = weights[0, 0, n - seen:].double().cpu().numpy()
    assert (np.abs(last - got[:seen]) <= got[:seen] * (2 * off + 2.0**-22 * 100 + new * 2.0**-23) + 1e-30).all()
    assert float(weights[0, 0, :n - seen].max()) < 1e-30


def test_weights_of_wide_bounds():
    """Bounds so wide that scores for all of them would take more than a GiB: weights are taken without them."""
    c = ref.Case(2, 16, 64, 16, [300, 77, 1], [1, 1, 1], seed=33)
    cache, _, q, _, _, tables, lens, _ = c.device()
    most = 3_000_000
    tables = torch.nn.functional.pad(tables, (0, most // 16 - tables.shape[1]), value=-1)
    want = ref.attend(c)
    weights = torch.zeros(3, 2, most, device=DEV)
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, weights=weights, max_len=most)
    assert torch.cuda.max_memory_allocated() - before <= 1 << 30
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")
        assert not weights[b, :, n:].any()


def fine(c, **options):
    """(reference, bound of out) where the weights exp(s - m) meet V as two numbers of the rows' type: in place of half a
    step of each weight, a half step of a half step (its square), and for float16 half of its smallest number, 2^-25, at
    weights of which the largest is at least 2^7."""
    want = ref.attend(c, **options)
    c.v, v = [np.abs(x) for x in c.v], c.v
    magnitude = ref.attend(c, **options)[0]
    c.v = v
    half = ref.HALF_STEP[c.dtype]
    largest = max((np.abs(x).max() for x in c.v if x.size), default=0.0) * c.v_scale
    tiny = max(c.lens) * 2.0**-32 * largest if c.dtype == F16 else 0.0
    return want, want[3] - half * magnitude + half * half * magnitude + tiny


@pytest.mark.parametrize("lens,new", [([1, 33, 700, 3000], [1, 1, 1, 1]), ([40, 300, 900], [2, 3, 4])])
@pytest.mark.parametrize("H,G,D,fp8,dtype", [(2, 5, 128, False, BF16), (1, 16, 64, False, F16), (1, 6, 256, True, BF16),
                                              (2, 12, 80, True, F16), (1, 4, 200, False, BF16)])
def test_few_rows_round_once(H, G, D, fp8, dtype, lens, new):
    """Sequences of up to 64 rows per KV head: only the output's rounding shows."""
    c = ref.Case(H, G, D, 16, lens, new, fp8=fp8, dtype=dtype, seed=34 + D)
    cache, _, q, _, _, tables, ln, starts = c.device()
    out, lse = attend.kv_attend(cache, 0, q, tables, ln, starts, k_scale=c.k_scale, v_scale=c.v_scale)
    want, off = fine(c)
    ref.check(out, want[0], off, "out")
    ref.check(lse, want[1], want[4], "lse")


@pytest.mark.parametrize("options", [{}, dict(softcap=5.0, window=90), dict(slopes=True)])
@pytest.mark.parametrize("lens,new", [([100, 33, 700], [100, 1, 70]), ([3000, 130], [70, 129])])
@pytest.mark.parametrize("H,G,D,fp8,dtype", [(2, 2, 128, False, BF16), (1, 3, 64, False, F16), (1, 2, 256, True, BF16),
                                              (1, 4, 80, True, F16), (1, 2, 200, False, F16), (1, 1, 64, True, BF16)])
def test_full_weights_round_once(H, G, D, fp8, dtype, lens, new, options):
    """Sequences of more than 64 rows too, whole and in parts, where the caller asks for it; lse and what tokens receive
    are the same either way."""
    c = ref.Case(H, G, D, 16, lens, new, fp8=fp8, dtype=dtype, seed=45 + D)
    cache, _, q, _, _, tables, ln, starts = c.device()
    plain = dict(options)
    if options.get("slopes"):
        plain["slopes"] = np.array([2.0**-(1 + i % 7) for i in range(H * G)])
        options = dict(slopes=torch.tensor(plain["slopes"], dtype=torch.float32, device=DEV))
    got = []
    for full in (True, False):
        weights = torch.zeros(len(lens), H, max(lens), device=DEV)
        got.append((*attend.kv_attend(cache, 0, q, tables, ln, starts, k_scale=c.k_scale, v_scale=c.v_scale, **options,
                                      weights=weights, full_weights=full), weights))
    want, off = fine(c, **plain)
    ref.check(got[0][0], want[0], off, "out")
    ref.check(got[0][1], want[1], want[4], "lse")
    ref.check(got[1][0], want[0], want[3], "out")
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])
    few = slice(int(c.starts[1]), int(c.starts[2])) if new[1] * G <= 64 else slice(0, 0)
    assert torch.equal(got[0][0][few], got[1][0][few])


@pytest.mark.parametrize("D,dtype", [(128, BF16), (64, F16), (256, BF16)])
def test_hundreds_of_parts(D, dtype):
    """One sequence on one KV head, cut into more parts than the join reads at first."""
    c = ref.Case(1, 2, D, 16, [33003], [1], dtype=dtype, seed=35 + D)
    cache, _, q, _, _, tables, lens, _ = c.device()
    weights = torch.zeros(1, 1, 33003, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, weights=weights)
    want, off = fine(c)
    ref.check(out, want[0], off, "out")
    ref.check(lse, want[1], want[4], "lse")
    ref.check(weights, want[2], want[5], "weights")


def test_more_sequences_than_one_round_lists():
    """Over 1,024 sequences, long ones on both sides of the 1,024th, shared out in parts of 512 tokens and more."""
    gen = np.random.default_rng(36)
    lens = [int(n) for n in gen.integers(0, 12, 1100)]
    for b, n in ((3, 700), (1023, 1300), (1024, 513), (1090, 1025)):
        lens[b] = n
    c = ref.Case(1, 2, 16, 8, lens, [1 if n % 7 else 0 for n in lens], seed=36)
    cache, _, q, _, _, tables, ln, starts = c.device()
    weights = torch.zeros(1100, 1, 1300, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q, tables, ln, starts, max_q=1, weights=weights)
    want = ref.attend(c)
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")


def test_keep_rows_of_several_sets():
    """128 rows, some of more than 262,144 tokens, with ties on both sides of that and of twice that."""
    L, B = 2 * 262144 + 5000, 128
    lens = [min(L, 50 + 7 * b) for b in range(B)]
    lens[5], lens[64], lens[127] = L, 262145, 262144
    gen = torch.Generator().manual_seed(37)
    w = torch.zeros(B, 1, L)
    for b in (5, 64, 127):
        w[b, 0] = (torch.rand(L, generator=gen) * 8).floor()  # an eighth of the tokens for each value
    w[:, 0, :1000] = torch.rand(B, 1000, generator=gen)
    w[5, 0, 262100:262200] = 9.0
    device = w.to(DEV)
    for budget in (40000, 300000):
        got = attend.kv_keep(device, torch.tensor(lens, **INTS), budget, sinks=4, recent=1000)
        for b in (0, 5, 64, 127):
            want = ref.keep(w[b:b + 1].numpy(), lens[b:b + 1], budget, 4, 1000)
            assert torch.equal(got[0][b:b + 1].cpu(), torch.from_numpy(want[0])) and int(got[1][b]) == want[1][0]
            assert np.array_equal(got[2][b:b + 1].cpu().numpy(), want[2])


def test_keep_very_long_rows():
    """128 rows, one of 20 million tokens (77 sets of rounds, each of which is read once per step and no more): few
    values, so that ties are everywhere, and a choice that ends in the first, in a middle and in the last set."""
    L, B = 20_000_003, 128
    w = (torch.rand(L, generator=torch.Generator().manual_seed(43)) * 50).floor()
    w[-3000:] += 100.0
    rows = w.to(DEV).expand(B, 1, L)  # one row in memory
    lens = [100 + b for b in range(B)]
    lens[77] = L
    far = w.numpy()
    for budget, sinks, recent in ((100_000, 7, 5), (3_000_000, 0, 100), (19_900_000, 4, 1000)):
        keep, kept, kw = attend.kv_keep(rows, torch.tensor(lens, **INTS), budget, sinks=sinks, recent=recent)
        middle = far[sinks:L - recent]
        heavy = np.sort(np.argsort(-middle, kind="stable")[:budget - sinks - recent]) + sinks
        want = np.concatenate([np.arange(sinks), heavy, np.arange(L - recent, L)])
        assert np.array_equal(keep[77, 0].cpu().numpy(), want) and np.array_equal(kw[77, 0].cpu().numpy(), far[want])
        assert kept.cpu().tolist() == [min(n, budget) for n in lens]
        assert torch.equal(keep[3, 0, :103].cpu(), torch.arange(103, dtype=torch.int32)) and (keep[3, 0, 103:] == -1).all()


@pytest.mark.parametrize("n", [1, 77])
def test_one_token_with_any_stride(n):
    """A batch of one new token cut from wider tensors, whose strides between tokens (and of single entries) are odd."""
    c = ref.Case(1, 3, 64, 16, [n], [1], seed=44)
    cache, t, q, k, v, tables, lens, _ = c.device()
    wide = torch.zeros(2, 5 * 64 + 1, dtype=BF16, device=DEV)
    parts = wide[:, :320].view(2, 5, 64)[:1]
    parts[:, :3], parts[:, 3:4], parts[:, 4:] = q, k, v
    meta = torch.zeros(1, 7, **INTS)
    meta[0, 3] = n
    assert parts.stride(0) == 321 and meta[:, 3].stride() == (7,)
    attend.kv_append(cache, 0, parts[:, 3:4], parts[:, 4:], tables, meta[:, 3])
    out, lse = attend.kv_attend(cache, 0, parts[:, :3], tables, meta[:, 3])
    for rows, stored in ((c.k, c.new_k), (c.v, c.new_v)):
        rows[0][n - 1] = stored[0].double().numpy()
    want = ref.attend(c)
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    keep, kept, _ = attend.kv_keep(torch.ones(1, 1, 3 * n, device=DEV)[:, :, ::3][:, :, :1], meta[:, 0], 2)
    assert keep.tolist() == [[[-1, -1]]] and kept.tolist() == [0]


@pytest.mark.parametrize("new", [1, 3, 40])
def test_sequences_of_no_tokens_and_no_pages(new):
    """A batch in which nothing is cached yet, its tables without an entry: rows of 0 and -infinity, nothing written."""
    c = ref.Case(2, 3, 64, 16, [5], [1], seed=46)
    cache, t, _, _, _, _, _, _ = c.device()
    before = t.clone()
    tables, lens = torch.zeros(2, 0, **INTS), torch.zeros(2, **INTS)
    starts = torch.tensor([0, new, 2 * new], **INTS)
    q, k = torch.ones(2 * new, 6, 64, dtype=BF16, device=DEV), torch.ones(2 * new, 2, 64, dtype=BF16, device=DEV)
    weights = torch.full((2, 2, 7), 3.0, device=DEV)
    attend.kv_append(cache, 0, k, k, tables, lens, starts)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, weights=weights, prior=weights)
    assert not out.any() and (lse == -torch.inf).all() and (weights == 3).all()
    assert torch.equal(t.view(torch.int16), before.view(torch.int16))


def test_streams_by_handle():
    """The null stream and torch's default stream, named."""
    c = ref.Case(2, 4, 128, 16, [3000, 40], [1, 1], seed=47)
    cache, _, q, _, _, tables, lens, _ = c.device()
    want = ref.attend(c)
    torch.cuda.synchronize()
    for stream in (0, torch.cuda.default_stream(), torch.cuda.current_stream().cuda_stream):
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, stream=stream)
        torch.cuda.synchronize()
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")


def test_group_beyond_a_step():
    """One new token of more query heads per KV head than the kernel for few rows takes."""
    for fp8 in (False, True):
        c = ref.Case(1, 100, 64, 16, [1, 130, 0], [1, 1, 1], fp8=fp8, seed=38)
        cache, _, q, _, _, tables, lens, _ = c.device()
        weights = torch.zeros(3, 1, 130, device=DEV)
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, k_scale=c.k_scale, v_scale=c.v_scale, weights=weights)
        want = ref.attend(c)
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")
        for b, n in enumerate(c.lens):
            ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")


def _overwrite(*shapes):
    """Fills what the allocator has free for tensors of these shapes on the current stream."""
    for shape, dtype in shapes:
        for _ in range(4):
            torch.empty(shape, dtype=dtype, device=DEV).fill_(-3)


def test_named_stream_keeps_what_it_reads():
    """Calls on a stream that is behind: their inputs are dropped at once, and the memory that the allocator then hands
    out on the current stream is overwritten before the calls run."""
    c = ref.Case(2, 4, 128, 16, [300, 40], [1, 1], seed=39)
    cache, t, q0, k0, v0, tables0, lens0, starts0 = c.device()
    s = torch.cuda.Stream()
    results, scales = [], (1.0, 0.5, -1.0, 0.25)
    for scale in scales:
        q, slopes = q0 * scale, torch.full((8,), 0.01, device=DEV)
        tables, lens, starts = tables0.clone(), lens0.clone(), starts0.clone()
        weights, prior = torch.zeros(2, 2, 300, device=DEV), torch.zeros(2, 2, 300, device=DEV)
        s.wait_stream(torch.cuda.current_stream())
        gpu.spin(20.0, s)
        out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, slopes=slopes, weights=weights, prior=prior,
                                    stream=s)
        shapes = [(x.shape, x.dtype) for x in (q, slopes, tables, lens, starts, prior)]
        del q, slopes, tables, lens, starts, prior
        _overwrite(*shapes)
        results.append((out, lse, weights))
    torch.cuda.synchronize()
    for scale, (out, lse, weights) in zip(scales, results):
        d = ref.Case(2, 4, 128, 16, [300, 40], [1, 1], seed=39)
        d.q = d.q * scale
        want = ref.attend(d, slopes=np.full(8, float(np.float32(0.01))))
        ref.check(out, want[0], want[3], "out")
        ref.check(lse, want[1], want[4], "lse")
        for b, n in enumerate(d.lens):
            ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")

    # The other calls, each behind a spin of its own.
    w0 = torch.rand(2, 2, 300, device=DEV)
    k, v, tables, lens = k0.clone(), v0.clone(), tables0.clone(), lens0.clone()
    fresh0 = torch.tensor([c.free[:2]], **INTS)
    w, keep0 = w0.clone(), torch.tensor([[[3, 9, 299]]], **INTS)
    kept0 = torch.tensor([3], **INTS)
    source, keep, kept, fresh = tables0[:1].clone(), keep0.clone(), kept0.clone(), fresh0.clone()
    lens_again = lens0.clone()
    s.wait_stream(torch.cuda.current_stream())
    gpu.spin(20.0, s)
    attend.kv_append(cache, 0, k, v, tables, lens, stream=s)
    chosen = attend.kv_keep(w, lens_again, 50, sinks=1, recent=9, stream=s)
    attend.kv_compact(cache, 0, source, keep, kept, fresh, stream=s)
    shapes = [(x.shape, x.dtype) for x in (k, v, tables, lens, w, lens_again, source, keep, kept, fresh)]
    del k, v, tables, lens, w, lens_again, source, keep, kept, fresh
    _overwrite(*shapes)
    torch.cuda.synchronize()
    want = ref.keep(w0.cpu().numpy(), c.lens, 50, 1, 9)
    assert torch.equal(chosen[0].cpu(), torch.from_numpy(want[0])) and np.array_equal(chosen[2].cpu().numpy(), want[2])
    now = t.cpu().view(c.num_blocks, *c.shape)
    for b, n in enumerate(c.lens):
        page = now[int(c.tables[b, (n - 1) // 16])]
        assert torch.equal(page[0, :, (n - 1) % 16], c.new_k[b]) and torch.equal(page[1, :, (n - 1) % 16], c.new_v[b])
    moved = now[c.free[0]]
    for j, token in enumerate((3, 9)):
        np.testing.assert_array_equal(moved[0, :, j].double().numpy(), c.k[0][token])
        np.testing.assert_array_equal(moved[1, :, j].double().numpy(), c.v[0][token])
    assert torch.equal(moved[0, :, 2], c.new_k[0])


def test_two_calls_at_once():
    """Two streams, each with calls of its own in a row: no workspace is shared."""
    cases = [ref.Case(2, 5, 128, 16, [5000, 17], [1, 1], seed=40), ref.Case(2, 5, 128, 16, [5000, 900], [40, 100], seed=41)]
    state, want = [c.device() for c in cases], [ref.attend(c) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (s, (cache, _, q, _, _, tables, lens, starts)) in enumerate(zip(streams, state)):
            weights = torch.zeros(2, 2, 5000, device=DEV)
            s.wait_stream(torch.cuda.current_stream())
            results[i].append((*attend.kv_attend(cache, 0, q, tables, lens, starts, weights=weights, stream=s), weights))
    torch.cuda.synchronize()
    for c, got, (out, lse, weights, out_off, lse_off, weights_off) in zip(cases, results, want):
        ref.check(got[0][0], out, out_off, "out")
        ref.check(got[0][1], lse, lse_off, "lse")
        for b, n in enumerate(c.lens):
            ref.check(got[0][2][b, :, :n], weights[b, :, :n], weights_off[b, :, :n], "weights")
        for again in got[1:]:
            for x, y in zip(got[0], again):
                assert torch.equal(x, y)


FIRST_CALL_CAPTURED = """
import sys
sys.path[:0] = sys.argv[1:]
import torch
import attend_reference as ref
from paper_2609_15021_amd import attend
c = ref.Case(2, 4, 64, 16, [300, 40], [1, 1], seed=42)
cache, _, q, k, v, tables, lens, _ = c.device()
weights = torch.zeros(2, 2, 300, device=ref.DEV)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, weights=weights)
want = ref.attend(c)
for _ in range(3):
    out.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
print("replayed")
"""


def test_first_call_of_a_process_may_be_captured():
    here = os.path.dirname(os.path.abspath(__file__))
    got = subprocess.run([sys.executable, "-c", FIRST_CALL_CAPTURED, here, os.path.dirname(here)], capture_output=True,
                         text=True, timeout=100)
    assert got.returncode == 0 and "replayed" in got.stdout, got.stderr[-2000:]
