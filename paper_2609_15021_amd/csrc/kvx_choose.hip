// kv_bounds and kv_score: what pages can score at most with a query, so that each new token can choose the pages that
// it attends over.
//
// For lo <= k <= hi in every column, q.k <= sum_d max(q_d lo_d, q_d hi_d), and the larger product is q_d hi_d where q_d
// is positive and q_d lo_d elsewhere: with q+ = max(q, 0) and q- = min(q, 0) the bound is q+.hi + q-.lo, two products
// on the matrix cores.
//
// Bounds: a group of lanes has a page and head, 16 bytes of its columns a lane, and takes the page's rows one after the
// other, so nothing passes between lanes: bound by reading K once.  Where there are few pages their rows are spread
// over the wave's groups instead, and joined by lane shuffles.  131,077 tokens of 8 heads of 128 (bf16, 302 MB): 57 us,
// 5.3 TB/s (a large copy moves 4.7); the pages of 48 new tokens (4 heads of 256, e4m3): 4.6 us, launch and waits.
//
// Scores: a wave holds the bounds of 16 or 32 pages in registers as the products' second operand (column: page), and
// goes over its share of the rows, 16 (new token, query head) at a time, as the first.  A token's heads are padded to a
// power of two by repeating the last, so that the largest over them lies in a lane's 4 results, or one or two shuffles
// away.  8,193 pages of 8 heads of 5 rows (34 MB, D 128): 8.7 us, of which reading takes 5.6 and table, bounds and
// products come one after the other.  Tails of up to 517 tokens over 1,057 pages, 3 sequences, 2 heads of 8 rows: 19
// us, the matrix cores busy for 11% of it: a wave's share of tiles is short, and its start (lengths, table, bounds) and
// every second tile's wait for the workgroup are not hidden.
#include <algorithm>
#include <cmath>

#include "kvx_attend_kernels.h"

namespace kvx {

namespace {

// ---- Bounds -------------------------------------------------------------------------------

struct BoundsArgs {
    Pages pages, bounds;
    Batch batch;
    int32_t touched;  // most pages of a sequence that new tokens lie in
};

// 16 bytes of a row as numbers, and back.  TYPE: KV_DTYPE_*.
template <int TYPE>
struct Piece {
    static constexpr int N = TYPE == KV_DTYPE_E4M3 ? 16 : 8;
    static __device__ __forceinline__ void read(const u32x4 &x, float *y) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (TYPE == KV_DTYPE_E4M3) {
                const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(x[w]), false);
                const auto high = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(x[w]), true);
                y[4 * w] = low[0];
                y[4 * w + 1] = low[1];
                y[4 * w + 2] = high[0];
                y[4 * w + 3] = high[1];
            } else if constexpr (TYPE == KV_DTYPE_BF16) {
                y[2 * w] = Bf16::low(x[w]);
                y[2 * w + 1] = Bf16::high(x[w]);
            } else {
                y[2 * w] = F16::low(x[w]);
                y[2 * w + 1] = F16::high(x[w]);
            }
        }
    }
    static __device__ __forceinline__ u32x4 write(const float *y) {
        u32x4 x;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (TYPE == KV_DTYPE_E4M3) {
                const int low = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
                x[w] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], low, true));
            } else if constexpr (TYPE == KV_DTYPE_BF16) {
                x[w] = Bf16::pack(y[2 * w], y[2 * w + 1]);
            } else {
                x[w] = F16::pack(y[2 * w], y[2 * w + 1]);
            }
        }
        return x;
    }
};

// LPR lanes have a row; SPREAD: a wave has one page, else one for each of its groups of lanes.  AT_ONCE: rows that a
// lane has on their way.  131,077 tokens of 8 heads of 128 in pages of 16 take 57 us with 16 of them and 60 with 8 in
// bfloat16, but 71 and 60 in float16, where the compiler does not keep 16 apart, and 30 with either in e4m3.
template <int TYPE, int LPR, bool SPREAD, int AT_ONCE>
__global__ __launch_bounds__(kThreads) void bounds_kernel(const BoundsArgs a) {
    constexpr int N = Piece<TYPE>::N, GROUPS = 64 / LPR;
    const Pages &p = a.pages;
    const int b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sequence s;
    if (!sequence(a.batch, b, p.err, s) || s.nq == 0 || s.n == 0)
        return;
    const int group = lane / LPR, vec = lane % LPR;
    const int64_t item = (int64_t{blockIdx.x} * (kThreads / 64) + wave) * (SPREAD ? 1 : GROUPS) + (SPREAD ? 0 : group);
    // (Heads run fastest: a page's heads lie behind each other.)
    const int64_t page64 = divide(max(s.n - s.nq, 0), p.by_bs) + item / p.H;
    const int h = static_cast<int>(item % p.H);
    if (item / p.H >= a.touched || page64 * p.BS >= s.n)
        return;
    const int page = static_cast<int>(page64), rows = min(p.BS, s.n - page * p.BS);
    const int block = a.batch.tables[b * a.batch.table_stride + page];
    if (!in_cache(p, block))
        return;
    const bool any = vec * 16 < p.row_bytes;
    const uint8_t *from = p.base + page_offset(p, block, 0, h) + (any ? vec * 16 : 0);
    float low[N], high[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        low[j] = INFINITY;
        high[j] = -INFINITY;
    }
    // (The last row again in place of those behind it.)
    constexpr int STEP = SPREAD ? GROUPS : 1;
    for (int row = SPREAD ? group : 0; row < rows; row += AT_ONCE * STEP) {
        u32x4 x[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(
                from + static_cast<uint32_t>(min(row + k * STEP, rows - 1)) * p.token_bytes));
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            float y[N];
            Piece<TYPE>::read(x[k], y);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                low[j] = fminf(low[j], y[j]);  // (the other one, if one is NaN)
                high[j] = fmaxf(high[j], y[j]);
            }
        }
    }
    if constexpr (SPREAD) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                low[j] = fminf(low[j], __shfl_xor(low[j], o));
                high[j] = fmaxf(high[j], __shfl_xor(high[j], o));
            }
    }
    if (!any || (SPREAD && group > 0))
        return;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (low[j] > high[j])
            low[j] = high[j] = 0.f;
    uint8_t *to = a.bounds.base + page_offset(a.bounds, block, 0, h) + vec * 16;
    *reinterpret_cast<u32x4 *>(to) = Piece<TYPE>::write(low);
    *reinterpret_cast<u32x4 *>(to + a.bounds.v_bytes) = Piece<TYPE>::write(high);
}

template <int TYPE, int LPR>
hipError_t launch_bounds(const BoundsArgs &a, int num_seqs, hipStream_t stream) {
    // A wave to a page while that leaves waves to spare (8 a SIMD).
    const int64_t items = int64_t{a.touched} * a.pages.H, waves = kThreads / 64;
    const bool spread = items * num_seqs <= 8192;
    const int64_t each = waves * (spread ? 1 : 64 / LPR);
    const dim3 grid(static_cast<uint32_t>((items + each - 1) / each), static_cast<uint32_t>(num_seqs));
    constexpr int MOST = TYPE == KV_DTYPE_BF16 ? 16 : 8;
    const auto kernel = spread            ? bounds_kernel<TYPE, LPR, true, 4>
                        : a.pages.BS <= 8 ? bounds_kernel<TYPE, LPR, false, 8>
                                          : bounds_kernel<TYPE, LPR, false, MOST>;
    return launch_kernel(kernel, grid, kThreads, stream, a);
}

template <int TYPE>
hipError_t launch_bounds(const BoundsArgs &a, int num_seqs, hipStream_t stream) {
    const int vecs = a.pages.row_bytes / 16;
    return vecs > 16  ? launch_bounds<TYPE, 32>(a, num_seqs, stream)
           : vecs > 8 ? launch_bounds<TYPE, 16>(a, num_seqs, stream)
                      : launch_bounds<TYPE, 8>(a, num_seqs, stream);
}

// The checks of a cache of bounds, beside check_layer's.
kv_status check_bounds(const kv_cache *bounds) {
    if (bounds->layout.block_size != 1)
        return fail(KV_EINVAL, "bounds have one token a block, not %d", bounds->layout.block_size);
    return KV_OK;
}

kv_status bounds_of(const kv_cache *cache, int32_t layer, const kv_batch *batch, int32_t cache_dtype,
                    const kv_cache *bounds, hipStream_t stream) {
    kv_status st = check_layer(cache, layer);
    if (st == KV_OK)
        st = check_dtype(cache, cache_dtype);
    if (st == KV_OK)
        st = check_batch(cache, batch);
    if (st == KV_OK)
        st = check_layer(bounds, layer);
    if (st == KV_OK)
        st = check_bounds(bounds);
    if (st != KV_OK)
        return st;
    const kv_layout &x = cache->layout, &y = bounds->layout;
    if (x.num_kv_heads != y.num_kv_heads || x.head_dim != y.head_dim || x.elem_bytes != y.elem_bytes)
        return fail(KV_EINVAL, "bounds of %d heads of %d elements of %d bytes for a cache of %d of %d of %d",
                    y.num_kv_heads, y.head_dim, y.elem_bytes, x.num_kv_heads, x.head_dim, x.elem_bytes);
    if (bounds->num_blocks < cache->num_blocks)
        return fail(KV_EINVAL, "bounds of %d blocks for a cache of %d", bounds->num_blocks, cache->num_blocks);
    if (bounds->device != cache->device)
        return fail(KV_EINVAL, "cache is on device %d, bounds on device %d", cache->device, bounds->device);
    const int most = std::min({batch->max_queries, batch->num_queries, batch->max_len});
    if (batch->num_seqs == 0 || most == 0)
        return KV_OK;
    st = check_on_current_device(cache);
    int32_t *err = nullptr;
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    BoundsArgs a{};
    a.pages = pages_of(cache, layer, err);
    a.bounds = pages_of(bounds, layer, err);
    a.batch = batch_of(batch);
    const int64_t touched = (int64_t{most} + a.pages.BS - 2) / a.pages.BS + 1;
    if (touched * a.pages.H > INT32_MAX / 64)
        return fail(KV_EUNSUPPORTED, "%lld pages of %d heads in one call are too many", static_cast<long long>(touched),
                    a.pages.H);
    a.touched = static_cast<int32_t>(touched);
    KVX_HIP(cache_dtype == KV_DTYPE_BF16  ? launch_bounds<KV_DTYPE_BF16>(a, batch->num_seqs, stream)
            : cache_dtype == KV_DTYPE_F16 ? launch_bounds<KV_DTYPE_F16>(a, batch->num_seqs, stream)
                                          : launch_bounds<KV_DTYPE_E4M3>(a, batch->num_seqs, stream));
    return KV_OK;
}

// ---- Scores -------------------------------------------------------------------------------

struct ScoreArgs {
    Pages bounds;
    Batch batch;
    Rows q;
    Scales scales;
    float *scores;
    int32_t *counts;
    int64_t token_stride, head_stride;  // elements
    float scale;
    int32_t BS, group, pad, shift;      // tokens of a page; query heads of a KV head, padded to 2^shift, up to 16
    int32_t shares, tokens;             // workgroups that share a sequence's tokens; tokens of each
    Divisor by_bs, by_shares, by_subs;
};

// Workgroups that tails are shared out to: 20 us for the tails above (2-byte bounds, D 128, of which 1,024 workgroups
// run at once; half of the launched ones may have no tokens); a third of them take 26, twice as many 24.  Other
// variants, of which 512 (wide e4m3) to 1,280 (up to 64 columns) run at once, have not been tried with other numbers.
constexpr int kShareTarget = 1536;

typedef short s16x2 __attribute__((ext_vector_type(2)));

// Of two numbers of 2 bytes their positive (or negative) parts: a sign bit makes either type's bits a negative integer.
__device__ __forceinline__ uint32_t positive(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, x), s16x2{0, 0}));
}
__device__ __forceinline__ uint32_t negative(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, x), s16x2{0, 0}));
}

__device__ __forceinline__ float from_lane(float x, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(lane * 4, __builtin_bit_cast(int, x)));
}

// Loads of 64 bytes of each of 16 rows, as the operands want them, come from the caches far slower than loads of whole
// rows.  So rows are loaded whole, and turned in LDS: bounds once for each wave, queries by the workgroup for all its
// waves, twice, so that the next are on their way while one set is used (the tails above took 36 us before).  Pieces of
// 16 bytes are permuted there, row by row, so that 16 rows' same piece lies in different banks.
//
// T: type of q; FP8: bounds are e4m3; DP >= D columns; PG: 16 pages of a wave; OUT: tokens that a lane has results of
// (4 heads are a lane's 4 results: 1 where a token's fill them, 2 or 4 of 2 heads or 1).
template <class T, bool FP8, int DP, int PG, int OUT>
__global__ __launch_bounds__(kThreads, 2) void score_kernel(const ScoreArgs a) {
    constexpr int E = FP8 ? 1 : 2, WAVES = kThreads / 64;
    constexpr int GB = DP * E / 16, KC = GB / 4;        // pieces of a row of bounds, and of them a lane's
    constexpr int NB = GB / 4;                          // loads of 16 rows by a wave
    constexpr int GQ = DP / 8, KQ = GQ / 4;             // the same of a row of queries
    constexpr int TILES = DP > 128 ? 1 : 2;             // of 16 rows that the workgroup loads at once
    constexpr int NQ = TILES * GQ * 16 / kThreads > 0 ? TILES * GQ * 16 / kThreads : 1;  // loads of them
    constexpr int kQueries = TILES * GQ * 16, kBounds = GB * 16;  // pieces
    __shared__ u32x4 lds[2 * kQueries > WAVES * kBounds ? 2 * kQueries : WAVES * kBounds];
    const Pages &pg = a.bounds;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, wave = tid >> 6;
    // (Heads run fastest, so that a head's workgroups come 8 apart where there are 8 heads, and so on one XCD, and then
    // the shares that read the same bounds: 512 new tokens over 2,048 pages, 8 heads of 5 rows, 55 us instead of 59.)
    const int b = blockIdx.y, place = blockIdx.x / pg.H, h = blockIdx.x - place * pg.H;
    const int chunk = divide(place, a.by_shares), share = place - chunk * a.shares;
    const int page0 = (chunk * WAVES + wave) * 16 * PG;
    // (The table is read, within what may be, while the sequence is looked up.)
    int blocks[PG];
#pragma unroll
    for (int j = 0; j < PG; ++j)
        blocks[j] = a.batch.table_len > 0 ? a.batch.tables[b * a.batch.table_stride +
                                                           min(page0 + j * 16 + c, a.batch.table_len - 1)] : -1;
    Sequence s;
    if (!sequence(a.batch, b, pg.err, s))
        return;
    const int64_t i64 = int64_t{share} * a.tokens;
    if (i64 >= s.nq)
        return;
    const int i0 = static_cast<int>(i64), i1 = static_cast<int>(min(i64 + a.tokens, int64_t{s.nq}));
    const int past = s.n - s.nq;
    if (a.counts && chunk == 0 && h == 0)
        for (int i = i0 + tid; i < i1; i += kThreads)
            a.counts[s.q0 + i] = past + i < 0 ? 0 : divide(past + i, a.by_bs) + 1;
    const int last = past + i1 - 1, pages = last < 0 ? 0 : divide(last, a.by_bs) + 1;
    if (chunk * WAVES * 16 * PG >= pages)
        return;
    const bool some = page0 < pages;  // (a wave without pages helps to load the others' queries)

    // Rows of queries: row m of a tile is token m / pad (of the tile's) and one of its heads.  A tile beyond the last
    // repeats it.
    const int each = 16 >> a.shift;                     // tokens of a tile
    const int subs = (a.group + 15) / 16;               // tiles of a token, where it has more heads
    const int tiles = ((i1 - i0 + each - 1) >> (4 - a.shift)) * subs;
    u32x4 next[NQ];
    const auto request = [&](int tile0) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int u = tid + n * kThreads, row = u / GQ % 16, piece = u % GQ;
            const int tile = min(tile0 + u / (GQ * 16), tiles - 1), of = divide(tile, a.by_subs);
            const int token = min(i0 + of * each + (row >> a.shift), i1 - 1);
            const int head = h * a.group + min((row & (a.pad - 1)) + (tile - of * subs) * 16, a.group - 1);
            const uint8_t *x = a.q.data + int64_t{s.q0 + token} * a.q.token_stride + head * a.q.head_stride;
            next[n] = *reinterpret_cast<const u32x4 *>(x + (piece * 8 < pg.D ? piece * 16 : 0));
            if (piece * 8 >= pg.D)
                next[n] = u32x4{0, 0, 0, 0};  // (where bounds repeat their first columns)
        }
    };
    const auto deposit = [&](int buffer) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int u = tid + n * kThreads, row = u / GQ, piece = u % GQ;
            if (kQueries >= kThreads || u < kQueries)
                lds[buffer * kQueries + row * GQ + (piece ^ (row & (GQ - 1) & 15))] = next[n];
        }
    };
    request(0);

    // This lane's pages, their first tokens, and their bounds.
    u32x4 low[PG][KC], high[PG][KC];
    float factor[PG];
    bool good[PG];
    int start[PG];
    if (some) {
        u32x4 raw[PG][2][NB];
#pragma unroll
        for (int j = 0; j < PG; ++j) {
            const int page = page0 + j * 16 + c;
            start[j] = page < pages ? page * a.BS : INT32_MAX;
            const int block = blocks[j];
            good[j] = page < pages && in_cache(pg, block);
            factor[j] = a.scale;
            if (FP8 && a.scales.data && good[j])
                factor[j] *= power_of(*scale_at(a.scales, block, 0, h));
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int piece = lane % GB, of = __shfl(good[j] ? block : 0, n * (64 / GB) + lane / GB);
                const uint8_t *x = pg.base + page_offset(pg, of, 0, h) + (piece * 16 < pg.row_bytes ? piece * 16 : 0);
                raw[j][0][n] = *reinterpret_cast<const u32x4 *>(x);
                raw[j][1][n] = *reinterpret_cast<const u32x4 *>(x + pg.v_bytes);
            }
        }
        u32x4 *mine = lds + wave * kBounds;
#pragma unroll
        for (int j = 0; j < PG; ++j)
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const int row = n * (64 / GB) + lane / GB, piece = lane % GB;
                    mine[row * GB + (piece ^ (row & (GB - 1) & 15))] = raw[j][kv][n];
                }
                __builtin_amdgcn_wave_barrier();  // (LDS serves a wave's accesses in order)
#pragma unroll
                for (int k = 0; k < KC; ++k)
                    (kv ? high : low)[j][k] = mine[c * GB + ((k * 4 + g) ^ (c & (GB - 1) & 15))];
                __builtin_amdgcn_wave_barrier();
            }
    }
    __syncthreads();
    deposit(0);
    __syncthreads();

    float *scores = a.scores + h * a.head_stride + page0 + c;
    f32x4 best[PG];
    for (int tile0 = 0, buffer = 0; tile0 < tiles; tile0 += TILES, buffer ^= 1) {
        const bool more = tile0 + TILES < tiles;
        if (more)
            request(tile0 + TILES);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int tile = tile0 + t;
            if (tile >= tiles || !some)
                break;
            f32x4 x[PG];
#pragma unroll
            for (int j = 0; j < PG; ++j)
                x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KQ; ++k) {
                // (Of e4m3 a lane's piece has 16 columns, and the two products' queries lie side by side.)
                const int piece = FP8 ? (k >> 1) * 8 + g * 2 + (k & 1) : k * 4 + g;
                const u32x4 q = lds[buffer * kQueries + (t * 16 + c) * GQ + (piece ^ (c & (GQ - 1) & 15))];
                u32x4 up, down;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    up[w] = positive(q[w]);
                    down[w] = negative(q[w]);
                }
#pragma unroll
                for (int j = 0; j < PG; ++j) {
                    if constexpr (FP8) {
                        const int w = (k & 1) * 2;
                        const uint32_t h0 = high[j][k >> 1][w], h1 = high[j][k >> 1][w + 1];
                        x[j] = mfma_16x16x32(up, u32x4{T::from_e4m3(h0, false), T::from_e4m3(h0, true),
                                                       T::from_e4m3(h1, false), T::from_e4m3(h1, true)}, x[j], T{});
                    } else {
                        x[j] = mfma_16x16x32(up, high[j][k], x[j], T{});
                    }
                }
#pragma unroll
                for (int j = 0; j < PG; ++j) {
                    if constexpr (FP8) {
                        const int w = (k & 1) * 2;
                        const uint32_t l0 = low[j][k >> 1][w], l1 = low[j][k >> 1][w + 1];
                        x[j] = mfma_16x16x32(down, u32x4{T::from_e4m3(l0, false), T::from_e4m3(l0, true),
                                                         T::from_e4m3(l1, false), T::from_e4m3(l1, true)}, x[j], T{});
                    } else {
                        x[j] = mfma_16x16x32(down, low[j][k], x[j], T{});
                    }
                }
            }
            const int of = divide(tile, a.by_subs);
            if (subs > 1) {  // the largest over a token's tiles
                const int sub = tile - of * subs;
#pragma unroll
                for (int j = 0; j < PG; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        x[j][r] = best[j][r] = sub == 0 ? x[j][r] : fmaxf(best[j][r], x[j][r]);
                if (sub + 1 < subs)
                    continue;
            }
#pragma unroll
            for (int j = 0; j < PG; ++j) {
                f32x4 y = x[j];
                if constexpr (OUT <= 2) {
                    y[0] = fmaxf(y[0], y[1]);
                    y[1] = fmaxf(y[2], y[3]);
                }
                if constexpr (OUT == 1) {
                    y[0] = fmaxf(y[0], y[1]);
                    if (a.shift >= 3)
                        y[0] = fmaxf(y[0], from_lane(y[0], lane ^ 16));
                    if (a.shift == 4)
                        y[0] = fmaxf(y[0], from_lane(y[0], lane ^ 32));
                    if (g & ((a.pad >> 2) - 1))
                        continue;
                }
#pragma unroll
                for (int r = 0; r < OUT; ++r) {
                    const int token = i0 + of * each + (OUT == 1 ? g * 4 >> a.shift : g * OUT + r);
                    if (token < i1 && start[j] <= past + token)
                        scores[int64_t{s.q0 + token} * a.token_stride + j * 16] = good[j] ? y[r] * factor[j] : -INFINITY;
                }
            }
        }
        if (more) {
            deposit(buffer ^ 1);
            __syncthreads();
        }
    }
}

template <class T, bool FP8, int DP, int PG>
hipError_t launch_score_to(const ScoreArgs &a, const dim3 &grid, hipStream_t stream) {
    const auto kernel = a.shift == 0   ? score_kernel<T, FP8, DP, PG, 4>
                        : a.shift == 1 ? score_kernel<T, FP8, DP, PG, 2>
                                       : score_kernel<T, FP8, DP, PG, 1>;
    return launch_kernel(kernel, grid, kThreads, stream, a);
}

template <class T, bool FP8, int DP, int PG>
hipError_t launch_score(ScoreArgs a, int num_seqs, int most, int64_t pages, hipStream_t stream) {
    const int64_t chunks = (pages + 16 * PG * (kThreads / 64) - 1) / (16 * PG * (kThreads / 64));
    // Rows are shared out where the pages alone leave CUs idle.
    const int each = 16 / a.pad;
    const int64_t tiles = (int64_t{most} + each - 1) / each, groups = chunks * a.bounds.H;
    // (Of all sequences there are about as many tiles as of their tokens in one.)
    const int64_t all = std::min(tiles * num_seqs, (int64_t{a.batch.num_queries} + each - 1) / each + num_seqs);
    const int64_t share = std::max<int64_t>(all * groups / kShareTarget, 1);
    a.tokens = static_cast<int32_t>(std::min((share + 1) / 2 * 2, tiles) * each);
    a.shares = static_cast<int32_t>((int64_t{most} + a.tokens - 1) / a.tokens);
    a.by_shares = divisor(a.shares);
    const int64_t grid = chunks * ((int64_t{most} + a.tokens - 1) / a.tokens) * a.bounds.H;
    return launch_score_to<T, FP8, DP, PG>(a, dim3(static_cast<uint32_t>(grid), static_cast<uint32_t>(num_seqs)), stream);
}

template <class T, bool FP8>
hipError_t launch_score(const ScoreArgs &a, int num_seqs, int most, int64_t pages, hipStream_t stream) {
    // (Wide 2-byte bounds of 32 pages would not leave registers for the queries.)
    if (a.bounds.D > 128)
        return launch_score<T, FP8, 256, FP8 ? 2 : 1>(a, num_seqs, most, pages, stream);
    if (a.bounds.D > 64)
        return launch_score<T, FP8, 128, 2>(a, num_seqs, most, pages, stream);
    return launch_score<T, FP8, 64, 2>(a, num_seqs, most, pages, stream);
}

kv_status score(const kv_cache *bounds, int32_t layer, const kv_batch *batch, const kv_score_options *o,
                const kv_rows *q, float *scores, int32_t *counts, hipStream_t stream) {
    kv_status st = check_layer(bounds, layer);
    if (st == KV_OK)
        st = check_bounds(bounds);
    if (st != KV_OK)
        return st;
    if (!o)
        return fail(KV_EINVAL, "options must not be NULL");
    st = check_dtype(bounds, o->cache_dtype);
    if (st != KV_OK)
        return st;
    if (o->block_size < 1)
        return fail(KV_EINVAL, "block_size must be positive (got %d)", o->block_size);
    kv_cache pages = *bounds;  // the batch counts in tokens of the cache
    pages.layout.block_size = o->block_size;
    st = check_batch(&pages, batch);
    if (st == KV_OK)
        st = check_rows(bounds, batch, q, "q");
    if (st == KV_OK && o->scales)
        st = check_scales(bounds, o->cache_dtype, o->scales);
    if (st != KV_OK)
        return st;
    const int H = bounds->layout.num_kv_heads;
    if (q->heads % H != 0)
        return fail(KV_EINVAL, "%d query heads for %d KV heads", q->heads, H);
    if (q->heads > 16383)
        return fail(KV_EUNSUPPORTED, "%d query heads (at most 16,383)", q->heads);
    if (o->cache_dtype != KV_DTYPE_E4M3 && q->dtype != o->cache_dtype)
        return fail(KV_EINVAL, "rows of type %d for bounds of type %d", q->dtype, o->cache_dtype);
    if (!(o->scale >= 0.f && std::isfinite(o->scale)))
        return fail(KV_EINVAL, "scale must be finite and not negative (got %g)", o->scale);
    if (o->reserved != 0)
        return fail(KV_EINVAL, "kv_score_options.reserved must be 0");
    const int most = std::min(batch->max_queries, batch->num_queries);
    if (batch->num_seqs == 0 || most == 0)
        return KV_OK;
    const int64_t most_pages = (int64_t{batch->max_len} + o->block_size - 1) / o->block_size;
    if (o->token_stride < 0 || o->head_stride < 0 || (H > 1 && o->head_stride < most_pages) ||
        (batch->num_queries > 1 && o->token_stride < most_pages))
        return fail(KV_EINVAL, "rows of scores (strides %lld and %lld) are shorter than %lld pages",
                    static_cast<long long>(o->token_stride), static_cast<long long>(o->head_stride),
                    static_cast<long long>(most_pages));
    if (!scores && most_pages > 0)
        return fail(KV_EINVAL, "scores must not be NULL");
    // (Shares add at most kShareTarget workgroups and as many again.)
    if ((most_pages + 63) / 64 * H > int64_t{1} << 21)
        return fail(KV_EUNSUPPORTED, "%lld pages of %d heads of a sequence in one call are too many",
                    static_cast<long long>(most_pages), H);
    st = check_on_current_device(bounds);
    int32_t *err = nullptr;
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    ScoreArgs a{};
    a.bounds = pages_of(bounds, layer, err);
    a.batch = batch_of(batch);
    a.q = rows_of(q);
    a.scales = scales_of(o->scales);
    a.scores = scores;
    a.counts = counts;
    a.token_stride = o->token_stride;
    a.head_stride = o->head_stride;
    a.scale = o->scale == 0.f ? 1.f : o->scale;
    a.by_bs = divisor(o->block_size);
    a.BS = o->block_size;
    a.group = q->heads / H;
    while ((1 << a.shift) < a.group && a.shift < 4)
        ++a.shift;
    a.pad = 1 << a.shift;
    a.by_subs = divisor((a.group + 15) / 16);
    const bool fp8 = o->cache_dtype == KV_DTYPE_E4M3;
    const int64_t some = std::max<int64_t>(most_pages, 1);  // (counts are written where no sequence has a token)
    if (q->dtype == KV_DTYPE_BF16)
        KVX_HIP((fp8 ? launch_score<Bf16, true>(a, batch->num_seqs, most, some, stream)
                     : launch_score<Bf16, false>(a, batch->num_seqs, most, some, stream)));
    else
        KVX_HIP((fp8 ? launch_score<F16, true>(a, batch->num_seqs, most, some, stream)
                     : launch_score<F16, false>(a, batch->num_seqs, most, some, stream)));
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" {

kv_status kv_bounds(const kv_cache *cache, int32_t layer, const kv_batch *batch, int32_t cache_dtype,
                    const kv_cache *bounds, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::bounds_of(cache, layer, batch, cache_dtype, bounds, static_cast<hipStream_t>(stream));
    });
}

kv_status kv_score(const kv_cache *bounds, int32_t layer, const kv_batch *batch, const kv_score_options *options,
                   const kv_rows *q, float *scores, int32_t *counts, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::score(bounds, layer, batch, options, q, scores, counts, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
