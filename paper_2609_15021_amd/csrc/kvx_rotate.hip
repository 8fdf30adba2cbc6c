// kv_rotate: the new tokens' queries and keys normed for each head and rotated by their position, in one pass; keys and
// values go straight into the cache's pages.
//
// Everything is read once and written once.  A lane has 8 columns of a row, so a row's norm is a few lane shuffles, and
// so are the partners that lie half a row away.  A workgroup has a few tokens of a sequence, whose rows (query heads,
// then heads of K, then of V) its groups of lanes take kAtOnce at a time, the next ones on their way.  Angles are the
// same for all heads: the workgroup works out its tokens' cosines and sines once, in LDS, and looks their pages up,
// while the first rows are on their way.
//
// 2,085 tokens of 40 query heads and 8 KV heads (bf16, D 128, norms; 60 MB, 12.7 us at a large copy's rate): 17 us,
// and 18 into e4m3 pages.  A third of it is the launch and a workgroup's start, whatever the size; then the vector units
// are busy for about half of the time.  Rows are stored past the caches (1.5 us more without).  A decoding step takes
// 4.6 us on the GPU, 8.2 with the host.
#include <algorithm>
#include <cmath>

#include "kvx_rows.h"

namespace kvx {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAtOnce = 2;
constexpr int kAngles = 1024;       // of a workgroup
constexpr int kPlaces = 32;         // tokens of a workgroup at most
constexpr int kShareTarget = 1280;  // workgroups that run at once, 5 a CU

// by * 2^exponent, by in [1, 2), and 1 / by
struct Divided {
    float by, inverse;
    int32_t exponent;
};

Divided divided(float scale) {
    int exponent = 0;
    const float by = 2.f * std::frexp(scale, &exponent);
    return Divided{by, 1.f / by, exponent - 1};
}

struct RotateArgs {
    Pages pages;
    Batch batch;
    Rows q, out, k, v;
    Turn turn[2];              // of q, k
    int32_t heads, rows_each;  // query heads; rows of a token
    int32_t tokens;            // of a workgroup
    int32_t splits;            // workgroups that share their rows
    Divisor by_splits, by_half, by_rows;
    Divided k_scale, v_scale;
};

// x / (by * 2^exponent), by in [1, 2), from by's inverse: off by hardly more than half a unit of the last place where it
// is within e4m3's range.  (A division takes three times the instructions: 2,085 tokens into e4m3 pages took 24 us.)
__device__ __forceinline__ float quotient(float x, const Divided &d) {
    x = ldexpf(x, -d.exponent);
    const float q = x * d.inverse;
    return fabsf(q) < 0x1p20f ? copysignf(fmaf(fmaf(-q, d.by, x), d.inverse, q), x) : q;  // (-0 stays)
}

// QUANT: the cache holds e4m3.  (kAnyHalves has twice the operands, and no registers for more than 3 waves a SIMD.)
template <int DTYPE, int LPR, Pairs PAIRS, bool QUANT>
__global__ __launch_bounds__(kThreads, PAIRS == kAnyHalves ? 3 : 5) void rotate_kernel(const RotateArgs a) {
    constexpr int kGroups = kThreads / LPR;                           // of lanes: rows at once
    __shared__ __align__(16) float cosines[kAngles], sines[kAngles];  // [token][pair], in the order of angle_at
    __shared__ __align__(16) float weights[2][LPR * 8];  // of q's and K's norms, in the order of weight_at
    __shared__ int64_t places[kPlaces];                  // of the tokens' slots in the cache, or -1
    const Pages &p = a.pages;
    const int b = blockIdx.y, tid = threadIdx.x;
    Sequence s;
    if (!sequence(a.batch, b, p.err, s))
        return;
    const int tile = divide(blockIdx.x, a.by_splits), split = blockIdx.x - tile * a.splits;
    const int i0 = tile * a.tokens, tokens = min(a.tokens, s.nq - i0);
    if (tokens <= 0)
        return;
    typedef Turner<DTYPE, PAIRS, LPR> Lane;
    const Lane lane(a.turn[0], tid % LPR, p.D);
    // A lane's 8 numbers lie in two pieces of 16 bytes, beside the other lanes' first and second pieces, so that a
    // wave's reads meet no bank of LDS twice.
    const int half = a.turn[0].half;
    const auto weight_at = [](int d) { return (d & 4) * LPR + (d >> 3) * 4 + (d & 3); };
    const auto angle_at = [half](int i) {
        return PAIRS == kHalves ? (i >> 2 & 1) * (half / 2) + (i >> 3) * 4 + (i & 3) : i;
    };
    const auto pieces = [](const float *x, int apart, float *y) {
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
            const f32x4 piece = *reinterpret_cast<const f32x4 *>(x + (j >> 2) * apart);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y[j + i] = piece[i];
        }
    };

    // The tile's rows are numbered, a token's one after the other; a group takes number u, u + step, ...
    const int rows = tokens * a.rows_each, step = kGroups * a.splits;
    struct Vecs {
        typename Lane::Vec of[kAtOnce];
        int token[kAtOnce], r[kAtOnce];  // of the tile; row of the token: of q, of K or of V
    };
    const auto load = [&](int u) {
        Vecs v;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int x = min(u + k * step, rows - 1);
            const int t = divide(x, a.by_rows), r = x - t * a.rows_each;
            const int of_k = r - a.heads, of_v = of_k - p.H;
            const Rows &src = of_k < 0 ? a.q : of_v < 0 ? a.k : a.v;
            const int64_t head = of_k < 0 ? r : of_v < 0 ? of_k : of_v;
            v.of[k] = lane.load(a.turn[0], src.data + int64_t{s.q0 + i0 + t} * src.token_stride + head * src.head_stride);
            v.token[k] = t;
            v.r[k] = r;
        }
        return v;
    };
    int u0 = split * kGroups + tid / LPR;
    Vecs next = load(u0);
    for (int u = tid; u < 2 * LPR * 8; u += kThreads) {
        const Turn &turn = u < LPR * 8 ? a.turn[0] : a.turn[1];
        const int d = u & (LPR * 8 - 1);
        weights[u / (LPR * 8)][weight_at(d)] = turn.weight && d < p.D ? norm_weight<DTYPE>(turn, d) : 1.f;
    }
    const int first = s.n - s.nq + i0;
    for (int u = tid; u < tokens * half; u += kThreads) {
        const int t = divide(u, a.by_half), i = u - t * half;
        const int position = a.turn[0].positions ? a.turn[0].positions[s.q0 + i0 + t] : first + t;
        const int at = t * half + angle_at(i);
        turn_by(position, a.turn[0].freqs[i], a.turn[0].magnitude, cosines[at], sines[at]);
    }
    if (tid < tokens && a.rows_each > a.heads) {
        const int t = first + tid, page = divide(max(t, 0), p.by_bs);
        int64_t place = -1;
        if (t >= 0) {
            const int block = a.batch.tables[b * a.batch.table_stride + page];
            if (in_cache(p, block))
                place = block * p.block_stride + static_cast<uint32_t>(t - page * p.BS) * p.token_bytes;
        }
        places[tid] = place;
    }
    __syncthreads();
    for (; u0 < rows; u0 += kAtOnce * step) {
        const Vecs now = next;
        if (u0 + kAtOnce * step < rows)
            next = load(u0 + kAtOnce * step);
        // (V's rows are worked out with the others, without a use, so that no row's work waits for another's.)
        float y[kAtOnce][8];
        typename Lane::Weights w;
        typename Lane::Angles angles;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const bool is_q = now.r[k] < a.heads;
            const float *of = weights[is_q ? 0 : 1];
            if (k == 0 || is_q != (now.r[k ? k - 1 : 0] < a.heads)) {
                if constexpr (PAIRS == kAnyHalves)
                    w = lane.weights(a.turn[0], [&](int d) { return of[weight_at(d)]; });
                else
                    pieces(of + tid % LPR * 4, 4 * LPR, w.own);
            }
            if (k == 0 || now.token[k] != now.token[k ? k - 1 : 0]) {
                const int angle0 = now.token[k] * half;
                if constexpr (PAIRS == kHalves) {
                    const int from = angle0 + (lane.turned ? angle_at(lane.pair(a.turn[0], 0)) : 0);
                    pieces(cosines + from, half / 2, angles.cosine);
                    pieces(sines + from, half / 2, angles.sine);
                    lane.settle(a.turn[0], angles);
                } else {
                    angles = lane.angles(a.turn[0], [&](int i, float &c, float &si) {
                        c = cosines[angle0 + i];
                        si = sines[angle0 + i];
                    });
                }
            }
            lane.finish(a.turn[0], now.of[k], (is_q ? a.turn[0].weight : a.turn[1].weight) != nullptr, w, angles, y[k]);
        }
        if (!lane.any)
            continue;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = now.r[k], of_k = r - a.heads, of_v = of_k - p.H;
            if (u0 + k * step >= rows)
                break;
            if (of_k < 0) {
                uint8_t *to = a.out.data + int64_t{s.q0 + i0 + now.token[k]} * a.out.token_stride +
                              r * a.out.head_stride;
                __builtin_nontemporal_store(from_floats<DTYPE>(y[k]), reinterpret_cast<vec16 *>(to + 2 * lane.d0));
                continue;
            }
            const int64_t place = places[now.token[k]];
            if (place < 0)
                continue;
            uint8_t *to = p.base + place + (of_v < 0 ? 0u : p.v_bytes) +
                          static_cast<uint32_t>(of_v < 0 ? of_k : of_v) * p.head_bytes;
            if constexpr (QUANT) {
                if (of_v >= 0)
                    to_floats<DTYPE>(now.of[k].own, y[k]);
                const Divided scale{of_v < 0 ? a.k_scale.by : a.v_scale.by,
                                    of_v < 0 ? a.k_scale.inverse : a.v_scale.inverse,
                                    of_v < 0 ? a.k_scale.exponent : a.v_scale.exponent};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[k][j] = quotient(y[k][j], scale);
                *reinterpret_cast<vec8 *>(to + lane.d0) = to_e4m3(y[k]);
            } else {
                // (V's bytes as they are.)
                __builtin_nontemporal_store(of_v < 0 ? from_floats<DTYPE>(y[k]) : now.of[k].own,
                                            reinterpret_cast<vec16 *>(to + 2 * lane.d0));
            }
        }
    }
}

template <int DTYPE, int LPR, bool QUANT>
hipError_t launch(const RotateArgs &a, const dim3 &grid, Pairs pairs, hipStream_t stream) {
    const auto kernel = pairs == kNeighbours ? rotate_kernel<DTYPE, LPR, kNeighbours, QUANT>
                        : pairs == kHalves   ? rotate_kernel<DTYPE, LPR, kHalves, QUANT>
                                             : rotate_kernel<DTYPE, LPR, kAnyHalves, QUANT>;
    return launch_kernel(kernel, grid, kThreads, stream, a);
}

template <int DTYPE, bool QUANT>
hipError_t launch(const RotateArgs &a, const dim3 &grid, Pairs pairs, hipStream_t stream) {
    const int lanes = lanes_of(a.pages.D);
    return lanes == 32   ? launch<DTYPE, 32, QUANT>(a, grid, pairs, stream)
           : lanes == 16 ? launch<DTYPE, 16, QUANT>(a, grid, pairs, stream)
                         : launch<DTYPE, 8, QUANT>(a, grid, pairs, stream);
}

kv_status check_rotate(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rotate_options *o,
                       const kv_rows *q, const kv_rows *out, const kv_rows *k, const kv_rows *v) {
    if (!o)
        return fail(KV_EINVAL, "options must not be NULL");
    kv_status st = check_append(cache, layer, batch, k, v, o->cache_dtype);
    if (st == KV_OK)
        st = check_rows(cache, batch, q, "q");
    if (st == KV_OK)
        st = check_rows(cache, batch, out, "out");
    if (st == KV_OK)
        st = check_factors(o->cache_dtype, o->k_scale, o->v_scale);
    if (st == KV_OK && o->scales)
        st = check_scales(cache, o->cache_dtype, o->scales);
    if (st == KV_OK && o->scales)
        st = check_append_scaled(cache, batch);
    if (st != KV_OK)
        return st;
    if (o->scales && ((o->k_scale != 0.f && o->k_scale != 1.f) || (o->v_scale != 0.f && o->v_scale != 1.f)))
        return fail(KV_EINVAL, "k_scale and v_scale (%g and %g) beside scales of pages", o->k_scale, o->v_scale);
    const int D = cache->layout.head_dim;
    if (q->dtype != k->dtype || out->dtype != q->dtype || out->heads != q->heads)
        return fail(KV_EINVAL, "q has %d heads of type %d, out %d of type %d, k rows of type %d", q->heads, q->dtype,
                    out->heads, out->dtype, k->dtype);
    if (q->heads > 16383 || cache->layout.num_kv_heads > 16383)
        return fail(KV_EUNSUPPORTED, "%d query heads and %d KV heads (at most 16,383)", q->heads,
                    cache->layout.num_kv_heads);
    if (batch->num_seqs > 0 && ((batch->num_queries > 1 && out->token_stride < D) ||
                                (batch->num_queries > 0 && out->heads > 1 && out->head_stride < D)))
        return fail(KV_EINVAL, "rows of out (strides %lld and %lld) are shorter than %d elements",
                    static_cast<long long>(out->token_stride), static_cast<long long>(out->head_stride), D);
    if (o->rotary_dim < 0 || o->rotary_dim > D || o->rotary_dim % 2 != 0)
        return fail(KV_EINVAL, "rotary_dim must be even and from 0 to %d (got %d)", D, o->rotary_dim);
    if (o->interleaved != 0 && o->interleaved != 1)
        return fail(KV_EINVAL, "interleaved must be 0 or 1 (got %d)", o->interleaved);
    if (o->reserved != 0)
        return fail(KV_EINVAL, "kv_rotate_options.reserved must be 0");
    if (o->rotary_dim > 0 && !o->freqs)
        return fail(KV_EINVAL, "freqs must not be NULL");
    if ((o->q_weight || o->k_weight) && o->weight_dtype != KV_DTYPE_F32 && o->weight_dtype != q->dtype)
        return fail(KV_EINVAL, "weights of type %d for rows of type %d", o->weight_dtype, q->dtype);
    if (!(o->eps >= 0.f && std::isfinite(o->eps)) || !std::isfinite(o->weight_offset) ||
        !(o->magnitude >= 0.f && std::isfinite(o->magnitude)))
        return fail(KV_EINVAL, "eps, weight_offset and magnitude must be finite, eps and magnitude not negative (got %g, "
                    "%g, %g)", o->eps, o->weight_offset, o->magnitude);
    return KV_OK;
}

kv_status rotate(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rotate_options *o,
                 const kv_rows *q, const kv_rows *out, const kv_rows *k, const kv_rows *v, hipStream_t stream) {
    kv_status st = check_rotate(cache, layer, batch, o, q, out, k, v);
    if (st != KV_OK || batch->num_seqs == 0 || batch->num_queries == 0)
        return st;
    st = check_on_current_device(cache);
    int32_t *err = nullptr;
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    RotateArgs a{};
    a.pages = pages_of(cache, layer, err);
    a.batch = batch_of(batch);
    a.q = rows_of(q);
    a.out = rows_of(out);
    a.k = rows_of(k);
    a.v = rows_of(v);
    Turn &t = a.turn[0];
    t.freqs = o->freqs;
    t.positions = o->positions;
    t.weight = o->q_weight;
    t.weight_f32 = o->weight_dtype == KV_DTYPE_F32;
    t.eps = o->eps;
    t.offset = o->weight_offset;
    t.magnitude = o->magnitude == 0.f ? 1.f : o->magnitude;
    t.mean = 1.f / static_cast<float>(cache->layout.head_dim);
    t.rotary = o->rotary_dim;
    t.half = o->rotary_dim / 2;
    a.turn[1] = t;
    a.turn[1].weight = o->k_weight;
    a.heads = q->heads;
    a.rows_each = q->heads + (o->scales ? 0 : 2 * a.pages.H);
    a.k_scale = divided(o->k_scale == 0.f ? 1.f : o->k_scale);
    a.v_scale = divided(o->v_scale == 0.f ? 1.f : o->v_scale);
    const Pairs pairs = o->interleaved ? kNeighbours : t.half % 8 == 0 ? kHalves : kAnyHalves;
    // A workgroup has as many tokens as its groups have kAtOnce rows of each, or more of them one after the other where
    // all workgroups would not run at once: what a workgroup does before its first row is then done once for them.  A
    // token whose rows are more is shared by workgroups, a row a group, while that leaves CUs idle.
    const int64_t most = std::min(batch->max_queries, batch->num_queries), groups_each = kThreads / lanes_of(a.pages.D);
    const int64_t side = std::max<int64_t>(kAtOnce * groups_each / a.rows_each, 1);
    a.splits = static_cast<int32_t>(std::max<int64_t>(
        std::min((a.rows_each + groups_each - 1) / groups_each, 1024 / std::max<int64_t>(batch->num_queries, 1)), 1));
    const int64_t wanted = std::max(std::min<int64_t>(side, batch->num_queries / 256),
                                    (int64_t{batch->num_queries} + kShareTarget - 1) / kShareTarget);
    const int64_t held = std::min<int64_t>(kAngles / std::max(t.half, 1), kPlaces);
    a.tokens = static_cast<int32_t>(std::max<int64_t>(std::min(wanted, held), 1));
    const int64_t groups = ((most - 1) / a.tokens + 1) * a.splits;
    if (groups > INT32_MAX / kThreads)
        return fail(KV_EUNSUPPORTED, "%lld new tokens of a sequence in one call are too many",
                    static_cast<long long>(most));
    a.by_splits = divisor(a.splits);
    a.by_half = divisor(std::max(t.half, 1));
    a.by_rows = divisor(a.rows_each);
    const dim3 grid(static_cast<uint32_t>(groups), static_cast<uint32_t>(batch->num_seqs));
    const bool quantised = o->cache_dtype == KV_DTYPE_E4M3;
    if (q->dtype == KV_DTYPE_BF16)
        KVX_HIP((quantised ? launch<KV_DTYPE_BF16, true>(a, grid, pairs, stream)
                           : launch<KV_DTYPE_BF16, false>(a, grid, pairs, stream)));
    else
        KVX_HIP((quantised ? launch<KV_DTYPE_F16, true>(a, grid, pairs, stream)
                           : launch<KV_DTYPE_F16, false>(a, grid, pairs, stream)));
    if (!o->scales)
        return KV_OK;
    KVX_HIP(launch_append_scaled(a.pages, a.batch, batch->num_seqs, a.k, a.v, k->dtype, scales_of(o->scales), a.turn[1],
                                 pairs, stream));
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" kv_status kv_rotate(const kv_cache *cache, int32_t layer, const kv_batch *batch,
                               const kv_rotate_options *options, const kv_rows *q, const kv_rows *out, const kv_rows *k,
                               const kv_rows *v, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::rotate(cache, layer, batch, options, q, out, k, v, static_cast<hipStream_t>(stream));
    });
}
