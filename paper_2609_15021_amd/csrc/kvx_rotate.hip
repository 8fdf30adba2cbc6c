// kv_rotate: the new tokens' queries and keys normed for each head and rotated by their position, in one pass; keys and
// values go straight into the cache's pages.
//
// Everything is read once and written once.  A lane has 8 columns of a row, so a row's norm is a few lane shuffles, and
// so are the partners that lie half a row away.  A group of lanes takes kAtOnce rows (query heads, then heads of K,
// then of V) of one token, all of them on their way at once; as many groups as a token needs share it, and a workgroup
// has as many tokens as that leaves room for.  Angles are the same for all heads: the workgroup works out its tokens'
// cosines and sines once, in LDS, and looks their pages up, while the rows are on their way.
//
// 2,085 tokens of 40 query heads and 8 KV heads (bf16, D 128, norms; 60 MB, 12.7 us at a large copy's rate): 18.8 us.
// About 6 of them are the launch and a workgroup's start, whatever the size; then rows pass at 4.3 TB/s, with the vector
// units busy for about half of the time.  Rows are stored past the caches (20.3 us without).  A decoding step takes 4.6
// us on the GPU, 8.2 with the host.
#include <algorithm>
#include <cmath>

#include "kvx_rows.h"

namespace kvx {

namespace {

constexpr int kAtOnce = 2;
constexpr int kAngles = 1024;  // of a workgroup

struct RotateArgs {
    Pages pages;
    Batch batch;
    Rows q, out, k, v;
    Turn turn[2];              // of q, k
    int32_t heads, rows_each;  // query heads; rows of a token
    int32_t each_shift;        // 2^each_shift groups of lanes share a token
    int32_t tokens;            // of a workgroup
    int32_t splits;            // workgroups that share their rows
    Divisor by_splits, by_half;
    float k_scale, v_scale;
};

// QUANT: the cache holds e4m3.
template <int DTYPE, int LPR, Pairs PAIRS, bool QUANT>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
    constexpr int kGroups = kThreads / LPR;         // of lanes: rows at once
    __shared__ float cosines[kAngles], sines[kAngles];  // [token][pair]
    __shared__ __align__(16) float weights[2][LPR * 8];  // of q's and K's norms
    __shared__ int64_t places[kGroups];             // of the tokens' slots in the cache, or -1
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
    const int each = 1 << a.each_shift, token_step = kGroups >> a.each_shift;
    const int step = each * a.splits, r0 = split * each + (tid / LPR & (each - 1));

    // What a group has at once: rows r, r + step, ... of a token (of the workgroup's).  A group without any goes along
    // with the last token's last row: lanes of a wave stay together.
    struct At {
        int token, r;
    };
    const auto after = [&](At at) {
        at.r += kAtOnce * step;
        return at.r < a.rows_each ? at : At{at.token + token_step, r0};
    };
    // Row r of the token: of q, of K or of V.
    const auto from = [&](int row, int r) {
        const int of_k = r - a.heads, of_v = of_k - p.H;
        const Rows &src = of_k < 0 ? a.q : of_v < 0 ? a.k : a.v;
        const int64_t head = of_k < 0 ? r : of_v < 0 ? of_k : of_v;
        return src.data + int64_t{row} * src.token_stride + head * src.head_stride;
    };
    struct Vecs {
        typename Lane::Vec of[kAtOnce];
    };
    const auto load = [&](const At &at) {
        Vecs v;
        const int row = s.q0 + i0 + min(at.token, tokens - 1);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            v.of[k] = lane.load(a.turn[0], from(row, min(at.r + k * step, a.rows_each - 1)));
        return v;
    };
    At at{tid / LPR >> a.each_shift, r0};
    Vecs next = load(at);
    for (int u = tid; u < 2 * LPR * 8; u += kThreads) {
        const Turn &turn = u < LPR * 8 ? a.turn[0] : a.turn[1];
        const int d = u & (LPR * 8 - 1);
        weights[u / (LPR * 8)][d] = turn.weight && d < p.D ? norm_weight<DTYPE>(turn, d) : 1.f;
    }
    const int first = s.n - s.nq + i0, half = a.turn[0].half;
    for (int u = tid; u < tokens * half; u += kThreads) {
        const int t = divide(u, a.by_half), i = u - t * half;
        const int position = a.turn[0].positions ? a.turn[0].positions[s.q0 + i0 + t] : first + t;
        turn_by(position, a.turn[0].freqs[i], a.turn[0].magnitude, cosines[u], sines[u]);
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
    while (at.token < tokens) {
        const Vecs vecs = next;
        const At now = at;
        at = after(at);
        if (at.token < tokens)
            next = load(at);
        const int row = s.q0 + i0 + now.token;
        const typename Lane::Angles angles = lane.angles(a.turn[0], [&](int i, float &c, float &si) {
            c = cosines[now.token * half + i];
            si = sines[now.token * half + i];
        });
        // (V's rows are worked out with the others, without a use, so that no row's work waits for another's.)
        float y[kAtOnce][8];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const bool is_q = now.r + k * step < a.heads;
            const float *of = weights[is_q ? 0 : 1];
            lane.finish(a.turn[0], vecs.of[k], (is_q ? a.turn[0].weight : a.turn[1].weight) != nullptr,
                        lane.weights(a.turn[0], [&](int d) { return of[d]; }), angles, y[k]);
        }
        if (!lane.any)
            continue;
        const int64_t place = places[now.token];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = now.r + k * step, of_k = r - a.heads, of_v = of_k - p.H;
            if (r >= a.rows_each)
                break;
            if (of_k < 0) {
                uint8_t *to = a.out.data + int64_t{row} * a.out.token_stride + r * a.out.head_stride;
                __builtin_nontemporal_store(from_floats<DTYPE>(y[k]), reinterpret_cast<vec16 *>(to + 2 * lane.d0));
                continue;
            }
            if (place < 0)
                continue;
            uint8_t *to = p.base + place + (of_v < 0 ? 0u : p.v_bytes) +
                          static_cast<uint32_t>(of_v < 0 ? of_k : of_v) * p.head_bytes;
            if constexpr (QUANT) {
                if (of_v >= 0)
                    to_floats<DTYPE>(vecs.of[k].own, y[k]);
                const float scale = of_v < 0 ? a.k_scale : a.v_scale;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[k][j] /= scale;
                *reinterpret_cast<vec8 *>(to + lane.d0) = to_e4m3(y[k]);
            } else {
                // (V's bytes as they are.)
                __builtin_nontemporal_store(of_v < 0 ? from_floats<DTYPE>(y[k]) : vecs.of[k].own,
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
    a.k_scale = o->k_scale == 0.f ? 1.f : o->k_scale;
    a.v_scale = o->v_scale == 0.f ? 1.f : o->v_scale;
    const Pairs pairs = o->interleaved ? kNeighbours : t.half % 8 == 0 ? kHalves : kAnyHalves;
    // A token has as many groups of lanes as have kAtOnce rows each (or a group for each row, while that leaves CUs
    // idle), and a workgroup as many tokens as its groups then have at once, or more of them one after the other where
    // all workgroups would not run at once: what a workgroup does before its first row is then done once for them.
    const int64_t most = std::min(batch->max_queries, batch->num_queries), groups_each = kThreads / lanes_of(a.pages.D);
    const int64_t wanted = int64_t{batch->num_queries} * a.rows_each > 16384 ? (a.rows_each + kAtOnce - 1) / kAtOnce
                                                                             : a.rows_each;
    while ((int64_t{1} << a.each_shift) < std::min(wanted, groups_each))
        ++a.each_shift;
    const int64_t side = groups_each >> a.each_shift;  // tokens side by side
    a.splits = static_cast<int32_t>(std::max<int64_t>(
        std::min((wanted + groups_each - 1) / groups_each, 1024 / std::max<int64_t>(batch->num_queries, 1)), 1));
    const int64_t behind = std::max<int64_t>(batch->num_queries / (side * 1024), 1);
    const int64_t held = std::min<int64_t>(kAngles / std::max(t.half, 1), groups_each);
    a.tokens = static_cast<int32_t>(std::max<int64_t>(std::min(side * behind, held), 1));
    const int64_t groups = ((most - 1) / a.tokens + 1) * a.splits;
    if (groups > INT32_MAX / kThreads)
        return fail(KV_EUNSUPPORTED, "%lld new tokens of a sequence in one call are too many",
                    static_cast<long long>(most));
    a.by_splits = divisor(a.splits);
    a.by_half = divisor(std::max(t.half, 1));
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
