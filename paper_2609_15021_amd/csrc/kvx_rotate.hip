// kv_rotate: the new tokens' queries and keys normed for each head and rotated by their position, in one pass; keys and
// values go straight into the cache's pages.
//
// Everything is read once and written once.  A workgroup takes a few tokens of a sequence and goes over their rows (query
// heads, then the heads of K, then of V), 8 columns a lane, so that a row's norm is a few lane shuffles.  The angles are
// the same for all heads: the workgroup works out its tokens' cosines and sines once, in LDS, while its first rows are on
// their way, and looks their pages up.  Where a column's partner is half a row away the lane loads the partners too
// (they come from the cache of the CU).
#include <algorithm>
#include <cmath>

#include "kvx_rows.h"

namespace kvx {

namespace {

constexpr int kTokens = 4;  // most tokens of a workgroup

struct RotateArgs {
    Pages pages;
    Batch batch;
    Rows q, out, k, v;
    Turn turn[2];  // of q, k
    int32_t heads, rows_each;  // query heads; rows of a token
    int32_t tokens, splits;    // tokens of a workgroup, and workgroups that share their rows
    Divisor by_rows, by_splits, by_half;
    float k_scale, v_scale;
};

// QUANT: the cache holds e4m3.
template <int DTYPE, int LPR, Pairs PAIRS, bool QUANT>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
    constexpr int kSlots = kThreads / LPR;  // rows at once
    __shared__ float cosines[kTokens][128], sines[kTokens][128];
    __shared__ int64_t places[kTokens];     // of the tokens' slots in the cache, or -1
    const Pages &p = a.pages;
    const int b = blockIdx.y, tid = threadIdx.x;
    Sequence s;
    if (!sequence(a.batch, b, p.err, s))
        return;
    const int tile = divide(blockIdx.x, a.by_splits), split = blockIdx.x - tile * a.splits;
    const int i0 = tile * a.tokens, tokens = min(a.tokens, s.nq - i0);
    if (tokens <= 0)
        return;
    const int rows = tokens * a.rows_each, step = a.splits * kSlots;
    typedef Turner<DTYPE, PAIRS, LPR> Lane;
    const Lane lane(a.turn[0], tid % LPR, p.D);

    struct Where {
        int token, head;  // head: of q, then of K, then of V
        const uint8_t *from;
    };
    const auto where = [&](int r) {
        Where w;
        w.token = divide(r, a.by_rows);
        w.head = r - w.token * a.rows_each;
        const int of_k = w.head - a.heads, of_v = of_k - p.H;
        const Rows &src = of_k < 0 ? a.q : of_v < 0 ? a.k : a.v;
        w.from = src.data + int64_t{s.q0 + i0 + w.token} * src.token_stride +
                 int64_t{of_k < 0 ? w.head : of_v < 0 ? of_k : of_v} * src.head_stride;
        return w;
    };
    // (Rows beyond the last are loaded as the last: all lanes of a row stay together, and a wave's lanes mostly do.)
    int r = split * kSlots + tid / LPR;
    Where next = where(min(r, rows - 1));
    typename Lane::Vec next_vec = lane.load(a.turn[0], next.from);
    const typename Lane::Weights q_weights = lane.weights(a.turn[0]), k_weights = lane.weights(a.turn[1]);
    const int first = s.n - s.nq + i0;
    for (int u = tid; u < tokens * a.turn[0].half; u += kThreads) {
        const int token = divide(u, a.by_half), i = u - token * a.turn[0].half;
        const int position = a.turn[0].positions ? a.turn[0].positions[s.q0 + i0 + token] : first + token;
        turn_by(position, a.turn[0].freqs[i], a.turn[0].magnitude, cosines[token][i], sines[token][i]);
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
    for (; r < rows; r += step) {
        const Where at = next;
        const typename Lane::Vec vec = next_vec;
        if (r + step < rows) {
            next = where(r + step);
            next_vec = lane.load(a.turn[0], next.from);
        }
        const int of_k = at.head - a.heads, of_v = of_k - p.H;
        float y[8];
        if (of_v < 0) {
            // (q's and K's norms differ by their weights alone, which may be missing for one of them.)
            const bool is_q = of_k < 0;
            Turn turn = a.turn[0];
            turn.weight = is_q ? a.turn[0].weight : a.turn[1].weight;
            typename Lane::Weights w;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w.own[j] = is_q ? q_weights.own[j] : k_weights.own[j];
                w.other[j] = is_q ? q_weights.other[j] : k_weights.other[j];
            }
            lane.finish(turn, vec, w,
                        [&](int j, float &c, float &si) {
                            const int i = lane.pair(turn, j);
                            c = cosines[at.token][i];
                            si = sines[at.token][i];
                        },
                        y);
        } else {
            to_floats<DTYPE>(vec.own, y);
        }
        if (!lane.any)
            continue;
        if (of_k < 0) {
            uint8_t *to = a.out.data + int64_t{s.q0 + i0 + at.token} * a.out.token_stride + at.head * a.out.head_stride;
            *reinterpret_cast<vec16 *>(to + 2 * lane.d0) = from_floats<DTYPE>(y);
            continue;
        }
        if (places[at.token] < 0)
            continue;
        uint8_t *to = p.base + places[at.token] + (of_v < 0 ? 0u : p.v_bytes) +
                      static_cast<uint32_t>(of_v < 0 ? of_k : of_v) * p.head_bytes;
        if constexpr (QUANT) {
            const float scale = of_v < 0 ? a.k_scale : a.v_scale;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                y[j] /= scale;
            *reinterpret_cast<vec8 *>(to + lane.d0) = to_e4m3(y);
        } else {
            // (V's bytes as they are.)
            *reinterpret_cast<vec16 *>(to + 2 * lane.d0) = of_v < 0 ? from_floats<DTYPE>(y) : vec.own;
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
        return fail(KV_EINVAL, "eps, weight_offset and magnitude must be finite, eps and magnitude not negative (got %g, %g, "
                    "%g)", o->eps, o->weight_offset, o->magnitude);
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
    // A few tokens share a workgroup; while that leaves CUs idle a token has its own, and while that does, several.
    const int64_t slots = kThreads / lanes_of(a.pages.D), most = std::min(batch->max_queries, batch->num_queries);
    const int64_t each = (a.rows_each + slots - 1) / slots;
    a.tokens = int64_t{batch->num_queries} > 1024 ? kTokens : 1;
    a.splits = static_cast<int32_t>(int64_t{batch->num_queries} * each > 4096 ? 1 : each);
    const int64_t groups = (most + a.tokens - 1) / a.tokens * a.splits;
    if (groups > INT32_MAX / kThreads)
        return fail(KV_EUNSUPPORTED, "%lld new tokens of a sequence in one call are too many",
                    static_cast<long long>(most));
    a.by_rows = divisor(a.rows_each);
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
    return launch_append_scaled(a.pages, a.batch, batch->num_seqs, a.k, a.v, k->dtype, scales_of(o->scales), a.turn[1],
                                pairs, stream);
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
