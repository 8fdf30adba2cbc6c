// kv_attend: attention of the new tokens over a paged cache.
//
// For a row (a new token and a query head) with scores s_t over the tokens it sees, out = sum exp(s_t - m) v_t / sum
// exp(s_t - m) in one pass over the tokens: m is the largest score so far, and what was summed under a smaller one is
// scaled down when it grows.
#include <algorithm>
#include <cmath>

#include "kvx_attend_kernels.h"

namespace kvx {

namespace {

__device__ __forceinline__ float load_2(const uint8_t *p, int type) {
    const uint16_t bits = *reinterpret_cast<const uint16_t *>(p);
    return type == KV_DTYPE_BF16 ? __builtin_bit_cast(float, static_cast<uint32_t>(bits) << 16)
                                 : static_cast<float>(__builtin_bit_cast(_Float16, bits));
}

__device__ __forceinline__ float load_cached(const uint8_t *row, int d, int type) {
    if (type == KV_DTYPE_E4M3)
        return __builtin_amdgcn_cvt_f32_fp8(row[d], 0);
    return load_2(row + 2 * d, type);
}

__device__ __forceinline__ void store_2(uint8_t *p, float x, int type) {
    if (type == KV_DTYPE_BF16)
        *reinterpret_cast<__bf16 *>(p) = static_cast<__bf16>(x);
    else
        *reinterpret_cast<_Float16 *>(p) = static_cast<_Float16>(x);
}

__device__ __forceinline__ const uint8_t *cached_row(const AttendArgs &a, int b, int t, int kv, int h) {
    const int page = divide(t, a.pages.by_bs);
    const int block = a.batch.tables[b * a.batch.table_stride + page];
    if (!in_cache(a.pages, block))
        return nullptr;
    return a.pages.base + page_offset(a.pages, block, kv, h) +
           static_cast<uint32_t>(t - page * a.pages.BS) * a.pages.token_bytes;
}

// The score of a row at token p with query `q` for token t.
__device__ __forceinline__ float score(const AttendArgs &a, const float *q, const uint8_t *k, int p, int t, int head) {
    float x = 0.f;
    for (int d = 0; d < a.pages.D; ++d)
        x = fmaf(q[d], load_cached(k, d, a.cache_type), x);
    x *= a.scale;
    if (a.softcap > 0.f)
        x = a.softcap * tanhf(x / a.softcap);
    if (a.slopes)
        x -= a.slopes[head] * static_cast<float>(p - t);
    return x;
}

// One row and query head per workgroup: each wave takes 64 tokens at a time, one per lane for the scores and D / 64
// columns per lane for the sums; the waves' sums are joined at the end.
__global__ __launch_bounds__(256) void attend_kernel(const AttendArgs a) {
    __shared__ float q[256], sums[4][256], most[4], total[4];
    const int b = blockIdx.z, head = blockIdx.y, i = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sequence s;
    if (!sequence(a.batch, b, a.pages.err, s) || i >= s.nq || s.nq * a.group <= kStepRows)
        return;
    const int row = s.q0 + i, h = head / a.group, D = a.pages.D, p = s.n - s.nq + i;
    if (static_cast<int>(threadIdx.x) < D)
        q[threadIdx.x] = load_2(a.q.data + row * a.q.token_stride + head * a.q.head_stride + 2 * threadIdx.x, a.q_type);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    const int begin = a.window > 0 ? max(0, p + 1 - a.window) : 0;
    for (int t0 = begin + wave * 64; t0 <= p; t0 += 256) {
        const int t = t0 + lane;
        const uint8_t *k = t <= p ? cached_row(a, b, t, 0, h) : nullptr;
        const float x = k ? score(a, q, k, p, t, head) : -INFINITY;
        float top = x;
        for (int o = 32; o; o >>= 1)
            top = fmaxf(top, __shfl_xor(top, o));
        const float next = fmaxf(m, top);
        if (next == -INFINITY && !__any(x != x))
            continue;
        const float keep = m == -INFINITY ? 0.f : expf(m - next), e = k ? expf(x - next) : 0.f;
        m = next;
        l = l * keep + e;
        for (int c = 0; c < 4; ++c)
            acc[c] *= keep;
        for (int j = 0; j < 64; ++j) {
            const float w = __shfl(e, j);
            const uint8_t *v = t0 + j <= p ? cached_row(a, b, t0 + j, 1, h) : nullptr;
            if (v)
                for (int c = 0; c < 4; ++c)
                    if (c * 64 + lane < D)
                        acc[c] = fmaf(w, load_cached(v, c * 64 + lane, a.cache_type), acc[c]);
        }
    }
    for (int o = 32; o; o >>= 1)
        l += __shfl_xor(l, o);
    for (int c = 0; c < 4; ++c)
        sums[wave][c * 64 + lane] = acc[c];
    if (lane == 0) {
        most[wave] = m;
        total[wave] = l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    float x = 0.f, all = 0.f;
    for (int w = 0; w < 4; ++w) {
        const float f = most[w] == -INFINITY ? 0.f : expf(most[w] - top);
        x += f * sums[w][threadIdx.x];
        all += f * total[w];
    }
    if (static_cast<int>(threadIdx.x) < D)
        store_2(a.out.data + row * a.out.token_stride + head * a.out.head_stride + 2 * threadIdx.x,
                all == 0.f ? 0.f : x / all * a.v_scale, a.q_type);
    if (threadIdx.x == 0)
        a.lse[static_cast<int64_t>(row) * a.heads + head] = all == 0.f ? -INFINITY : top + logf(all);
}

// What each token received: one token per lane, over all rows that see it.
__global__ __launch_bounds__(64) void weigh_kernel(const AttendArgs a) {
    __shared__ float q[256];
    const int b = blockIdx.z, h = blockIdx.y, t = blockIdx.x * 64 + threadIdx.x;
    Sequence s;
    if (!sequence(a.batch, b, a.pages.err, s))
        return;
    const int begin = a.window > 0 ? s.n - s.nq + 1 - a.window : 0;  // the first token that a row sees
    const uint8_t *k = t < s.n && t >= begin && s.nq > 0 ? cached_row(a, b, t, 0, h) : nullptr;
    float sum = 0.f;
    for (int r = 0; r < s.nq * a.group; ++r) {
        const int i = r / a.group, head = h * a.group + r - i * a.group, row = s.q0 + i, p = s.n - s.nq + i;
        __syncthreads();
        for (int d = threadIdx.x; d < a.pages.D; d += 64)
            q[d] = load_2(a.q.data + row * a.q.token_stride + head * a.q.head_stride + 2 * d, a.q_type);
        __syncthreads();
        const float lse = a.lse[static_cast<int64_t>(row) * a.heads + head];
        if (k && t <= p && (a.window == 0 || p - t < a.window) && lse != -INFINITY)
            sum += expf(score(a, q, k, p, t, head) - lse);
    }
    const int64_t at = b * a.weights_seq_stride + h * a.weights_head_stride + t;
    if (t < s.n)
        a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + sum;
}

// The checks of kv_attend that need no stream.
kv_status check_attend(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *o, const kv_rows *q) {
    if (!cache)
        return fail(KV_EINVAL, "cache must not be NULL");
    kv_status st = check_layer(cache, 0);
    if (st != KV_OK)
        return st;
    if (!o)
        return fail(KV_EINVAL, "options must not be NULL");
    st = check_dtype(cache, o->cache_dtype);
    if (st == KV_OK)
        st = check_batch(cache, batch);
    if (st == KV_OK)
        st = check_rows(cache, batch, q, "q");
    if (st != KV_OK)
        return st;
    const int H = cache->layout.num_kv_heads;
    if (q->heads % H != 0)
        return fail(KV_EINVAL, "%d query heads for %d KV heads", q->heads, H);
    if (q->heads > 16383)
        return fail(KV_EUNSUPPORTED, "%d query heads (at most 16,383)", q->heads);
    const bool quantised = o->cache_dtype == KV_DTYPE_E4M3;
    if (!quantised && q->dtype != o->cache_dtype)
        return fail(KV_EINVAL, "rows of type %d for a cache of type %d", q->dtype, o->cache_dtype);
    if (!(o->scale >= 0.f && std::isfinite(o->scale)) || !(o->softcap >= 0.f && std::isfinite(o->softcap)) ||
        o->window < 0)
        return fail(KV_EINVAL, "scale, softcap and window must not be negative (got %g, %g, %d)", o->scale, o->softcap,
                    o->window);
    const float ks = o->k_scale == 0.f ? 1.f : o->k_scale, vs = o->v_scale == 0.f ? 1.f : o->v_scale;
    if (!(ks > 0.f && std::isfinite(ks)) || !(vs > 0.f && std::isfinite(vs)) ||
        (!quantised && (ks != 1.f || vs != 1.f)))
        return fail(KV_EINVAL, "scales must be positive, and 1 for a cache of 2-byte elements (got %g and %g)", ks, vs);
    if (o->weights_in && !o->weights_out)
        return fail(KV_EINVAL, "weights_in without weights_out");
    if (o->weights_out && (o->weights_seq_stride < 0 || o->weights_head_stride < 0 ||
                           (batch->num_seqs > 0 && H > 1 && o->weights_head_stride < batch->max_len) ||
                           (batch->num_seqs > 1 && o->weights_seq_stride < batch->max_len)))
        return fail(KV_EINVAL, "rows of weights (strides %lld and %lld) are shorter than max_len %d",
                    static_cast<long long>(o->weights_seq_stride), static_cast<long long>(o->weights_head_stride),
                    batch->max_len);
    return KV_OK;
}

// How a call is cut, and what its workspace holds.  Only the host's numbers count.
struct Plan {
    int32_t max_queries, max_rows, row_cap, split_len, splits;
    bool tail, scores;  // some sequence may have more than kStepRows rows; weights_out from the step kernel's scores
    int64_t score_len, lse_at, stats_at, sums_at, scores_at, bytes;
};

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

Plan plan_of(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *o, const kv_rows *q) {
    const int64_t H = cache->layout.num_kv_heads, D = cache->layout.head_dim, group = q->heads / H;
    const int64_t sequences = batch->num_seqs;
    Plan p{};
    p.max_queries = std::min(batch->max_queries, batch->num_queries);
    if (sequences == 0 || p.max_queries == 0)
        return p;
    const int64_t all_rows = p.max_queries * group;
    p.max_rows = static_cast<int32_t>(std::min<int64_t>(all_rows, kStepRows));
    p.tail = all_rows > kStepRows;
    // A sequence of more than one row per head has its weights recomputed (kept scores would outgrow K).
    p.scores = o->weights_out && all_rows <= 16;
    p.row_cap = p.max_rows;
    // Parts: about 4 workgroups of the step kernel per CU, of 128 to 4,096 tokens each (a ragged batch's longest
    // sequence must not be one workgroup's).
    const int64_t tile = step_tile_rows(p.max_rows, static_cast<int>(D)), tiles = (p.max_rows + tile - 1) / tile;
    int64_t longest = batch->max_len;
    if (o->window > 0)
        longest = std::min<int64_t>(longest, static_cast<int64_t>(o->window) + p.max_rows / group + 31);
    longest = std::max<int64_t>(longest, 1);
    const int64_t wanted = (1024 + sequences * H * tiles - 1) / (sequences * H * tiles);
    p.split_len = static_cast<int32_t>(
        std::min<int64_t>(4096, round_up((longest + wanted - 1) / wanted, 128)));
    p.splits = static_cast<int32_t>((longest + p.split_len - 1) / p.split_len);
    p.score_len = round_up(batch->max_len, 32);
    const int64_t slots = sequences * H * p.row_cap;
    p.lse_at = 0;
    p.stats_at = round_up(static_cast<int64_t>(batch->num_queries) * q->heads * 4, 16);
    p.sums_at = p.stats_at + (p.splits > 1 ? round_up(slots * p.splits * 8, 16) : 0);
    p.scores_at = p.sums_at + (p.splits > 1 ? slots * p.splits * D * 4 : 0);
    p.bytes = p.scores_at + (p.scores ? slots * p.score_len * 4 : 0);
    return p;
}

kv_status attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *o,
                 const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                 hipStream_t stream) {
    kv_status st = check_layer(cache, layer);
    if (st == KV_OK)
        st = check_attend(cache, batch, o, q);
    if (st == KV_OK)
        st = check_rows(cache, batch, out, "out");
    if (st != KV_OK)
        return st;
    if (out->heads != q->heads || out->dtype != q->dtype)
        return fail(KV_EINVAL, "out has %d heads of type %d, q %d of type %d", out->heads, out->dtype, q->heads,
                    q->dtype);
    const Plan plan = plan_of(cache, batch, o, q);
    const int64_t need = plan.bytes;
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(KV_EINVAL, "workspace of %lld bytes; %lld are needed", static_cast<long long>(workspace_bytes),
                    static_cast<long long>(need));
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(KV_EUNSUPPORTED, "workspace is not 16-byte aligned");
    if (batch->num_seqs == 0)
        return KV_OK;
    int32_t *err = nullptr;
    st = check_on_current_device(cache);
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    AttendArgs a{};
    a.pages = pages_of(cache, layer, err);
    a.batch = batch_of(batch);
    a.q = Rows{static_cast<uint8_t *>(q->data), q->token_stride * 2, q->head_stride * 2};
    a.out = Rows{static_cast<uint8_t *>(out->data), out->token_stride * 2, out->head_stride * 2};
    uint8_t *space = static_cast<uint8_t *>(workspace);
    a.lse = lse ? lse : reinterpret_cast<float *>(space + plan.lse_at);
    a.split_len = plan.split_len;
    a.splits = plan.splits;
    a.row_cap = plan.row_cap;
    a.part_stats = reinterpret_cast<float *>(space + plan.stats_at);
    a.part_sums = reinterpret_cast<float *>(space + plan.sums_at);
    a.scores = plan.scores ? reinterpret_cast<float *>(space + plan.scores_at) : nullptr;
    a.score_len = plan.score_len;
    a.slopes = o->slopes;
    a.weights_in = o->weights_in;
    a.weights_out = o->weights_out;
    a.weights_seq_stride = o->weights_seq_stride;
    a.weights_head_stride = o->weights_head_stride;
    a.scale = (o->scale == 0.f ? 1.f / std::sqrt(static_cast<float>(cache->layout.head_dim)) : o->scale) *
              (o->k_scale == 0.f ? 1.f : o->k_scale);
    a.softcap = o->softcap;
    a.v_scale = o->v_scale == 0.f ? 1.f : o->v_scale;
    a.window = o->window;
    a.heads = q->heads;
    a.group = q->heads / cache->layout.num_kv_heads;
    a.num_seqs = batch->num_seqs;
    a.q_type = q->dtype;
    a.cache_type = o->cache_dtype;
    a.by_group = divisor(a.group);
    if (plan.max_queries > 0) {
        KVX_HIP(launch_step(a, plan.max_queries, stream));
        if (plan.tail) {
            const dim3 grid(static_cast<uint32_t>(plan.max_queries), static_cast<uint32_t>(q->heads),
                            static_cast<uint32_t>(batch->num_seqs));
            hipLaunchKernelGGL(attend_kernel, grid, dim3(256), 0, stream, a);
            KVX_HIP(hipGetLastError());
        }
    }
    if (a.weights_out && !a.scores && batch->max_len > 0) {
        const dim3 grid(static_cast<uint32_t>((batch->max_len + 63) / 64), static_cast<uint32_t>(a.pages.H),
                        static_cast<uint32_t>(batch->num_seqs));
        hipLaunchKernelGGL(weigh_kernel, grid, dim3(64), 0, stream, a);
        KVX_HIP(hipGetLastError());
    }
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" {

int64_t kv_attend_workspace(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *options,
                            const kv_rows *q) {
    int64_t bytes = 0;
    const kv_status st = kvx::guarded([&]() -> kv_status {
        const kv_status checked = kvx::check_attend(cache, batch, options, q);
        if (checked == KV_OK)
            bytes = kvx::plan_of(cache, batch, options, q).bytes;
        return checked;
    });
    return st == KV_OK ? bytes : st;
}

kv_status kv_attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *options,
                    const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                    void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::attend(cache, layer, batch, options, q, out, lse, workspace, workspace_bytes,
                           static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
