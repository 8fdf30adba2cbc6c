// kv_append: the new tokens' K and V rows into a paged cache, as they are or as e4m3.
//
// One 16-byte vector of the cache per lane: consecutive lanes run along a row, then along a token's heads, as the
// source lies.  2,608 new tokens of 4 heads of 256 to e4m3 (16 MB read and written once, 3.5 us at a large copy's
// rate) take 6.5 to 7.2 us on the GPU: a lane waits for its page's number, then for its row, and has one of each on
// its way.  A decoding step is bound by the launch (2.4 to 2.8 us on the GPU, 10 with the host).
#include <algorithm>
#include <cmath>

#include "kvx_rows.h"

namespace kvx {

namespace {

struct AppendArgs {
    Pages pages;
    Batch batch;
    Rows k, v;
    Divisor by_row, by_head;  // division by vectors of a row and by H
    int32_t row_vecs, token_vecs;
    float k_scale, v_scale;
};

// Eight 2-byte values as e4m3 of x / scale, rounded to nearest even: 8 bytes.  (A division, not a product with the
// inverse: the quotient is rounded once to 32 bits and once to 8.)
template <int DTYPE>
__device__ __forceinline__ void quantise(const vec16 &x, float scale, uint32_t *out) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int packed = 0;
        const uint32_t a = x[2 * w], b = x[2 * w + 1];
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(to_float(a & 0xffff, DTYPE) / scale),
                                                 clamp_e4m3(to_float(a >> 16, DTYPE) / scale), packed, false);
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(to_float(b & 0xffff, DTYPE) / scale),
                                                 clamp_e4m3(to_float(b >> 16, DTYPE) / scale), packed, true);
        out[w] = static_cast<uint32_t>(packed);
    }
}

// QUANT: 0 as they are, else the rows' KV_DTYPE.
template <int QUANT>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendArgs a) {
    const int b = blockIdx.y;
    Sequence s;
    if (!sequence(a.batch, b, a.pages.err, s))
        return;
    const int half = s.nq * a.token_vecs;  // vectors of K (or V)
    for (int at = blockIdx.x * kThreads + threadIdx.x; at < 2 * half; at += gridDim.x * kThreads) {
        const int kv = at >= half, u = at - kv * half;
        const int r = divide(u, a.by_row), vec = u - r * a.row_vecs;  // r: (row, head)
        const int row = divide(r, a.by_head), h = r - row * a.pages.H;
        const int t = s.n - s.nq + row;
        if (t < 0)
            continue;
        const int page = divide(t, a.pages.by_bs);
        const int block = a.batch.tables[b * a.batch.table_stride + page];
        if (!in_cache(a.pages, block))
            continue;
        const Rows &src = kv ? a.v : a.k;
        const uint8_t *from = src.data + (s.q0 + row) * src.token_stride + h * src.head_stride;
        uint8_t *to = a.pages.base + page_offset(a.pages, block, kv, h) +
                      static_cast<uint32_t>(t - page * a.pages.BS) * a.pages.token_bytes + vec * 16;
        if constexpr (QUANT == 0) {
            *reinterpret_cast<vec16 *>(to) = *reinterpret_cast<const vec16 *>(from + vec * 16);
        } else {
            const vec16 *x = reinterpret_cast<const vec16 *>(from + vec * 32);
            const float scale = kv ? a.v_scale : a.k_scale;
            uint32_t out[4];
            quantise<QUANT>(x[0], scale, out);
            quantise<QUANT>(x[1], scale, out + 2);
            *reinterpret_cast<vec16 *>(to) = vec16{out[0], out[1], out[2], out[3]};
        }
    }
}

}  // namespace

kv_status check_append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k, const kv_rows *v,
                       int32_t cache_dtype) {
    kv_status st = check_layer(cache, layer);
    if (st == KV_OK)
        st = check_dtype(cache, cache_dtype);
    if (st == KV_OK)
        st = check_batch(cache, batch);
    if (st == KV_OK)
        st = check_rows(cache, batch, k, "k");
    if (st == KV_OK)
        st = check_rows(cache, batch, v, "v");
    if (st != KV_OK)
        return st;
    const int H = cache->layout.num_kv_heads;
    if (k->heads != H || v->heads != H)
        return fail(KV_EINVAL, "rows of %d and %d heads for a cache of %d", k->heads, v->heads, H);
    if (k->dtype != v->dtype)
        return fail(KV_EINVAL, "k and v have different types");
    if (cache_dtype != KV_DTYPE_E4M3 && k->dtype != cache_dtype)
        return fail(KV_EINVAL, "rows of type %d for a cache of type %d", k->dtype, cache_dtype);
    return KV_OK;
}

kv_status check_factors(int32_t cache_dtype, float k_scale, float v_scale) {
    k_scale = k_scale == 0.f ? 1.f : k_scale;
    v_scale = v_scale == 0.f ? 1.f : v_scale;
    if (!(k_scale > 0.f && std::isfinite(k_scale)) || !(v_scale > 0.f && std::isfinite(v_scale)) ||
        (cache_dtype != KV_DTYPE_E4M3 && (k_scale != 1.f || v_scale != 1.f)))
        return fail(KV_EINVAL, "scales must be positive and finite, and 1 for a cache of 2-byte elements (got %g and "
                    "%g)", k_scale, v_scale);
    return KV_OK;
}

namespace {

kv_status append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k, const kv_rows *v,
                 int32_t cache_dtype, float k_scale, float v_scale, hipStream_t stream) {
    kv_status st = check_append(cache, layer, batch, k, v, cache_dtype);
    if (st == KV_OK)
        st = check_factors(cache_dtype, k_scale, v_scale);
    if (st != KV_OK)
        return st;
    const int H = cache->layout.num_kv_heads;
    const bool quantised = cache_dtype == KV_DTYPE_E4M3;
    k_scale = k_scale == 0.f ? 1.f : k_scale;
    v_scale = v_scale == 0.f ? 1.f : v_scale;
    if (batch->num_seqs == 0 || batch->num_queries == 0)
        return KV_OK;
    st = check_on_current_device(cache);
    int32_t *err = nullptr;
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    AppendArgs a{};
    a.pages = pages_of(cache, layer, err);
    a.batch = batch_of(batch);
    a.k = rows_of(k);
    a.v = rows_of(v);
    a.row_vecs = a.pages.row_bytes / 16;
    a.token_vecs = a.row_vecs * H;
    a.by_row = divisor(a.row_vecs);
    a.by_head = divisor(H);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    const int64_t most = std::min(batch->max_queries, batch->num_queries);
    if (2 * most * a.token_vecs > INT32_MAX - (int64_t{1} << 24))
        return fail(KV_EUNSUPPORTED, "%lld new tokens of a sequence in one call are too many",
                    static_cast<long long>(most));
    const int64_t groups = (2 * most * a.token_vecs + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(groups, 32768)), static_cast<uint32_t>(batch->num_seqs));
    const auto kernel = !quantised                  ? append_kernel<0>
                        : k->dtype == KV_DTYPE_BF16 ? append_kernel<KV_DTYPE_BF16>
                                                    : append_kernel<KV_DTYPE_F16>;
    KVX_HIP(launch_kernel(kernel, grid, kThreads, stream, a));
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" kv_status kv_append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k,
                               const kv_rows *v, int32_t cache_dtype, float k_scale, float v_scale, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::append(cache, layer, batch, k, v, cache_dtype, k_scale, v_scale, static_cast<hipStream_t>(stream));
    });
}
