// kv_compact: the kept tokens' rows of a paged cache into fresh pages.
//
// One 16-byte vector per lane; consecutive lanes run along a row and then along one head's kept tokens, so reads are
// whole rows, and writes contiguous in HND pages.  Bound by HBM: every kept byte is read once and written once.
#include <algorithm>

#include "kvx_paged.h"

namespace kvx {

namespace {

typedef uint32_t vec16 __attribute__((ext_vector_type(4)));

struct CompactArgs {
    Pages pages;
    const int32_t *src, *dst, *keep, *kept_lens;
    int64_t src_stride, dst_stride;
    int32_t src_len, heads, budget;
    Divisor by_row;  // division by vectors of a row
    int32_t row_vecs;
};

__global__ __launch_bounds__(kThreads) void compact_kernel(const CompactArgs a) {
    const Pages &p = a.pages;
    const int b = blockIdx.y, kv = blockIdx.z & 1, h = blockIdx.z >> 1;
    const int kept = a.kept_lens[b];
    if (kept < 0 || kept > a.budget) {
        if (threadIdx.x == 0)
            report(p.err, KV_ASYNC_BAD_BATCH);
        return;
    }
    const int units = kept * a.row_vecs;
    for (int u = blockIdx.x * kThreads + threadIdx.x; u < units; u += gridDim.x * kThreads) {
        const int j = divide(u, a.by_row), vec = u - j * a.row_vecs;
        const int t = a.keep[(static_cast<int64_t>(b) * a.heads + (a.heads > 1 ? h : 0)) * a.budget + j];
        const int from = divide(max(t, 0), p.by_bs), to = divide(j, p.by_bs);
        if (t < 0 || from >= a.src_len) {
            report(p.err, KV_ASYNC_BAD_BATCH);
            continue;
        }
        const int src = a.src[b * a.src_stride + from], dst = a.dst[b * a.dst_stride + to];
        if (!in_cache(p, src) || !in_cache(p, dst))
            continue;
        const uint8_t *x = p.base + page_offset(p, src, kv, h) + static_cast<uint32_t>(t - from * p.BS) * p.token_bytes;
        uint8_t *y = p.base + page_offset(p, dst, kv, h) + static_cast<uint32_t>(j - to * p.BS) * p.token_bytes;
        reinterpret_cast<vec16 *>(y)[vec] = reinterpret_cast<const vec16 *>(x)[vec];
    }
}

kv_status compact(const kv_cache *cache, int32_t layer, int32_t num_seqs, const int32_t *block_tables,
                  int64_t table_stride, int32_t table_len, const int32_t *keep, int32_t heads, int32_t budget,
                  const int32_t *kept_lens, const int32_t *dst_tables, int64_t dst_stride, int32_t dst_len,
                  hipStream_t stream) {
    kv_status st = check_layer(cache, layer);
    if (st != KV_OK)
        return st;
    const kv_layout &lay = cache->layout;
    if (num_seqs < 0 || budget < 1 || table_len < 0 || dst_len < 0 || table_stride < 0 || dst_stride < 0)
        return fail(KV_EINVAL, "num_seqs, table lengths and strides must not be negative, budget positive (num_seqs %d, "
                    "budget %d, table_len %d, dst_len %d)", num_seqs, budget, table_len, dst_len);
    if (heads != 1 && heads != lay.num_kv_heads)
        return fail(KV_EINVAL, "keep has %d heads for a cache of %d", heads, lay.num_kv_heads);
    if (num_seqs > 65535)
        return fail(KV_EUNSUPPORTED, "%d sequences in one call (at most 65,535)", num_seqs);
    if (num_seqs == 0)
        return KV_OK;
    if (budget > static_cast<int64_t>(dst_len) * lay.block_size)
        return fail(KV_EINVAL, "a budget of %d tokens exceeds %d pages of %d", budget, dst_len, lay.block_size);
    if (num_seqs > 1 && (table_stride < table_len || dst_stride < dst_len))
        return fail(KV_EINVAL, "table strides %lld and %lld are smaller than the tables (%d and %d)",
                    static_cast<long long>(table_stride), static_cast<long long>(dst_stride), table_len, dst_len);
    if (!block_tables || !keep || !kept_lens || !dst_tables)
        return fail(KV_EINVAL, "block_tables, keep, kept_lens and dst_tables must not be NULL");
    CompactArgs a{};
    if (lay.num_kv_heads > 32767)
        return fail(KV_EUNSUPPORTED, "%d KV heads (at most 32,767)", lay.num_kv_heads);
    const int64_t vecs = geometry(lay, 0).row_bytes / 16;
    if (budget * vecs > INT32_MAX - (int64_t{1} << 24))
        return fail(KV_EUNSUPPORTED, "%d kept tokens of a sequence in one call are too many", budget);
    int32_t *err = nullptr;
    st = check_on_current_device(cache);
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    a.pages = pages_of(cache, layer, err);
    a.src = block_tables;
    a.dst = dst_tables;
    a.keep = keep;
    a.kept_lens = kept_lens;
    a.src_stride = table_stride;
    a.dst_stride = dst_stride;
    a.src_len = table_len;
    a.heads = heads;
    a.budget = budget;
    a.row_vecs = a.pages.row_bytes / 16;
    a.by_row = divisor(a.row_vecs);
    const int64_t groups = (budget * vecs + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(groups, 32768)), static_cast<uint32_t>(num_seqs),
                    static_cast<uint32_t>(2 * lay.num_kv_heads));
    hipLaunchKernelGGL(compact_kernel, grid, dim3(kThreads), 0, stream, a);
    KVX_HIP(hipGetLastError());
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" kv_status kv_compact(const kv_cache *cache, int32_t layer, int32_t num_seqs, const int32_t *block_tables,
                                int64_t table_stride, int32_t table_len, const int32_t *keep, int32_t heads,
                                int32_t budget, const int32_t *kept_lens, const int32_t *dst_tables,
                                int64_t dst_stride, int32_t dst_len, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::compact(cache, layer, num_seqs, block_tables, table_stride, table_len, keep, heads, budget,
                            kept_lens, dst_tables, dst_stride, dst_len, static_cast<hipStream_t>(stream));
    });
}
