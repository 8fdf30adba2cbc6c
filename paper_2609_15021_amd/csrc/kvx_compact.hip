// kv_compact: the kept tokens' rows of a paged cache into fresh pages.
//
// One 16-byte vector per lane, of kEach rows at once; consecutive lanes run along a row and then along one head's
// kept tokens, so reads are whole rows, and writes contiguous in HND pages.  Bound by HBM: every kept byte is read
// once and written once, 4,096 of 16,384 tokens of 8 sequences (8 heads of 256 bytes) at 4.9 TB/s, a large copy's
// rate; 3.8 with one row at a time and through the caches.
#include <algorithm>

#include "kvx_paged.h"

namespace kvx {

namespace {

typedef uint32_t vec16 __attribute__((ext_vector_type(4)));

constexpr int kEach = 4;  // rows that a lane has on their way

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
    const int units = kept * a.row_vecs, stride = gridDim.x * kThreads;
    const int32_t *keep = a.keep + (static_cast<int64_t>(b) * a.heads + (a.heads > 1 ? h : 0)) * a.budget;
    for (int u0 = blockIdx.x * kThreads + threadIdx.x; u0 < units; u0 += kEach * stride) {
        // kEach rows at once: their tokens, then their blocks, then their bytes.
        int token[kEach], src[kEach], dst[kEach];
        vec16 x[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            token[k] = keep[divide(min(u0 + k * stride, units - 1), a.by_row)];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int from = divide(max(token[k], 0), p.by_bs);
            const bool fits = token[k] >= 0 && from < a.src_len;
            src[k] = fits ? a.src[b * a.src_stride + from] : -1;
            dst[k] = a.dst[b * a.dst_stride + divide(divide(min(u0 + k * stride, units - 1), a.by_row), p.by_bs)];
            if (!fits) {
                report(p.err, KV_ASYNC_BAD_BATCH);
                continue;
            }
            const bool known = in_cache(p, src[k]), fresh = in_cache(p, dst[k]);
            src[k] = known && fresh ? src[k] : -1;
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = min(u0 + k * stride, units - 1), vec = u - divide(u, a.by_row) * a.row_vecs;
            const int slot = max(token[k], 0) - divide(max(token[k], 0), p.by_bs) * p.BS;
            const uint8_t *row =
                p.base + page_offset(p, max(src[k], 0), kv, h) + static_cast<uint32_t>(slot) * p.token_bytes;
            x[k] = __builtin_nontemporal_load(reinterpret_cast<const vec16 *>(row) + vec);
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = u0 + k * stride, j = divide(min(u, units - 1), a.by_row), vec = u - j * a.row_vecs;
            if (u < units && src[k] >= 0) {
                uint8_t *row = p.base + page_offset(p, dst[k], kv, h) +
                               static_cast<uint32_t>(j - divide(j, p.by_bs) * p.BS) * p.token_bytes;
                __builtin_nontemporal_store(x[k], reinterpret_cast<vec16 *>(row) + vec);
            }
        }
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
    if (budget * vecs > INT32_MAX - (int64_t{1} << 26))
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
    const int64_t groups = (budget * vecs + kEach * kThreads - 1) / (kEach * kThreads);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(groups, 32768)), static_cast<uint32_t>(num_seqs),
                    static_cast<uint32_t>(2 * lay.num_kv_heads));
    KVX_HIP(launch_kernel(compact_kernel, grid, kThreads, stream, a));
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
