// Host side shared by the operators on a paged cache: the checks of what they are given, and the async error word.
#include "kvx_paged.h"

// Faults that only the device can see, of every operator of kvx_attend.h on the device (zero when the process starts).
static __device__ int32_t attend_error;

namespace kvx {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_error_mu;
int32_t *g_error_ptr[kMaxDevices] = {};

}  // namespace

kv_status error_word(int32_t **out) {
    int dev = -1;
    KVX_HIP(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices)
        return fail(KV_EUNSUPPORTED, "device ordinal %d is beyond the %d the library tracks", dev, kMaxDevices);
    std::lock_guard<std::mutex> lock(g_error_mu);
    if (!g_error_ptr[dev]) {
        void *p = nullptr;
        KVX_HIP(hipGetSymbolAddress(&p, HIP_SYMBOL(attend_error)));
        if (!p)
            return fail(KV_EHIP, "hipGetSymbolAddress(attend_error) returned NULL on device %d", dev);
        g_error_ptr[dev] = static_cast<int32_t *>(p);
    }
    *out = g_error_ptr[dev];
    return KV_OK;
}

kv_status check_layer(const kv_cache *cache, int32_t layer) {
    if (!cache)
        return fail(KV_EINVAL, "cache must not be NULL");
    kv_status st = check_layout(cache->layout);
    if (st != KV_OK)
        return st;
    if (cache->num_blocks <= 0)
        return fail(KV_EINVAL, "num_blocks must be positive (got %d)", cache->num_blocks);
    if (cache->block_order != KV_BLOCK_HND && cache->block_order != KV_BLOCK_NHD)
        return fail(KV_EINVAL, "block_order must be KV_BLOCK_HND or KV_BLOCK_NHD (got %d)", cache->block_order);
    if (cache->reserved != 0)
        return fail(KV_EINVAL, "kv_cache.reserved must be 0");
    const Geometry g = geometry(cache->layout, cache->block_stride_bytes);
    if (cache->block_stride_bytes != 0 && cache->block_stride_bytes < g.block_bytes)
        return fail(KV_EINVAL, "block_stride_bytes %lld is smaller than one block (%lld bytes)",
                    static_cast<long long>(cache->block_stride_bytes), static_cast<long long>(g.block_bytes));
    if (g.block_stride % 16 != 0)
        return fail(KV_EUNSUPPORTED, "block_stride_bytes %lld is not 16-byte aligned",
                    static_cast<long long>(g.block_stride));
    if (layer < 0 || layer >= cache->layout.num_layers)
        return fail(KV_EINVAL, "layer %d is outside [0, %d)", layer, cache->layout.num_layers);
    if (!cache->layer_ptrs || !cache->layer_ptrs[layer])
        return fail(KV_EINVAL, "layer_ptrs[%d] is NULL", layer);
    if (reinterpret_cast<uintptr_t>(cache->layer_ptrs[layer]) % 16 != 0)
        return fail(KV_EUNSUPPORTED, "layer_ptrs[%d] is not 16-byte aligned", layer);
    return KV_OK;
}

kv_status check_batch(const kv_cache *cache, const kv_batch *batch) {
    if (!batch)
        return fail(KV_EINVAL, "batch must not be NULL");
    if (batch->num_seqs < 0 || batch->num_queries < 0 || batch->max_queries < 1 || batch->max_len < 0 ||
        batch->table_len < 0 || batch->table_stride < 0)
        return fail(KV_EINVAL, "batch sizes must not be negative, and max_queries at least 1 (num_seqs %d, num_queries "
                    "%d, max_queries %d, max_len %d, table_len %d, table_stride %lld)", batch->num_seqs,
                    batch->num_queries, batch->max_queries, batch->max_len, batch->table_len,
                    static_cast<long long>(batch->table_stride));
    if (batch->reserved != 0)
        return fail(KV_EINVAL, "kv_batch.reserved must be 0");
    if (batch->num_seqs == 0)
        return KV_OK;
    if (batch->num_seqs > 65535)
        return fail(KV_EUNSUPPORTED, "%d sequences in one call (at most 65,535)", batch->num_seqs);
    if (batch->max_len > INT32_MAX - 1023)
        return fail(KV_EUNSUPPORTED, "sequences of up to %d tokens (at most 2^31 - 1024)", batch->max_len);
    if (batch->max_len > static_cast<int64_t>(batch->table_len) * cache->layout.block_size)
        return fail(KV_EINVAL, "max_len %d exceeds %d pages of %d tokens", batch->max_len, batch->table_len,
                    cache->layout.block_size);
    if (batch->num_seqs > 1 && batch->table_stride < batch->table_len)
        return fail(KV_EINVAL, "table_stride %lld is smaller than table_len %d",
                    static_cast<long long>(batch->table_stride), batch->table_len);
    if ((!batch->block_tables && batch->table_len > 0) || !batch->lens)
        return fail(KV_EINVAL, "block_tables and lens must not be NULL");
    if (!batch->starts && (batch->num_queries < batch->num_seqs))
        return fail(KV_EINVAL, "%d rows of new tokens for %d sequences of one each", batch->num_queries,
                    batch->num_seqs);
    return KV_OK;
}

kv_status check_dtype(const kv_cache *cache, int32_t cache_dtype) {
    if (cache_dtype != KV_DTYPE_BF16 && cache_dtype != KV_DTYPE_F16 && cache_dtype != KV_DTYPE_E4M3)
        return fail(KV_EINVAL, "cache_dtype must be a KV_DTYPE (got %d)", cache_dtype);
    const int size = cache_dtype == KV_DTYPE_E4M3 ? 1 : 2;
    if (cache->layout.elem_bytes != size)
        return fail(KV_EINVAL, "cache_dtype of %d bytes for a cache of %d-byte elements", size,
                    cache->layout.elem_bytes);
    if (cache->layout.head_dim > 256)
        return fail(KV_EUNSUPPORTED, "head_dim %d is over 256", cache->layout.head_dim);
    return KV_OK;
}

kv_status check_rows(const kv_cache *cache, const kv_batch *batch, const kv_rows *rows, const char *name) {
    if (!rows)
        return fail(KV_EINVAL, "%s must not be NULL", name);
    if (rows->dtype != KV_DTYPE_BF16 && rows->dtype != KV_DTYPE_F16)
        return fail(KV_EINVAL, "%s: rows are KV_DTYPE_BF16 or KV_DTYPE_F16 (got %d)", name, rows->dtype);
    if (rows->heads < 1)
        return fail(KV_EINVAL, "%s: heads must be positive (got %d)", name, rows->heads);
    if (rows->token_stride < 0 || rows->head_stride < 0)
        return fail(KV_EINVAL, "%s: strides must not be negative", name);
    if (batch->num_seqs == 0 || batch->num_queries == 0)
        return KV_OK;
    if (!rows->data)
        return fail(KV_EINVAL, "%s: data must not be NULL", name);
    // (A stride over one token or head leads nowhere, and tensors have any there.)
    if (reinterpret_cast<uintptr_t>(rows->data) % 16 != 0 || (batch->num_queries > 1 && rows->token_stride % 8 != 0) ||
        (rows->heads > 1 && rows->head_stride % 8 != 0))
        return fail(KV_EUNSUPPORTED, "%s: rows must start at multiples of 16 bytes", name);
    return KV_OK;
}

kv_status check_scales(const kv_cache *cache, int32_t cache_dtype, const kv_page_scales *scales) {
    if (cache_dtype != KV_DTYPE_E4M3)
        return fail(KV_EINVAL, "scales of pages for a cache of type %d", cache_dtype);
    const int64_t H = cache->layout.num_kv_heads;
    if (!scales->data)
        return fail(KV_EINVAL, "scales: data must not be NULL");
    if (scales->kv_stride < H || scales->block_stride < scales->kv_stride ||
        scales->block_stride - scales->kv_stride < H)
        return fail(KV_EINVAL, "scales of %lld heads overlap (strides of %lld and %lld bytes)", static_cast<long long>(H),
                    static_cast<long long>(scales->block_stride), static_cast<long long>(scales->kv_stride));
    return KV_OK;
}

kv_status check_on_current_device(const kv_cache *cache) {
    int cur = -1;
    KVX_HIP(hipGetDevice(&cur));
    if (cache->device != cur)
        return fail(KV_EINVAL, "cache is on device %d, current device %d", cache->device, cur);
    return KV_OK;
}

Pages pages_of(const kv_cache *cache, int32_t layer, int32_t *err) {
    const Geometry g = geometry(cache->layout, cache->block_stride_bytes);
    const bool nhd = cache->block_order == KV_BLOCK_NHD;
    Pages p{};
    p.base = static_cast<uint8_t *>(cache->layer_ptrs[layer]);
    p.block_stride = g.block_stride;
    p.num_blocks = cache->num_blocks;
    p.BS = static_cast<int32_t>(g.BS);
    p.by_bs = divisor(g.BS);
    p.token_bytes = static_cast<uint32_t>(nhd ? g.H * g.row_bytes : g.row_bytes);
    p.head_bytes = static_cast<uint32_t>(nhd ? g.row_bytes : g.BS * g.row_bytes);
    p.v_bytes = static_cast<uint32_t>(g.block_bytes / 2);
    p.row_bytes = static_cast<int32_t>(g.row_bytes);
    p.H = static_cast<int32_t>(g.H);
    p.D = static_cast<int32_t>(g.D);
    p.err = err;
    return p;
}

Batch batch_of(const kv_batch *batch) {
    Batch b{};
    b.tables = batch->block_tables;
    b.lens = batch->lens;
    b.starts = batch->starts;
    b.table_stride = batch->table_stride;
    b.table_len = batch->table_len;
    b.num_queries = batch->num_queries;
    b.max_queries = batch->max_queries;
    b.max_len = batch->max_len;
    return b;
}

Scales scales_of(const kv_page_scales *scales) {
    return scales ? Scales{scales->data, scales->block_stride, scales->kv_stride} : Scales{nullptr, 0, 0};
}

Rows rows_of(const kv_rows *rows) {
    return Rows{static_cast<uint8_t *>(rows->data), rows->token_stride * 2, rows->head_stride * 2};
}

}  // namespace kvx

extern "C" int32_t kv_attend_async_error(int clear) {
    int32_t mask = 0;
    const kv_status st = kvx::guarded([&]() -> kv_status {
        int32_t *word = nullptr;
        const kv_status found = kvx::error_word(&word);
        if (found != KV_OK)
            return found;
        KVX_HIP(hipMemcpy(&mask, word, sizeof(mask), hipMemcpyDeviceToHost));
        const int32_t zero = 0;
        if (clear)
            KVX_HIP(hipMemcpy(word, &zero, sizeof(zero), hipMemcpyHostToDevice));
        return KV_OK;
    });
    return st == KV_OK ? mask : st;
}
