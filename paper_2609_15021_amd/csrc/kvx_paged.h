// Internal declarations of the operators on a paged cache (include/kvx_attend.h).
#pragma once

#include <tuple>

#include "kvx_internal.h"

#include "kvx_attend.h"

namespace kvx {

// One layer of a paged cache, as the kernels address it: row (kv, h) of token t, in block table[t / BS], is at
//   base + block * block_stride + kv * v_bytes + h * head_bytes + (t % BS) * token_bytes.
// Offsets inside a block fit 31 bits (a block has at most 2 GiB), blocks need 64.
struct Pages {
    uint8_t *base;
    int64_t block_stride;
    int32_t num_blocks, BS;
    Divisor by_bs;
    uint32_t token_bytes, head_bytes, v_bytes;
    int32_t row_bytes;
    int32_t H, D;
    int32_t *err;  // the device's async error word
};

// kv_batch on the device.
struct Batch {
    const int32_t *tables, *lens, *starts;
    int64_t table_stride;
    int32_t table_len, num_queries, max_queries, max_len;
};

struct Rows {
    uint8_t *data;
    int64_t token_stride, head_stride;  // bytes
};

// kv_page_scales on the device; data NULL: pages have none.
struct Scales {
    uint8_t *data;
    int64_t block_stride, kv_stride;
};

__device__ __forceinline__ uint8_t *scale_at(const Scales &s, int block, int kv, int h) {
    return s.data + block * s.block_stride + kv * s.kv_stride + h;
}

// 2^(e - 127) for e from 1 to 254.
__device__ __forceinline__ float power_of(int e) { return __builtin_bit_cast(float, e << 23); }

// One sequence of a batch: n tokens, its new ones the rows q0 .. q0 + nq.
struct Sequence {
    int n, q0, nq;
};

__device__ __forceinline__ void report(int32_t *err, int bit) { atomicOr(err, bit); }

// Sequence b, or false (reported) where its numbers are outside the batch's bounds.
__device__ __forceinline__ bool sequence(const Batch &batch, int b, int32_t *err, Sequence &s) {
    s.n = batch.lens[b];
    s.q0 = batch.starts ? batch.starts[b] : b;
    const int q1 = batch.starts ? batch.starts[b + 1] : b + 1;
    if (s.n < 0 || s.n > batch.max_len || s.q0 < 0 || q1 < s.q0 || q1 > batch.num_queries ||
        q1 - s.q0 > batch.max_queries) {
        if (threadIdx.x == 0)
            report(err, KV_ASYNC_BAD_BATCH);
        return false;
    }
    s.nq = q1 - s.q0;
    return true;
}

// Byte offset of slot 0 of page `block` for head h of K (kv 0) or V.
__device__ __forceinline__ int64_t page_offset(const Pages &p, int block, int kv, int h) {
    return block * p.block_stride + (kv ? p.v_bytes : 0u) + static_cast<uint32_t>(h) * p.head_bytes;
}

// Whether a block id names a page; reported if not.
__device__ __forceinline__ bool in_cache(const Pages &p, int block) {
    if (static_cast<uint32_t>(block) < static_cast<uint32_t>(p.num_blocks))
        return true;
    report(p.err, KV_ASYNC_BAD_BLOCK);
    return false;
}

// Launches kernel(args...), whose own error it returns.
template <class... Args, class... Given>
hipError_t launch_kernel(void (*kernel)(Args...), dim3 grid, int threads, hipStream_t stream, const Given &...given) {
    std::tuple<Args...> args(given...);
    return std::apply(
        [&](auto &...arg) {
            void *kernel_args[] = {&arg...};
            return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(static_cast<uint32_t>(threads)),
                                   kernel_args, 0, stream);
        },
        args);
}

// Host side.
kv_status check_layer(const kv_cache *cache, int32_t layer);
kv_status check_batch(const kv_cache *cache, const kv_batch *batch);
kv_status check_rows(const kv_cache *cache, const kv_batch *batch, const kv_rows *rows, const char *name);
kv_status check_dtype(const kv_cache *cache, int32_t cache_dtype);
kv_status check_scales(const kv_cache *cache, int32_t cache_dtype, const kv_page_scales *scales);
kv_status check_on_current_device(const kv_cache *cache);
kv_status error_word(int32_t **out);  // the current device's
Pages pages_of(const kv_cache *cache, int32_t layer, int32_t *err);
Batch batch_of(const kv_batch *batch);
Scales scales_of(const kv_page_scales *scales);  // NULL: none
Rows rows_of(const kv_rows *rows);

}  // namespace kvx
