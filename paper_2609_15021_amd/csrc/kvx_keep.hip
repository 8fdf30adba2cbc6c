// kv_keep: which tokens a sequence keeps under a budget, by accumulated attention weight.
//
// The heaviest m of the tokens between the sinks and the recent ones are those whose weight, as a 32-bit key that
// orders as the weights do, is above the m-th largest key, and as many of those equal to it, from the lowest token on,
// as are left.  One workgroup per row finds that key digit by digit from counts of the digit's values (a radix
// selection, 4 passes of 8 bits) and then writes the chosen tokens in order.
#include <algorithm>

#include "kvx_paged.h"

namespace kvx {

namespace {

constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / 64;

struct KeepArgs {
    const float *weights;
    int64_t seq_stride, head_stride;
    const int32_t *lens;
    int32_t heads, max_len, budget, sinks, recent;
    int32_t *keep, *kept_lens;
    float *kept_weights;
    int32_t *err;
};

// Orders as the weights do; both zeros alike, every NaN 0 (below -infinity).
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, w + 0.f);
    return w != w ? 0u : bits ^ (bits >> 31 ? 0xffffffffu : 0x80000000u);
}

__global__ __launch_bounds__(kKeepThreads) void keep_kernel(const KeepArgs a) {
    __shared__ int counts[256];
    __shared__ int found[2];
    __shared__ int wave_sums[2][kKeepWaves];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = a.lens[b];
    const int64_t row = static_cast<int64_t>(b) * a.heads + h;
    int32_t *keep = a.keep + row * a.budget;
    float *kept_weights = a.kept_weights ? a.kept_weights + row * a.budget : nullptr;
    if (n < 0 || n > a.max_len) {
        if (tid == 0)
            report(a.err, KV_ASYNC_BAD_BATCH);
        return;
    }
    const float *w = a.weights + b * a.seq_stride + h * a.head_stride;
    const int kept = min(n, a.budget);
    if (h == 0 && tid == 0)
        a.kept_lens[b] = kept;
    for (int j = kept + tid; j < a.budget; j += kKeepThreads) {
        keep[j] = -1;
        if (kept_weights)
            kept_weights[j] = 0.f;
    }
    if (n <= a.budget) {
        for (int j = tid; j < n; j += kKeepThreads) {
            keep[j] = j;
            if (kept_weights)
                kept_weights[j] = w[j];
        }
        return;
    }
    const int first = a.sinks, last = n - a.recent;  // chosen by weight: tokens [first, last)
    uint32_t threshold = 0, known = 0;               // the digits found so far, and their mask
    int left = a.budget - a.sinks - a.recent;        // tokens still to find at or below `threshold`'s digits
    const bool any = left > 0;
    for (int shift = 24; any && shift >= 0; shift -= 8) {
        if (tid < 256)
            counts[tid] = 0;
        __syncthreads();
        for (int t = first + tid; t < last; t += kKeepThreads) {
            const uint32_t key = key_of(w[t]);
            if ((key & known) == threshold)
                atomicAdd(&counts[key >> shift & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int digit = 255, above = 0;
            while (above + counts[digit] < left)
                above += counts[digit--];
            found[0] = digit;
            found[1] = above;
        }
        __syncthreads();
        threshold |= static_cast<uint32_t>(found[0]) << shift;
        known |= 255u << shift;
        left -= found[1];
    }
    // Chosen tokens in order: `at` tokens are written before this round's, `equal` of the threshold's key are seen.
    int at = 0, equal = 0;
    for (int t0 = 0; t0 < n; t0 += kKeepThreads) {
        const int t = t0 + tid;
        const float x = t < n ? w[t] : 0.f;
        const bool middle = t >= first && t < last;
        const uint32_t key = key_of(x);
        const bool tie = any && middle && key == threshold;
        const uint64_t ties = __ballot(tie);
        if (lane == 0)
            wave_sums[0][wave] = __popcll(ties);
        __syncthreads();
        int seen = equal;
        for (int i = 0; i < kKeepWaves; ++i) {
            const int c = wave_sums[0][i];
            seen += i < wave ? c : 0;
            equal += c;
        }
        const uint64_t below = (uint64_t{1} << lane) - 1;
        const bool chosen = t < n && (!middle || (any && (key > threshold || (tie && seen + static_cast<int>(__popcll(ties & below)) < left))));
        const uint64_t all = __ballot(chosen);
        if (lane == 0)
            wave_sums[1][wave] = __popcll(all);
        __syncthreads();
        int to = at + __popcll(all & below);
        for (int i = 0; i < kKeepWaves; ++i) {
            const int c = wave_sums[1][i];
            to += i < wave ? c : 0;
            at += c;
        }
        if (chosen) {
            keep[to] = t;
            if (kept_weights)
                kept_weights[to] = x;
        }
        __syncthreads();
    }
}

kv_status keep(const float *weights, int64_t seq_stride, int64_t head_stride, const int32_t *lens, int32_t num_seqs,
               int32_t heads, int32_t max_len, int32_t budget, int32_t sinks, int32_t recent, int32_t *keep,
               int32_t *kept_lens, float *kept_weights, hipStream_t stream) {
    if (num_seqs < 0 || heads < 1 || max_len < 0 || budget < 1 || sinks < 0 || recent < 0 || seq_stride < 0 ||
        head_stride < 0)
        return fail(KV_EINVAL, "num_seqs, max_len, sinks, recent and strides must not be negative, heads and budget "
                    "positive (num_seqs %d, heads %d, max_len %d, budget %d, sinks %d, recent %d)", num_seqs, heads,
                    max_len, budget, sinks, recent);
    if (static_cast<int64_t>(sinks) + recent > budget)
        return fail(KV_EINVAL, "%d sinks and %d recent tokens exceed the budget of %d", sinks, recent, budget);
    if (num_seqs > 65535)
        return fail(KV_EUNSUPPORTED, "%d sequences in one call (at most 65,535)", num_seqs);
    if (num_seqs == 0)
        return KV_OK;
    if (!lens || !keep || !kept_lens || (!weights && max_len > 0))
        return fail(KV_EINVAL, "weights, lens, keep and kept_lens must not be NULL");
    int32_t *err = nullptr;
    const kv_status st = error_word(&err);
    if (st != KV_OK)
        return st;
    const KeepArgs a{weights, seq_stride, head_stride, lens, heads, max_len, budget, sinks, recent,
                     keep, kept_lens, kept_weights, err};
    const dim3 grid(static_cast<uint32_t>(heads), static_cast<uint32_t>(num_seqs));
    hipLaunchKernelGGL(keep_kernel, grid, dim3(kKeepThreads), 0, stream, a);
    KVX_HIP(hipGetLastError());
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" kv_status kv_keep(const float *weights, int64_t seq_stride, int64_t head_stride, const int32_t *lens,
                             int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget, int32_t sinks,
                             int32_t recent, int32_t *keep, int32_t *kept_lens, float *kept_weights, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::keep(weights, seq_stride, head_stride, lens, num_seqs, heads, max_len, budget, sinks, recent, keep,
                         kept_lens, kept_weights, static_cast<hipStream_t>(stream));
    });
}
