// kv_append_scaled: the new tokens' K and V rows into e4m3 pages with a scale for each page, K or V, and head.
//
// The scale is a power of two, 2^k with the largest |x| in (224, 448] * 2^k: e4m3 is a floating-point type, so a finer
// scale would only move where its smallest numbers are, and a power of two makes everything around it exact: x / scale,
// rounding a page's older rows again when its scale grows, and applying it in attention.
//
// A workgroup has one (page, K or V, head): it takes the new rows of the page, finds their largest |x|, and with the
// page's old scale the new one; rounds older rows if the scale grew; and writes the new ones, of which it holds kHeld
// in a lane's registers.  2,608 new tokens of 4 heads of 256 (16 MB read and written once, 3.4 us at a large copy's
// rate) take 8.0 us on the GPU: beside the launch, lengths, then rows and tables are waited for one after the other (a
// scale only where a page has older rows), and there is one set of rows for each workgroup.  A decoding step of 48
// tokens takes 4.1 (5.8 with the host).
//
// For kv_rotate K is normed and rotated here, with angles worked out in every lane, for every row and head: that is
// most of kv_rotate's time with scales.  2,085 tokens of 40 query heads and 8 KV heads (D 128) take 39 us in both
// launches (17 with one factor for the cache, 12 at a large copy's rate; 23 without norms and angles), 3 tokens 14
// (4.5).
#include <algorithm>

#include "kvx_rows.h"

namespace kvx {

namespace {

constexpr int kHeld = 4;

struct ScaledArgs {
    Pages pages;
    Batch batch;
    Rows rows[2];  // K, V
    Scales scales;
    Turn turn;     // of K
};

// The exponent byte of the smallest power of two that |x| <= 448 * 2^(e - 127) holds for, from the bits of |x| (448 is
// 1.75 * 2^8: a larger mantissa needs one more).
__device__ __forceinline__ int exponent_for(uint32_t bits) {
    return max(static_cast<int>((bits + 0x1fffff) >> 23) - 8, 1);
}

template <int DTYPE, int LPR, Pairs PAIRS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void append_scaled_kernel(const ScaledArgs a) {
    constexpr int kSlots = 64 * WAVES / LPR;  // rows at once
    __shared__ uint32_t wave_most[WAVES];
    const Pages &p = a.pages;
    const int b = blockIdx.y, kv = blockIdx.z & 1, h = blockIdx.z >> 1, tid = threadIdx.x;
    Sequence s;
    if (!sequence(a.batch, b, p.err, s) || s.nq == 0 || s.n == 0)
        return;
    const int first = s.n - s.nq, begin = max(first, 0);  // (rows before token 0 have no place)
    const int64_t page64 = int64_t{divide(begin, p.by_bs)} + blockIdx.x;
    if (page64 * p.BS >= s.n)
        return;
    const int page = static_cast<int>(page64), start = page * p.BS;
    const int t0 = max(begin, start), old = t0 - start;
    const int rows = static_cast<int>(min(int64_t{s.n}, int64_t{start} + p.BS)) - t0;
    const int block = a.batch.tables[b * a.batch.table_stride + page];
    const Turner<DTYPE, PAIRS, LPR> turner(a.turn, tid % LPR, p.D);
    const Turner<DTYPE, kAsIs, LPR> as_is(a.turn, tid % LPR, p.D);
    const bool turn = PAIRS != kAsIs && kv == 0;
    typename Turner<DTYPE, PAIRS, LPR>::Weights weights;
    if (turn)
        weights = turner.weights(a.turn, [&](int d) { return a.turn.weight ? norm_weight<DTYPE>(a.turn, d) : 1.f; });
    const int slot = tid / LPR, d0 = turner.d0;
    const Rows &src = a.rows[kv];
    const uint8_t *from = src.data + (int64_t{s.q0} + (t0 - first)) * src.token_stride + h * src.head_stride;
    const auto load = [&](int row) {
        const uint8_t *x = from + row * src.token_stride;
        return turn ? turner.load(a.turn, x) : typename Turner<DTYPE, PAIRS, LPR>::Vec{as_is.load(a.turn, x).own, {}};
    };
    const auto finish = [&](const typename Turner<DTYPE, PAIRS, LPR>::Vec &v, int row, float *y) {
        if (turn) {
            const int position = a.turn.positions ? a.turn.positions[s.q0 + t0 - first + row] : t0 + row;
            const auto angles = turner.angles(a.turn, [&](int i, float &c, float &si) {
                turn_by(position, a.turn.freqs[i], a.turn.magnitude, c, si);
            });
            turner.finish(a.turn, v, a.turn.weight != nullptr, weights, angles, y);
        } else {
            to_floats<DTYPE>(v.own, y);
        }
    };
    // (All lanes of a row take part in its norm; rows beyond the last repeat it.  They are on their way while the page
    // is looked up.)
    typename Turner<DTYPE, PAIRS, LPR>::Vec v[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        v[k] = load(min(slot + k * kSlots, rows - 1));
    if (!in_cache(p, block))
        return;
    uint8_t *exponent = scale_at(a.scales, block, kv, h);
    const int before = old > 0 ? *exponent : 0;
    uint32_t most = 0;  // bits of the largest finite |x|
    const auto count = [&](const float *y) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, y[j]) & 0x7fffffff;
            most = max(most, bits < 0x7f800000 ? bits : 0);
        }
    };

    float held[kHeld][8];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        finish(v[k], min(slot + k * kSlots, rows - 1), held[k]);
        count(held[k]);
    }
    for (int row = slot + kHeld * kSlots; row < rows; row += kSlots) {
        float y[8];
        finish(load(row), row, y);
        count(y);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1)
        most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), o)));
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0)
            wave_most[tid >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            most = max(most, wave_most[w]);
    }
    const int e = max(exponent_for(most), before);
    if (tid == 0)
        *exponent = static_cast<uint8_t>(e);

    uint8_t *to = p.base + page_offset(p, block, kv, h) + d0;
    if (old > 0 && e > before && turner.any) {
        for (int row = slot; row < old; row += kSlots) {
            vec8 *x = reinterpret_cast<vec8 *>(to + static_cast<uint32_t>(row) * p.token_bytes);
            const vec8 stored = *x;
            float y[8];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(stored[w]), false);
                const auto high = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(stored[w]), true);
                y[4 * w] = low[0];
                y[4 * w + 1] = low[1];
                y[4 * w + 2] = high[0];
                y[4 * w + 3] = high[1];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                y[j] = ldexpf(y[j], before - e);
            *x = to_e4m3(y);
        }
    }
    const auto put = [&](int row, const float *y) {
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = ldexpf(y[j], 127 - e);
        if (turner.any)
            *reinterpret_cast<vec8 *>(to + static_cast<uint32_t>(old + row) * p.token_bytes) = to_e4m3(z);
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (slot + k * kSlots < rows)
            put(slot + k * kSlots, held[k]);
    for (int row = slot + kHeld * kSlots; row < rows; row += kSlots) {
        float y[8];
        finish(load(row), row, y);
        put(row, y);
    }
}

template <int DTYPE, int LPR, Pairs PAIRS>
hipError_t launch(const ScaledArgs &a, const dim3 &grid, int most_rows, hipStream_t stream) {
    // One wave where it has all rows of a page at once, 4 where it does not.
    if (most_rows <= 64 / LPR)
        return launch_kernel(append_scaled_kernel<DTYPE, LPR, PAIRS, 1>, grid, 64, stream, a);
    return launch_kernel(append_scaled_kernel<DTYPE, LPR, PAIRS, 4>, grid, 256, stream, a);
}

template <int DTYPE, int LPR>
hipError_t launch(const ScaledArgs &a, const dim3 &grid, int most_rows, Pairs pairs, hipStream_t stream) {
    switch (pairs) {
    case kAsIs: return launch<DTYPE, LPR, kAsIs>(a, grid, most_rows, stream);
    case kNeighbours: return launch<DTYPE, LPR, kNeighbours>(a, grid, most_rows, stream);
    case kHalves: return launch<DTYPE, LPR, kHalves>(a, grid, most_rows, stream);
    default: return launch<DTYPE, LPR, kAnyHalves>(a, grid, most_rows, stream);
    }
}

template <int DTYPE>
hipError_t launch(const ScaledArgs &a, const dim3 &grid, int most_rows, Pairs pairs, hipStream_t stream) {
    const int lanes = lanes_of(a.pages.D);
    return lanes == 32   ? launch<DTYPE, 32>(a, grid, most_rows, pairs, stream)
           : lanes == 16 ? launch<DTYPE, 16>(a, grid, most_rows, pairs, stream)
                         : launch<DTYPE, 8>(a, grid, most_rows, pairs, stream);
}

kv_status append_scaled(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k, const kv_rows *v,
                        const kv_page_scales *scales, hipStream_t stream) {
    kv_status st = check_append(cache, layer, batch, k, v, KV_DTYPE_E4M3);
    if (st != KV_OK)
        return st;
    if (!scales)
        return fail(KV_EINVAL, "scales must not be NULL");
    st = check_scales(cache, KV_DTYPE_E4M3, scales);
    if (st == KV_OK)
        st = check_append_scaled(cache, batch);
    if (st != KV_OK || batch->num_seqs == 0 || batch->num_queries == 0)
        return st;
    st = check_on_current_device(cache);
    int32_t *err = nullptr;
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    KVX_HIP(launch_append_scaled(pages_of(cache, layer, err), batch_of(batch), batch->num_seqs, rows_of(k), rows_of(v),
                                 k->dtype, scales_of(scales), Turn{}, kAsIs, stream));
    return KV_OK;
}

// Tokens of a sequence that are new at most, and pages that they may lie in.
int most_new(int max_queries, int num_queries, int max_len) { return std::min({max_queries, num_queries, max_len}); }
int64_t most_touched(int most, int BS) { return (int64_t{most} + BS - 2) / BS + 1; }

}  // namespace

kv_status check_append_scaled(const kv_cache *cache, const kv_batch *batch) {
    if (cache->layout.num_kv_heads > 32767)
        return fail(KV_EUNSUPPORTED, "%d KV heads (at most 32,767)", cache->layout.num_kv_heads);
    const int most = most_new(batch->max_queries, batch->num_queries, batch->max_len);
    if (most_touched(most, cache->layout.block_size) > int64_t{1} << 23)
        return fail(KV_EUNSUPPORTED, "%d new tokens of a sequence in one call are too many", most);
    return KV_OK;
}

hipError_t launch_append_scaled(const Pages &pages, const Batch &batch, int32_t num_seqs, const Rows &k, const Rows &v,
                                int32_t dtype, const Scales &scales, const Turn &turn, Pairs pairs, hipStream_t stream) {
    ScaledArgs a{};
    a.pages = pages;
    a.batch = batch;
    a.rows[0] = k;
    a.rows[1] = v;
    a.scales = scales;
    a.turn = turn;
    const int most = most_new(batch.max_queries, batch.num_queries, batch.max_len);
    if (most == 0)
        return hipSuccess;
    const dim3 grid(static_cast<uint32_t>(most_touched(most, pages.BS)), static_cast<uint32_t>(num_seqs),
                    static_cast<uint32_t>(2 * pages.H));
    const int rows = std::min(most, pages.BS);
    return dtype == KV_DTYPE_BF16 ? launch<KV_DTYPE_BF16>(a, grid, rows, pairs, stream)
                                  : launch<KV_DTYPE_F16>(a, grid, rows, pairs, stream);
}

}  // namespace kvx

extern "C" kv_status kv_append_scaled(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k,
                                      const kv_rows *v, const kv_page_scales *scales, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::append_scaled(cache, layer, batch, k, v, scales, static_cast<hipStream_t>(stream));
    });
}
