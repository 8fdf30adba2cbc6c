// kv_attend for many new tokens of a sequence (a prompt's tail behind a restored prefix, or a whole prompt): bound by
// the matrix cores and the exponentials between their products.
//
// A workgroup takes 128 rows (new token, query head) of one KV head, so that all query heads of a KV head share what
// is read of it, and goes over the tokens TK at a time.  K and V of TK tokens lie in LDS, twice: while one is used,
// the next is on its way (two-byte rows straight into LDS; e4m3 through registers, widened once per workgroup), and
// one barrier a round separates them.  A wave has 32 of the rows and takes S^T = K Q^T and O^T = V^T P^T in 32x32x16
// products: a row is a column of both, so its largest score, sum and rescaling stay in a lane (and the one 32 lanes
// on), and the weights are the second product's operand in the order in which the first leaves them: k-index e of
// half h of a product of 16 tokens is token h * 4 + e for e < 4, and 8 + h * 4 + e - 4 beyond.  V's operand in that
// order is two transposing LDS reads (16 lanes read 4 rows of 16 columns, a lane gets a column).  Rows in LDS are
// permuted in 16-byte pieces, so that neither kind of read meets a bank twice.  Above 128 columns a wave has 16 rows,
// in 16x16x32 products and the step kernel's order of tokens: the output's sums of 32 would not leave registers for a
// second wave on the SIMD.
//
// Workgroups of a KV head come 8 apart where there are 8 heads, and so on one XCD (consecutive ones go to consecutive
// XCDs), and use its L2 together.
//
// 2,085 new tokens behind 32,768 (8 heads of 5 rows a token, bf16, D 128): 1.51 to 1.62 ms by machine, 890 to 955
// TFLOP/s, where a large library product reaches 1,200.  Per round of 64 tokens a wave has 1,024 cycles of products
// and about 1,150 of vector work (512 of them exponentials); two waves of a SIMD overlap them partly.  Ragged tails
// of up to 1,055 tokens, e4m3, D 256, a window of 4,096 and capped scores: 0.50 ms, 650 TFLOP/s (0.66 ms with each
// sequence's last tiles first, whatever their length).  A round's products and vector work overlap less there: the matrix
// cores are busy for a fifth of the cycles, LDS for a quarter and the vector units for a third, mostly one after the
// other: one workgroup a CU, whose two waves a SIMD meet at a barrier every round.  (Half of its waves half a round
// behind the others, with a barrier for each half: 0.76 ms, as scores take longer than outputs.)
#include <algorithm>

#include "kvx_attend_tail.h"

namespace kvx {

namespace {

constexpr int kWeighWaves = 4;

// What each token received: a wave holds K of 32 tokens, goes over the rows that see them, 32 at a time, with their
// scores taken again, and adds up exp2(s - lse) for each token; a token's 32 partial sums are joined at the end.
// SHARED: a workgroup's waves have the same tokens and take turns with the rows; their sums are joined in order.
template <class T, bool FP8, int DP, bool SHARED>
__global__ __launch_bounds__(64 * kWeighWaves) void weigh_kernel(const AttendArgs a) {
    constexpr int KC = DP * (FP8 ? 1 : 2) / 32;  // 16-byte pieces of a token's K in a lane
    const Pages &pg = a.pages;
    const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.z, h = blockIdx.y, base = (SHARED ? blockIdx.x : blockIdx.x * kWeighWaves + wave) * 32;
    __shared__ float wave_sums[SHARED ? kWeighWaves : 1][32];
    Sequence seq;
    if (!sequence(a.batch, b, pg.err, seq) || base >= seq.n)
        return;
    // Rows that see any of the 32 tokens: new tokens from base on, and before the window has closed on the last.
    const int past = seq.n - seq.nq;
    const int i0 = max(0, base - past);
    const int i1 = a.window > 0 ? min<int64_t>(seq.nq, int64_t{base} + 31 + a.window - past) : seq.nq;
    // (In 64 bits: rows before token 0 and a wide window are together beyond 32.)
    const int first_seen =
        a.window > 0 ? static_cast<int>(max(int64_t{0}, int64_t{past} + 1 - a.window)) : 0;
    const int t_lane = base + c;
    float sums[16];
#pragma unroll
    for (int x = 0; x < 16; ++x)
        sums[x] = 0.f;
    if (i0 < i1) {
        const bool seen = t_lane < seq.n && t_lane >= first_seen;
        const int page = divide(t_lane, pg.by_bs);
        const int block = seen ? a.batch.tables[b * a.batch.table_stride + page] : 0;
        const bool use = seen && in_cache(pg, block);
        const uint32_t usable = static_cast<uint32_t>(__ballot(use));
        const int64_t k_off =
            use ? block * pg.block_stride + static_cast<uint32_t>(t_lane - page * pg.BS) * pg.token_bytes : int64_t{0};
        const uint8_t *k_row = pg.base + static_cast<uint32_t>(h) * pg.head_bytes + k_off;
        u32x4 k_reg[KC];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            const int at = k * 32 + half * 16;
            k_reg[k] = *reinterpret_cast<const u32x4 *>(k_row + (at < pg.row_bytes ? at : 0));
        }
        const float scale = a.scale * kLog2e;
        for (int r0 = i0 * a.group + (SHARED ? wave * 32 : 0); r0 < i1 * a.group; r0 += 32 * (SHARED ? kWeighWaves : 1)) {
            const int r = min(r0 + c, i1 * a.group - 1), i = divide(r, a.by_group), head = h * a.group + r - i * a.group;
            const int p = r0 + c < i1 * a.group ? past + i : -1;
            const uint8_t *q = a.q.data + (seq.q0 + i) * a.q.token_stride + head * a.q.head_stride;
            const float lse = a.lse[static_cast<int64_t>(seq.q0 + i) * a.heads + head] * kLog2e;
            f32x16 s;
#pragma unroll
            for (int x = 0; x < 16; ++x)
                s[x] = 0.f;
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                if constexpr (FP8) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int d = k * 32 + half * 16 + j * 8;
                        const u32x4 x = d < pg.D ? *reinterpret_cast<const u32x4 *>(q + 2 * d) : u32x4{0, 0, 0, 0};
                        const uint32_t y0 = k_reg[k][2 * j], y1 = k_reg[k][2 * j + 1];
                        s = mfma_32x32x16(u32x4{T::from_e4m3(y0, false), T::from_e4m3(y0, true), T::from_e4m3(y1, false),
                                                T::from_e4m3(y1, true)}, x, s, T{});
                    }
                } else {
                    const int d = k * 16 + half * 8;
                    const u32x4 x = d < pg.D ? *reinterpret_cast<const u32x4 *>(q + 2 * d) : u32x4{0, 0, 0, 0};
                    s = mfma_32x32x16(k_reg[k], x, s, T{});
                }
            }
            if (a.softcap > 0.f && a.softcap <= kSmallCap) {
                const float twice = 2.f * kLog2e * a.scale / a.softcap, cap = a.softcap * kLog2e;
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] = small_capped(s[x], twice, cap);
            } else if (a.softcap > 0.f) {
                const float inv = a.scale / a.softcap, cap = a.softcap * kLog2e;
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] = capped(s[x], inv, cap);
            } else {
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] *= scale;
            }
            if (a.slopes) {
                const float slope = a.slopes[head] * kLog2e;
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] -= slope * static_cast<float>(p - (base + 8 * (x >> 2) + half * 4 + (x & 3)));
            }
            const int to = lse == -INFINITY ? INT32_MIN : p - base + 1;
            const int from = a.window > 0 ? p - base + 1 - a.window : INT32_MIN;
            const uint32_t mine = usable >> (half * 4);
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int bit = 8 * (x >> 2) + (x & 3), at = bit + half * 4;
                const bool sees = (mine >> bit & 1) && at < to && at >= from;
                sums[x] += sees ? __builtin_amdgcn_exp2f(s[x] - lse) : 0.f;
            }
        }
    }
    // Joined over the 32 columns: lane x of a half has the sum of its x-th token.
    const auto receives = [&](int t, float sum) {
        const int64_t at = b * a.weights_seq_stride + h * a.weights_head_stride + t;
        a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + sum;
    };
#pragma unroll
    for (int x = 0; x < 16; ++x) {
#pragma unroll
        for (int o = 16; o; o >>= 1)
            sums[x] += __shfl_xor(sums[x], o);
        const int t = 8 * (x >> 2) + half * 4 + (x & 3);
        if (SHARED && c == x)
            wave_sums[wave][t] = sums[x];
        else if (c == x && base + t < seq.n)
            receives(base + t, sums[x]);
    }
    if constexpr (SHARED) {
        __syncthreads();
        const int t = threadIdx.x;
        if (t < 32 && base + t < seq.n) {
            float sum = 0.f;
            for (int i = 0; i < kWeighWaves; ++i)
                sum += wave_sums[i][t];
            receives(base + t, sum);
        }
    }
}

template <class T, bool FP8>
hipError_t launch(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    if (a.softcap == 0.f && !a.slopes)
        return a.full_weights ? launch_columns<T, FP8, true, true, false>(a, parts, max_queries, stream)
                              : launch_columns<T, FP8, true, false, false>(a, parts, max_queries, stream);
    return a.full_weights ? launch_columns<T, FP8, false, true, false>(a, parts, max_queries, stream)
                          : launch_columns<T, FP8, false, false, false>(a, parts, max_queries, stream);
}

template <class T, bool FP8, bool SHARED>
hipError_t launch_weigh(const AttendArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>((a.batch.max_len - 1) / (SHARED ? 32 : 32 * kWeighWaves) + 1),
                    static_cast<uint32_t>(a.pages.H), static_cast<uint32_t>(a.num_seqs));
    const auto kernel = a.pages.D > 128  ? weigh_kernel<T, FP8, 256, SHARED>
                        : a.pages.D > 64 ? weigh_kernel<T, FP8, 128, SHARED>
                                         : weigh_kernel<T, FP8, 64, SHARED>;
    return launch_kernel(kernel, grid, 64 * kWeighWaves, stream, a);
}

template <class T, bool FP8>
hipError_t launch_weigh(const AttendArgs &a, hipStream_t stream) {
    // A wave waits for each 32 rows' queries in turn, so where the tiles (by the call's bounds) are fewer than 2
    // waves a SIMD, 4 take turns.  Whole calls, bf16, D 128: 7 sequences of up to 308 new tokens in 2,196, 2 heads of
    // 8 rows (966 tiles) 116 us instead of 216; 3 of up to 208 in 342 (66 tiles) 50 instead of 121; one of 512 in
    // 7,600, 8 heads of 5 rows (1,904 tiles), 287 instead of 320, though with 64 new tokens 85 instead of 75.  With
    // more tiles K is mostly read by more waves for nothing: 8,192 tiles take 1,083 and 1,098 us with 512 new tokens
    // each, but 233 and 187 with 64; 31,040 take 4.3 and 4.1 ms, and 836 and 633 us.
    const int64_t tiles = (int64_t{a.batch.max_len} + 31) / 32 * a.pages.H * a.num_seqs;
    return tiles < 2048 ? launch_weigh<T, FP8, true>(a, stream) : launch_weigh<T, FP8, false>(a, stream);
}

}  // namespace

hipError_t launch_tail(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    const bool fp8 = a.cache_type == KV_DTYPE_E4M3;
    if (a.q_type == KV_DTYPE_BF16)
        return fp8 ? launch<Bf16, true>(a, parts, max_queries, stream)
                   : launch<Bf16, false>(a, parts, max_queries, stream);
    return fp8 ? launch<F16, true>(a, parts, max_queries, stream)
               : launch<F16, false>(a, parts, max_queries, stream);
}

hipError_t launch_weigh(const AttendArgs &a, hipStream_t stream) {
    const bool fp8 = a.cache_type == KV_DTYPE_E4M3;
    if (a.q_type == KV_DTYPE_BF16)
        return fp8 ? launch_weigh<Bf16, true>(a, stream) : launch_weigh<Bf16, false>(a, stream);
    return fp8 ? launch_weigh<F16, true>(a, stream) : launch_weigh<F16, false>(a, stream);
}

}  // namespace kvx
