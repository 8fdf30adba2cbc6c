// kv_attend for few new tokens per sequence (a decoding step): bound by reading the cache.
//
// A KV head's rows (its query heads times the new tokens, up to 16 or 32 of them at a time) share one pass over K and
// V. Per 32 tokens a wave takes the scores as K Q^T and the output as V^T P^T on the matrix cores (16x16x32): then a
// row is a column of both results, and its largest score, sum and rescaling stay inside a lane.
//
//  * K's operand wants a token's consecutive elements per lane: 16-byte loads straight into registers.  Its 32 tokens
//    are given to the two products' rows in the order in which the second product wants them: row m of product j is
//    token (m / 4) * 8 + j * 4 + m % 4, so that a lane's 8 scores are those of 8 consecutive tokens, and their weights
//    are the operand of the second product as they stand.  Nothing passes through LDS.
//  * V's operand wants 8 consecutive tokens of one column per lane.  A lane loads 8 rows of VE columns, and byte
//    permutations in registers turn them (one per pair of elements); e4m3 is turned while it is widened.
//  * The pages of 32 tokens are looked up by 32 lanes, one token each, a round ahead, and handed out by lane shuffles.
//
// The sequences' tokens are shared out to workgroups (Shares) so that they fill the chip evenly, and inside a
// workgroup over its 4 waves; the waves' sums are joined through LDS, the workgroups' by join_kernel.  K of the next
// 32 tokens is requested as soon as the scores have used the last, V as soon as the second product has: a wave has 16
// KiB in flight (bf16, D 128) without a second set of registers, and 2 waves of a SIMD 128 KiB a CU.
//
// One sequence behind 131,077 tokens (8 heads of 5 rows, bf16, D 128): 95 us and 6 to join, 5.3 TB/s with both (a
// large reduction reads 6.1, a large copy moves 4.8).  16 sequences of up to 32,768 tokens in e4m3 (4 heads of 6
// rows, D 256): 114 us and 6 to join, 4.9 TB/s.  48 of up to 8,192 with weights (2 heads of 8 rows): 52 us (209 MB of
// K and V read, 13 MB of scores written), 6 to join, 7 for what each token received.
#include <algorithm>

#include "kvx_attend_step.h"

namespace kvx {

namespace {

// The lists of Shares, by one workgroup.
__global__ __launch_bounds__(1024) void share_kernel(const AttendArgs a, const Shares shares) {
    __shared__ int64_t wave_sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const auto sum = [&](int64_t x) {
        x = sum_of_wave(x);
        __syncthreads();
        if (lane == 0)
            wave_sums[wave] = x;
        __syncthreads();
        x = 0;
        for (int i = 0; i < 16; ++i)
            x += wave_sums[i];
        return x;
    };
    bool told = false;
    const auto each = [&](auto &&f) {
        for (int b = tid; b < shares.num_seqs; b += 1024) {
            bool rows;
            const int tokens = share_tokens(a, b, !told, rows);
            f(tokens, rows);
        }
        told = true;
    };
    const int len = share_len(shares, each, sum);
    int32_t *seqs = shares.items_of + 2, *items = seqs + 2 * static_cast<int64_t>(shares.num_seqs);
    int base = 0;
    for (int b0 = 0; b0 < shares.num_seqs; b0 += 1024) {
        const int b = b0 + tid;
        bool rows = false;
        const int tokens = b < shares.num_seqs ? share_tokens(a, b, false, rows) : 0;
        const int mine = share_parts(tokens, rows, len), upto = sum_up_to_lane(mine);
        __syncthreads();
        if (lane == 63)
            wave_sums[wave] = upto;
        __syncthreads();
        int from = base + upto - mine;
        for (int i = 0; i < 16; ++i) {
            from += i < wave ? static_cast<int>(wave_sums[i]) : 0;
            base += static_cast<int>(wave_sums[i]);
        }
        if (b < shares.num_seqs) {
            seqs[2 * b] = from;
            seqs[2 * b + 1] = mine;
        }
        for (int k = 0; k < mine; ++k) {
            items[2 * (from + k)] = b;
            items[2 * (from + k) + 1] = k;
        }
    }
    for (int i = base + tid; i < shares.items; i += 1024)
        items[2 * i] = -1;
    if (tid == 0)
        shares.items_of[0] = len;
}

// Where the parts of a row lie.
struct Row {
    int64_t slot, stride;  // of its first part, and between parts
    int parts;
};

// Row i of head h's sequence b, or no parts.
__device__ __forceinline__ Row parts_at(const AttendArgs &a, const Shares &from, int b, int h, int r, const Sequence &) {
    Share share;
    if (!share_of(a, from, b, true, share))
        return Row{0, 0, 0};
    return Row{(static_cast<int64_t>(h) * from.items + share.item0) * from.row_cap + r, from.row_cap, share.parts};
}
__device__ __forceinline__ Row parts_at(const AttendArgs &a, const Parts &from, int, int h, int r, const Sequence &seq) {
    const int rows = seq.nq * a.group, row0 = r - r % kTailRows;
    if (rows <= a.tail_above)
        return Row{0, 0, 0};
    const Span span = span_of(seq.n, seq.nq, divide(row0, a.by_group),
                              divide(min(row0 + kTailRows, rows) - 1, a.by_group) + 1, a.window);
    const int i = divide(r, a.by_group), head = h * a.group + r - i * a.group;
    return Row{(static_cast<int64_t>(seq.q0 + i) * a.heads + head) * from.splits, 1, parts_of(span, from.len)};
}

__device__ __forceinline__ Row parts_at(const AttendArgs &a, const Chosen &from, int, int h, int r, const Sequence &seq) {
    if (seq.nq == 0)
        return Row{0, 0, 0};
    const int i = divide(r, a.by_group), head = h * a.group + r - i * a.group;
    return Row{(static_cast<int64_t>(seq.q0 + i) * a.heads + head) * from.splits, 1,
               max(chosen_parts(a, from, from.counts[seq.q0 + i]), 0)};
}

// The parts of a row joined: sum_s 2^(m_s - m) x_s / sum_s 2^(m_s - m) l_s.  4 columns per lane; a workgroup takes one
// row and spreads its parts over its lanes' groups (SPREAD: many parts, few rows), or a row per group of lanes.
template <bool SPREAD, class From>
__global__ __launch_bounds__(256) void join_kernel(const AttendArgs a, const From from) {
    __shared__ f32x4 sums[SPREAD ? 256 : 1];
    const int b = blockIdx.z, head = blockIdx.y, h = divide(head, a.by_group), D = a.pages.D, tid = threadIdx.x;
    const int lanes = D / 4, groups = 256 / lanes, mine = tid / lanes, d = (tid - mine * lanes) * 4;
    const int i = SPREAD ? blockIdx.x : blockIdx.x * groups + mine;
    Sequence seq;
    if (!sequence(a.batch, b, a.pages.err, seq) || (SPREAD && i >= seq.nq))
        return;
    // (All lanes look the parts up together; the lanes of a row that is none then leave.)
    const Row row_at = parts_at(a, from, b, h, min(i, max(seq.nq - 1, 0)) * a.group + head - h * a.group, seq);
    const int parts = row_at.parts;
    const bool row = i < seq.nq && mine < groups;
    if (parts <= 1 || (!SPREAD && !row))
        return;
    const float *stats = from.stats + row_at.slot * 2;
    const int64_t step = row_at.stride;
    float most = kLowest, total = 0.f;
    // (A lane's first parts are on their way together, their sums while the row's largest score is looked for.)
    constexpr int EARLY = SPREAD ? 8 : 4;
    const int s0 = SPREAD ? mine : 0, ds = SPREAD ? groups : 1;
    struct Sums {
        f32x4 x[EARLY];
        float most[EARLY];
    };
    const auto load = [&](int first) {
        Sums sums_of;
#pragma unroll
        for (int k = 0; k < EARLY; ++k) {
            const int s = first + k * ds;
            const bool is = row && s < parts;
            sums_of.x[k] = is ? *reinterpret_cast<const f32x4 *>(from.sums + (row_at.slot + s * step) * D + d)
                              : f32x4{0.f, 0.f, 0.f, 0.f};
            sums_of.most[k] = is ? stats[2 * s * step] : kLowest;
        }
        return sums_of;
    };
    constexpr int HELD = 4;  // statistics that a lane keeps
    const int t0 = SPREAD ? tid & 63 : 0, dt = SPREAD ? 64 : 1;
    f32x2 held[HELD];
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        const int s = t0 + k * dt;
        held[k] = s < parts ? *reinterpret_cast<const f32x2 *>(stats + 2 * s * step) : f32x2{kLowest, 0.f};
    }
    const Sums early = load(s0);
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        most = fmaxf(most, held[k][0]);
    for (int s = t0 + HELD * dt; s < parts; s += dt)
        most = fmaxf(most, stats[2 * s * step]);
    if constexpr (SPREAD)  // every wave for itself
        for (int o = 32; o; o >>= 1)
            most = fmaxf(most, __shfl_xor(most, o));
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        total += held[k][1] * __builtin_amdgcn_exp2f(held[k][0] - most);
    for (int s = t0 + HELD * dt; s < parts; s += dt)
        total += stats[2 * s * step + 1] * __builtin_amdgcn_exp2f(stats[2 * s * step] - most);
    if constexpr (SPREAD)
        for (int o = 32; o; o >>= 1)
            total += __shfl_xor(total, o);
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    const auto add = [&](const Sums &sums_of) {
#pragma unroll
        for (int k = 0; k < EARLY; ++k)
            x += sums_of.x[k] * __builtin_amdgcn_exp2f(sums_of.most[k] - most);
    };
    add(early);
    if (row)
        for (int s = s0 + EARLY * ds; s < parts; s += EARLY * ds)
            add(load(s));
    if constexpr (SPREAD) {
        sums[tid] = x;
        __syncthreads();
        if (mine > 0)
            return;
        for (int s = 1; s < groups; ++s)
            x += sums[s * lanes + tid];
    }
    const float inv = total == 0.f ? 0.f : a.v_scale / total;
    u32x2 y;
    if (a.q_type == KV_DTYPE_BF16)
        y = u32x2{Bf16::pack(x[0] * inv, x[1] * inv), Bf16::pack(x[2] * inv, x[3] * inv)};
    else
        y = u32x2{F16::pack(x[0] * inv, x[1] * inv), F16::pack(x[2] * inv, x[3] * inv)};
    *reinterpret_cast<u32x2 *>(a.out.data + (seq.q0 + i) * a.out.token_stride + head * a.out.head_stride + 2 * d) = y;
    if (d == 0)
        a.lse[static_cast<int64_t>(seq.q0 + i) * a.heads + head] =
            total == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(total)) * kLn2;
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // weights' rows start anywhere

// What each token received from the rows of a sequence, from the scores that the step kernel left; 4 tokens a lane.
__global__ __launch_bounds__(256) void weigh_step_kernel(const AttendArgs a) {
    const int b = blockIdx.z, h = blockIdx.y, t = (blockIdx.x * 256 + threadIdx.x) * 4;
    Sequence seq;
    if (!sequence(a.batch, b, a.pages.err, seq) || t >= seq.n)
        return;
    const int64_t at = b * a.weights_seq_stride + h * a.weights_head_stride + t;
    const bool all = seq.n - t >= 4;
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
    if (a.weights_in) {
        if (all) {
            sum = *reinterpret_cast<const f32x4_any *>(a.weights_in + at);
        } else {
            for (int j = 0; j < seq.n - t; ++j)
                sum[j] = a.weights_in[at + j];
        }
    }
    f32x4 got{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < seq.nq; ++i) {
        // Of these tokens the row sees [from, to); others' scores may not be there.
        const int p = seq.n - seq.nq + i, to = p - t + 1, from = a.window > 0 ? to - a.window : INT32_MIN;
        if (to <= 0 || from >= 4)
            continue;
        const float *lse = a.lse + static_cast<int64_t>(seq.q0 + i) * a.heads + h * a.group;
        const int64_t slot = (static_cast<int64_t>(b) * a.pages.H + h) * a.score_cap + i * a.group;
        const float *scores = a.scores + slot * a.score_len + t;
        for (int k = 0; k < a.group; ++k) {
            const float zero = lse[k] * kLog2e;
            const f32x4 x = *reinterpret_cast<const f32x4 *>(scores + k * a.score_len);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                got[j] += j < to && j >= from && lse[k] != -INFINITY ? __builtin_amdgcn_exp2f(x[j] - zero) : 0.f;
        }
    }
    sum += got;
    if (all) {
        *reinterpret_cast<f32x4_any *>(a.weights_out + at) = sum;
    } else {
        for (int j = 0; j < seq.n - t; ++j)
            a.weights_out[at + j] = sum[j];
    }
}

template <bool SPREAD, class From>
hipError_t launch_join(const AttendArgs &a, const From &from, int max_queries, hipStream_t stream) {
    const int groups = SPREAD ? 1 : 256 / (a.pages.D / 4);
    const dim3 grid(static_cast<uint32_t>((max_queries + groups - 1) / groups), static_cast<uint32_t>(a.heads),
                    static_cast<uint32_t>(a.num_seqs));
    return launch_kernel(join_kernel<SPREAD, From>, grid, 256, stream, a, from);
}

}  // namespace

hipError_t launch_share(const AttendArgs &a, const Shares &shares, hipStream_t stream) {
    return launch_kernel(share_kernel, dim3(1), 1024, stream, a, shares);
}

hipError_t launch_step(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream) {
    const int max_rows = static_cast<int>(std::min<int64_t>(a.step_rows, static_cast<int64_t>(max_queries) * a.group));
    const bool fp8 = a.cache_type == KV_DTYPE_E4M3;
    if (a.q_type == KV_DTYPE_BF16)
        return fp8 ? launch_rows<Bf16, true, false>(a, shares, shares.items, max_rows, stream)
                   : launch_rows<Bf16, false, false>(a, shares, shares.items, max_rows, stream);
    return fp8 ? launch_rows<F16, true, false>(a, shares, shares.items, max_rows, stream)
               : launch_rows<F16, false, false>(a, shares, shares.items, max_rows, stream);
}

hipError_t launch_join_step(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream) {
    const int most = std::min(max_queries, std::max(a.step_rows / a.group, 1));
    const int64_t rows = int64_t{most} * a.heads * a.num_seqs;
    return a.scales.data && shares.most <= 8 && rows >= 1024 ? launch_join<false>(a, shares, most, stream)
                                            : launch_join<true>(a, shares, most, stream);
}

hipError_t launch_join_tail(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    // (8 parts one after the other take about as long as one row's launch.)
    return parts.splits > 8 ? launch_join<true>(a, parts, max_queries, stream)
                            : launch_join<false>(a, parts, max_queries, stream);
}

hipError_t launch_join_pages(const AttendArgs &a, const Chosen &chosen, int max_queries, hipStream_t stream) {
    return chosen.splits > 8 ? launch_join<true>(a, chosen, max_queries, stream)
                             : launch_join<false>(a, chosen, max_queries, stream);
}

hipError_t launch_weigh_step(const AttendArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>((a.batch.max_len + 1023) / 1024), static_cast<uint32_t>(a.pages.H),
                    static_cast<uint32_t>(a.num_seqs));
    return launch_kernel(weigh_step_kernel, grid, 256, stream, a);
}

}  // namespace kvx
