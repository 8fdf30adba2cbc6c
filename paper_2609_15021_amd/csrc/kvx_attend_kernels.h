// What the kernels of kv_attend share.
#pragma once

#include "kvx_paged.h"

namespace kvx {

// Rows of a workgroup of the tail kernel.
constexpr int kTailRows = 128;
inline int64_t tail_tiles(int64_t max_queries, int64_t group) {
    return (max_queries * group + kTailRows - 1) / kTailRows;
}

// Sequences of at most this many (new token, query head) rows per KV head go to the step kernel, others to the tail
// one.
constexpr int kStepRows = 64;

struct AttendArgs {
    Pages pages;
    Batch batch;
    Rows q, out;
    float *lse;  // never NULL (the caller's or the workspace's)
    const float *slopes, *weights_in;
    float *weights_out;
    int64_t weights_seq_stride, weights_head_stride;
    float scale, softcap, v_scale;  // scale: with k_scale
    int32_t window, heads, group, num_seqs;
    Divisor by_group;
    int32_t q_type, cache_type;
    int32_t full_weights;
    float *scores;  // [sequence][KV head][score_cap][score_len] in powers of 2, for weights_out; or NULL
    int64_t score_len;
    int32_t score_cap;
};

// How the tail kernel splits the tokens of a tile of rows over workgroups, and what the parts of a row leave for the
// join.
struct Parts {
    int32_t len, splits;  // tokens of a part; most parts of a row
    float *sums;          // [row][query head][splits][D], unscaled
    float *stats;         // [row][query head][splits][2]: largest score and sum, in powers of 2
};

// Tokens that the new tokens [i0, i1) of a sequence see between them: [first, end); parts start at `start`.
struct Span {
    int first, start, end;
};

__host__ __device__ __forceinline__ Span span_of(int n, int nq, int i0, int i1, int window) {
    const int p0 = n - nq + i0;
    Span s;
    s.first = window > 0 && p0 + 1 > window ? p0 + 1 - window : 0;
    s.start = s.first & ~31;
    s.end = n - nq + i1;
    return s;
}

// Rows of a tile of the step kernel.
inline int step_tile_rows(int max_rows, int head_dim) { return max_rows > 16 && head_dim <= 128 ? 32 : 16; }

// How the step kernel shares its sequences' tokens out: in parts of one length for all, on the device, where the
// lengths are.  A long sequence among short ones is then no workgroup's alone, and the parts number about `target`,
// which fill the chip once, or three times where the sequences alone fill half of it (or twice the sequences, where
// those are more).  Up to kShareSeqs sequences every wave works out the sharing for itself; more of them are shared
// out by a kernel of its own, which leaves the lists below.
struct Shares {
    int32_t target, items, num_seqs;  // items >= the parts of any batch
    int32_t shortest;                 // tokens of a part at least
    int32_t alone;                    // every sequence is one part
    int32_t row_cap;                  // most rows per KV head of a sequence
    float *sums;                      // [KV head][item][row_cap][D], unscaled
    float *stats;                     // [KV head][item][row_cap][2]: largest score and sum, in powers of 2
    int32_t *items_of;                // NULL, or: length of a part; [sequence]: first item, parts; [item]: sequence, split
};

// A sequence's part: `split` of `parts`, `len` tokens each; its first part is item `item0`.
struct Share {
    int b, split, parts, len, item0;
};

constexpr int kShareSeqs = 64;

// Tokens of sequence b that the step kernel takes, from span.start on; 0 and no rows if none.
__device__ __forceinline__ int share_tokens(const AttendArgs &a, int b, bool tell, bool &rows) {
    const int n = a.batch.lens[b], q0 = a.batch.starts ? a.batch.starts[b] : b;
    const int q1 = a.batch.starts ? a.batch.starts[b + 1] : b + 1, nq = q1 - q0;
    const bool good = n >= 0 && n <= a.batch.max_len && q0 >= 0 && q1 >= q0 && q1 <= a.batch.num_queries &&
                      nq <= a.batch.max_queries;
    if (!good && tell)
        report(a.pages.err, KV_ASYNC_BAD_BATCH);
    rows = good && nq > 0 && nq <= kStepRows && nq * a.group <= kStepRows;
    if (!rows)
        return 0;
    const Span span = span_of(n, nq, 0, nq, a.window);
    return max(span.end - span.start, 0);
}

__device__ __forceinline__ int64_t sum_of_wave(int64_t x) {
#pragma unroll
    for (int o = 32; o; o >>= 1)
        x += __shfl_xor(x, o);
    return x;
}

__device__ __forceinline__ int sum_up_to_lane(int x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        x += lane >= o ? y : 0;
    }
    return x;
}

// Parts of sequence b at a length.
__device__ __forceinline__ int share_parts(const AttendArgs &a, int b, int64_t len) {
    bool rows;
    const int tokens = share_tokens(a, b, false, rows);
    return rows ? static_cast<int>(max((tokens + len - 1) / len, int64_t{1})) : 0;
}

// The shortest length of a part, up to a few percent, that makes no more parts than wanted.  `first` and `step`: this
// lane's sequences; sum(x): x over all lanes.
template <class Sum>
__device__ __forceinline__ int64_t share_len(const AttendArgs &a, const Shares &shares, int first, int step, bool tell,
                                             Sum &&sum) {
    const auto round_len = [&](int64_t len) { return max((len + 31) / 32 * 32, int64_t{shares.shortest}); };
    int64_t total = 0;
    for (int b = first; b < shares.num_seqs; b += step) {
        bool rows;
        total += share_tokens(a, b, tell, rows);
    }
    int64_t len = round_len((sum(total) + shares.target - 1) / shares.target);
    for (int tries = 0; tries < 4 && shares.num_seqs > 1; ++tries) {
        int64_t parts = 0;
        for (int b = first; b < shares.num_seqs; b += step)
            parts += share_parts(a, b, len);
        parts = sum(parts);
        if (parts <= max(int64_t{shares.target}, 2 * int64_t{shares.num_seqs}))
            break;
        len = round_len(len * parts / shares.target);
    }
    return min(len, int64_t{INT32_MAX});
}

// The part that is item `item`, or (by_seq) sequence `item`'s parts; false if there is none.  Every wave for itself.
__device__ __forceinline__ bool share_of(const AttendArgs &a, const Shares &shares, int item, bool by_seq, Share &s) {
    if (shares.alone) {
        s = Share{item, 0, 1, INT32_MAX, item};
        bool rows;
        share_tokens(a, item, !by_seq && blockIdx.y == 0 && threadIdx.x == 0, rows);
        return rows;
    }
    if (shares.items_of) {
        const int32_t *seqs = shares.items_of + 2, *items = seqs + 2 * static_cast<int64_t>(shares.num_seqs);
        s.b = by_seq ? item : items[2 * item];
        if (s.b < 0)
            return false;
        s.split = by_seq ? 0 : items[2 * item + 1];
        s.item0 = seqs[2 * s.b];
        s.parts = seqs[2 * s.b + 1];
        s.len = shares.items_of[0];
        return s.parts > 0;
    }
    const int lane = threadIdx.x & 63;
    const bool tell = !by_seq && item == 0 && blockIdx.y == 0 && threadIdx.x < 64;
    const int64_t len = share_len(a, shares, lane, 64, tell, sum_of_wave);
    const int mine = lane < shares.num_seqs ? share_parts(a, lane, len) : 0;
    const int from = sum_up_to_lane(mine) - mine;
    const uint64_t found = __ballot(by_seq ? lane == item : item >= from && item < from + mine);
    if (!found)
        return false;
    s.b = __builtin_ctzll(found);
    s.parts = __builtin_amdgcn_readlane(mine, s.b);
    s.item0 = __builtin_amdgcn_readlane(from, s.b);
    s.split = by_seq ? 0 : item - s.item0;
    s.len = static_cast<int>(len);
    return s.parts > 0;
}

__device__ __forceinline__ int parts_of(const Span &s, int len) {
    return s.end > s.start ? (s.end - s.start - 1) / len + 1 : 1;
}

// Two-byte element types on the matrix cores.  kShift: weights are exp2(s - m + kShift), and m is at least the largest
// score less 8: a float16 weight is at most 2^15, and its smallest normal 2^-21 or less of the largest.
struct Bf16 {
    typedef __bf16 frag __attribute__((ext_vector_type(8)));
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr float kShift = 0.f;
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t x, bool high) {
        return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true))
                    : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        pair p;
        p[0] = static_cast<__bf16>(a);
        p[1] = static_cast<__bf16>(b);
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ __forceinline__ float low(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
    static __device__ __forceinline__ float high(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
};

struct F16 {
    typedef _Float16 frag __attribute__((ext_vector_type(8)));
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr float kShift = 7.f;
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t x, bool high) {
        return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true))
                    : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        pair p;
        p[0] = static_cast<_Float16>(a);
        p[1] = static_cast<_Float16>(b);
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ __forceinline__ float low(uint32_t x) { return static_cast<float>(__builtin_bit_cast(pair, x)[0]); }
    static __device__ __forceinline__ float high(uint32_t x) { return static_cast<float>(__builtin_bit_cast(pair, x)[1]); }
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma_16x16x32(const u32x4 &a, const u32x4 &b, const f32x4 &c, Bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16::frag, a), __builtin_bit_cast(Bf16::frag, b),
                                                   c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_16x16x32(const u32x4 &a, const u32x4 &b, const f32x4 &c, F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(F16::frag, a), __builtin_bit_cast(F16::frag, b), c,
                                                  0, 0, 0);
}

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.402823466e+38f;  // the largest score of nothing (finite: its differences are numbers)

// cap * tanh(x / cap) for x * inv = x / cap: tanh by its series below 1/4 (the first term left out is 2^-27 of it),
// else from exp2; an error of 2^-23 or so of cap.
__device__ __forceinline__ float capped(float x, float inv, float cap) {
    const float y = x * inv, y2 = y * y, t = fabsf(y);
    const float series =
        y * (1.f + y2 * (-1.f / 3 + y2 * (2.f / 15 + y2 * (-17.f / 315 + y2 * (62.f / 2835)))));
    const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * t));
    return cap * (t < 0.25f ? series : copysignf(far, y));
}

// The same for caps up to kSmallCap, from exp2 alone (twice = 2 log2(e) inv): its error of 2^-22 or so of cap,
// whatever x, is then at most that of a score of 16.
constexpr float kSmallCap = 64.f;
__device__ __forceinline__ float small_capped(float x, float twice, float cap) {
    return fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * twice)), cap);
}

// Each covers the sequences of its kind only, whatever else is in the batch.
hipError_t launch_share(const AttendArgs &a, const Shares &shares, hipStream_t stream);
hipError_t launch_step(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream);
hipError_t launch_tail(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream);
// Join what these left of rows in parts.
hipError_t launch_join_step(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream);
hipError_t launch_join_tail(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream);
// weights_out, from the scores that the step kernel left, or with the scores taken again.
hipError_t launch_weigh_step(const AttendArgs &a, hipStream_t stream);
hipError_t launch_weigh(const AttendArgs &a, hipStream_t stream);

}  // namespace kvx
