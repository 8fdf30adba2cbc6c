// kv_keep: which tokens a sequence keeps under a budget, by accumulated attention weight.
//
// The heaviest m of the tokens between the sinks and the recent ones are those whose weight, as a 32-bit key that
// orders as the weights do, is above the m-th largest key, and as many of those equal to it, from the lowest token
// on, as are left.  That key is found from counts of its digits' values (a radix selection of 11, 11 and 10 bits: the
// first digit already has the exponent and two bits more, so that the counters of a wave are spread); then what every
// wave will write is counted, and the chosen tokens are written in order.
//
// One workgroup does all of that for a row whose 8,192 tokens fit its registers, and for longer rows where there are
// enough of them to fill the chip; it is bound by its own instructions (15 us for 8,192 tokens, 148 for 131,077).  A
// few long rows are cut into pieces of 8,192 tokens instead, a workgroup each, in five launches (27-29 us for 131,077
// tokens): clear the counters, a digit each, write.  For every value that the last digit may have, a piece leaves how
// many of its tokens are above it, so that the pieces behind it know where they begin to write without counting
// again.
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
    int32_t pieces;                   // of a row; 1: rows are not cut
    int32_t *digit_counts;            // [row][3][kBins]
    int32_t *states;                  // [row][2][2]: the threshold's first digits, and the tokens still to find
    int32_t *piece_counts;            // [row][pieces][kPieceCounts]: tokens with keys above each of the last digit's values
};

// Orders as the weights do; both zeros alike, every NaN 0 (below -infinity).
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, w + 0.f);
    return w != w ? 0u : bits ^ (bits >> 31 ? 0xffffffffu : 0x80000000u);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // rows start anywhere

constexpr int kRound = 4 * kKeepThreads;  // tokens that the workgroup takes at once, 4 consecutive ones a lane
constexpr int kBins = 2048, kCopies = 4;  // counters of a digit, and sets of them
constexpr int kAtOnce = 4;
constexpr int kMaxRounds = 64;            // rounds whose waves' counts are kept at once

// Sum of x over the lanes before this one, and over all.
__device__ __forceinline__ int before_in_wave(int x, int lane, int &all) {
    int sum = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(sum, o);
        sum += lane >= o ? y : 0;
    }
    all = __shfl(sum, 63);
    return sum - x;
}

// `from` and the number of `lanes` before this one.
__device__ __forceinline__ int lanes_before(uint64_t lanes, int from) {
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(lanes >> 32),
                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(lanes), from));
}

// The highest value of a digit whose tokens, with those of higher values, are `left` or more, and how many have higher
// ones.  count(value); two values a lane, from the highest down.
template <class Count>
__device__ __forceinline__ void find_digit(Count &&count, int left, int (&wave_sums)[kKeepWaves], int (&found)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, high = kBins - 1 - 2 * static_cast<int>(threadIdx.x);
    const int c0 = count(high), c1 = count(high - 1);
    int all;
    int above = before_in_wave(c0 + c1, lane, all);
    if (lane == 0)
        wave_sums[wave] = all;
    __syncthreads();
    for (int i = 0; i < wave; ++i)
        above += wave_sums[i];
    if (above < left && above + c0 + c1 >= left) {
        const bool second = above + c0 < left;
        found[0] = high - second;
        found[1] = above + (second ? c0 : 0);
    }
    __syncthreads();
}

constexpr int kWhole = -1, kWrite = 3;  // steps; 0 to 2: digits
constexpr int kPiece = 2 * kRound;
constexpr int kLastBins = 1024, kPieceCounts = kLastBins + 1;

constexpr int shift_of(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
constexpr uint32_t mask_of(int digit) { return digit < 2 ? kBins - 1 : kLastBins - 1; }

// ROUNDS: keys of so many rounds stay in registers; 0: none.  STEP: everything of a row, or one step of a piece of it.
template <int ROUNDS, int STEP>
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(const KeepArgs a) {
    __shared__ int counts[kCopies][kBins];
    __shared__ int wave_sums[kKeepWaves];
    __shared__ int found[2];
    __shared__ int of_wave[kMaxRounds * kKeepWaves][2];  // chosen outright, and ties, of each wave in each round
    const int h = blockIdx.x, b = blockIdx.y, piece = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = a.lens[b], origin = piece * kPiece;
    const int64_t row = static_cast<int64_t>(b) * a.heads + h;
    int32_t *keep = a.keep + row * a.budget;
    float *kept_weights = a.kept_weights ? a.kept_weights + row * a.budget : nullptr;
    if (n < 0 || n > a.max_len) {
        if (tid == 0)
            report(a.err, KV_ASYNC_BAD_BATCH);
        return;
    }
    const float *w = a.weights + b * a.seq_stride + h * a.head_stride;
    if constexpr (STEP == kWhole || STEP == kWrite) {
        const int kept = min(n, a.budget), lanes = kKeepThreads * a.pieces;
        if (h == 0 && piece == 0 && tid == 0)
            a.kept_lens[b] = kept;
        for (int j = kept + piece * kKeepThreads + tid; j < a.budget; j += lanes) {
            keep[j] = -1;
            if (kept_weights)
                kept_weights[j] = 0.f;
        }
        if (n <= a.budget)
            for (int j = piece * kKeepThreads + tid; j < n; j += lanes) {
                keep[j] = j;
                if (kept_weights)
                    kept_weights[j] = w[j];
            }
    }
    if (n <= a.budget || origin >= n)
        return;
    const int rounds = STEP == kWhole ? (n - 1) / kRound + 1 : min(ROUNDS, (n - 1 - origin) / kRound + 1);
    const int first = a.sinks, last = n - a.recent;  // chosen by weight: tokens [first, last)
    int left = a.budget - a.sinks - a.recent;        // tokens still to find at or below the digits known

    struct Keys {
        uint32_t k[4];
    };
    // The row's 4 tokens from t on, or its last 4 where there are not so many; then their keys (0 beyond the row).
    // The load does not depend on where it is, so many can be on their way.
    const int last4 = max(n - 4, 0);
    const auto load = [&](int t) {
        if (n >= 4)
            return static_cast<f32x4>(*reinterpret_cast<const f32x4_any *>(w + min(t, last4)));
        return f32x4{w[0], w[min(1, n - 1)], w[min(2, n - 1)], w[n - 1]};
    };
    const auto keys_of = [&](f32x4 y, int t) {
        Keys x;
        if (t > last4 || n < 4) {
            const int skip = n < 4 ? t : t - last4;  // 4 or more: nothing is left
            f32x4 z = y;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                z[j] = skip + j == 0 ? y[0] : skip + j == 1 ? y[1] : skip + j == 2 ? y[2] : y[3];
            y = z;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            x.k[j] = key_of(y[j]);
        return x;
    };
    Keys keys[ROUNDS ? ROUNDS : 1];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
        keys[i] = keys_of(load(origin + i * kRound + tid * 4), origin + i * kRound + tid * 4);
    // f(round, first token, its 4 keys) for the rounds [from, to) of the row.
    const auto each = [&](int from, int to, auto &&f) {
        if constexpr (ROUNDS > 0) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i)
                if (i >= from && i < to)
                    f(i, origin + i * kRound + tid * 4, keys[i]);
        } else {
            // kAtOnce rounds are on their way (64 KiB) while as many are used.
            f32x4 next[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                next[j] = load((from + j) * kRound + tid * 4);
            for (int i = from; i < to; i += kAtOnce) {
                f32x4 x[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    x[j] = next[j];
                    next[j] = load((i + kAtOnce + j) * kRound + tid * 4);
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (i + j < to)
                        f(i + j, (i + j) * kRound + tid * 4, keys_of(x[j], (i + j) * kRound + tid * 4));
            }
        }
    };

    const int middle = last - first;
    const auto inside = [&](int t) { return static_cast<uint32_t>(t - first) < static_cast<uint32_t>(middle); };
    int *mine = counts[wave & (kCopies - 1)];
    uint32_t threshold = 0, known = 0;  // the digits found so far, and their mask
    const bool any = left > 0;
    // Counts the values of a digit among the tokens whose digits before it are the threshold's.
    const auto count_digit = [&](int digit) {
        for (int j = tid; j < kCopies * kBins; j += kKeepThreads)
            counts[0][j] = 0;
        __syncthreads();
        each(0, rounds, [&](int, int t, const Keys &x) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!inside(t + j) || ((x.k[j] ^ threshold) & known) != 0)
                    continue;
                // (One counter for a whole wave, as among equal weights, is raised once.)
                const int bin = static_cast<int>(x.k[j] >> shift_of(digit) & mask_of(digit));
                const int one = __builtin_amdgcn_readfirstlane(bin);
                const uint64_t lanes = __ballot(true);
                if (__ballot(bin == one) != lanes)
                    atomicAdd(&mine[bin], 1);
                else if (lane == __builtin_ctzll(lanes))
                    atomicAdd(&mine[bin], __popcll(lanes));
            }
        });
        __syncthreads();
    };
    const auto counted = [&](int value) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kCopies; ++j)
            c += counts[j][value];
        return c;
    };
    // Adds a digit to the threshold.
    const auto find = [&](int digit, auto &&count) {
        find_digit(count, left, wave_sums, found);
        threshold |= static_cast<uint32_t>(found[0]) << shift_of(digit);
        known |= mask_of(digit) << shift_of(digit);
        left -= found[1];
    };
    int32_t *digit_counts = a.digit_counts + row * 3 * kBins, *states = a.states + row * 4;
    int32_t *piece_counts = a.piece_counts + (row * a.pieces + piece) * kPieceCounts;
    if constexpr (STEP == kWhole) {
        for (int digit = 0; any && digit < 3; ++digit) {
            count_digit(digit);
            find(digit, counted);
        }
    } else if (any && STEP > 0) {
        if constexpr (STEP > 1) {
            threshold = static_cast<uint32_t>(states[2 * (STEP - 2)]);
            left = states[2 * (STEP - 2) + 1];
            known = ~0u << shift_of(STEP - 2);
        }
        find(STEP - 1, [&](int value) { return digit_counts[(STEP - 1) * kBins + value]; });
        if (STEP < kWrite && piece == 0 && tid == 0) {
            states[2 * (STEP - 1)] = static_cast<int32_t>(threshold);
            states[2 * (STEP - 1) + 1] = left;
        }
    }
    if constexpr (STEP >= 0 && STEP < kWrite) {
        if (!any)
            return;
        count_digit(STEP);
        for (int value = tid; value <= static_cast<int>(mask_of(STEP)); value += kKeepThreads) {
            const int c = counted(value);
            if (c > 0)
                atomicAdd(&digit_counts[STEP * kBins + value], c);
        }
        if constexpr (STEP == 2) {
            // What the pieces behind this one will want to know of it, whatever the last digit turns out to be: the
            // tokens with keys above (the threshold's first digits, value - 1), for each value and one more.
            int above = 0, all;
            each(0, rounds, [&](int, int t, const Keys &x) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    above += inside(t + j) && (x.k[j] & known) > threshold;
            });
            for (int o = 32; o; o >>= 1)
                above += __shfl_xor(above, o);
            const int value = kLastBins - 1 - tid, c = counted(value), higher = before_in_wave(c, lane, all);
            if (lane == 0)
                wave_sums[wave] = all + (above << 16);
            __syncthreads();
            int sum = higher + c, above_all = 0;
            for (int i = 0; i < kKeepWaves; ++i) {
                sum += i < wave ? wave_sums[i] & 0xffff : 0;
                above_all += wave_sums[i] >> 16;
            }
            piece_counts[value] = above_all + sum;
            if (tid == 0)
                piece_counts[kLastBins] = above_all;
        }
        return;
    }

    // Chosen: every token outside [first, last), keys above the threshold, and the first `left` ties.
    const auto state_of = [&](int t, uint32_t key, bool &sure, bool &tie) {
        const bool is_inside = inside(t);
        sure = t < n && (!is_inside || (any && key > threshold));
        tie = any && is_inside && key == threshold;
    };
    int sure_done = 0, ties_done = 0;  // in the rounds before this set of kMaxRounds
    if constexpr (STEP == kWrite) {  // in the pieces before this one
        int s = 0, q = 0;
        for (int i = lane; any && i < piece; i += 64) {
            const int32_t *of = piece_counts + (i - piece) * kPieceCounts + (threshold & mask_of(2));
            s += of[1];
            q += of[0] - of[1];
        }
        for (int o = 32; o; o >>= 1) {
            s += __shfl_xor(s, o);
            q += __shfl_xor(q, o);
        }
        sure_done = s + min(origin, first) + max(origin - last, 0);
        ties_done = q;
    }
    for (int set = 0; set < rounds; set += kMaxRounds) {
        const int set_end = min(rounds, set + kMaxRounds);
        each(set, set_end, [&](int i, int t, const Keys &x) {
            int sure_count = 0, tie_count = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bool sure, tie;
                state_of(t + j, x.k[j], sure, tie);
                sure_count += __popcll(__ballot(sure));
                tie_count += __popcll(__ballot(tie));
            }
            if (lane == 0) {
                of_wave[(i - set) * kKeepWaves + wave][0] = sure_count;
                of_wave[(i - set) * kKeepWaves + wave][1] = tie_count;
            }
        });
        __syncthreads();
        // Sums before each wave of each round: one entry a lane, carried from wave to wave.
        const int entries = (set_end - set) * kKeepWaves;
        int s = 0, q = 0, s_all, q_all;
        if (tid < entries) {
            s = of_wave[tid][0];
            q = of_wave[tid][1];
        }
        int s_before = before_in_wave(s, lane, s_all), q_before = before_in_wave(q, lane, q_all);
        if (lane == 0) {
            wave_sums[wave] = s_all;
            counts[0][wave] = q_all;
        }
        __syncthreads();
        int s_set = 0, q_set = 0;
        for (int i = 0; i < kKeepWaves; ++i) {
            s_before += i < wave ? wave_sums[i] : 0;
            q_before += i < wave ? counts[0][i] : 0;
            s_set += wave_sums[i];
            q_set += counts[0][i];
        }
        if (tid < entries) {
            of_wave[tid][0] = s_before + sure_done;
            of_wave[tid][1] = q_before + ties_done;
        }
        sure_done += s_set;
        ties_done += q_set;
        __syncthreads();
        each(set, set_end, [&](int i, int t, const Keys &x) {
            bool sure[4], tie[4];
            const int(&before)[2] = of_wave[(i - set) * kKeepWaves + wave];
            int sure_before = before[0], ties_before = before[1];
            uint64_t lanes = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                state_of(t + j, x.k[j], sure[j], tie[j]);
                const uint64_t s_lanes = __ballot(sure[j]), t_lanes = __ballot(tie[j]);
                lanes |= s_lanes | t_lanes;
                sure_before = lanes_before(s_lanes, sure_before);
                ties_before = lanes_before(t_lanes, ties_before);
            }
            if (lanes == 0)
                return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (sure[j] || (tie[j] && ties_before < left)) {
                    const int to = sure_before + min(ties_before, left);
                    keep[to] = t + j;
                    if (kept_weights)
                        kept_weights[to] = w[t + j];
                }
                sure_before += sure[j];
                ties_before += tie[j];
            }
        });
        __syncthreads();
    }
}

__global__ __launch_bounds__(kThreads) void clear_kernel(int32_t *x, int64_t n) {
    for (int64_t i = blockIdx.x * int64_t{kThreads} + threadIdx.x; i < n; i += gridDim.x * int64_t{kThreads})
        x[i] = 0;
}

// Pieces of a row: where a few long rows would leave most CUs idle.  From 128 rows on, a workgroup a row takes about
// as long: 127 rows in pieces and 128 whole ones take 43 and 47 us (32,768 tokens), 76 and 76 (65,536), 137 and 165
// (131,072; 256 whole ones 181).
int pieces_of(int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget) {
    const int pieces = max_len > 0 ? (max_len - 1) / kPiece + 1 : 1;
    if (max_len <= 2 * kPiece || max_len <= budget || static_cast<int64_t>(num_seqs) * heads >= 128 || pieces > 65535)
        return 1;
    return pieces;
}

int64_t workspace_bytes_of(int32_t num_seqs, int32_t heads, int32_t pieces) {
    return pieces == 1 ? 0 : static_cast<int64_t>(num_seqs) * heads * (3 * kBins + 4 + int64_t{kPieceCounts} * pieces) * 4;
}

kv_status check_keep(int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget, int32_t sinks, int32_t recent) {
    if (num_seqs < 0 || heads < 1 || max_len < 0 || budget < 1 || sinks < 0 || recent < 0)
        return fail(KV_EINVAL, "num_seqs, max_len, sinks and recent must not be negative, heads and budget positive "
                    "(num_seqs %d, heads %d, max_len %d, budget %d, sinks %d, recent %d)", num_seqs, heads, max_len,
                    budget, sinks, recent);
    if (static_cast<int64_t>(sinks) + recent > budget)
        return fail(KV_EINVAL, "%d sinks and %d recent tokens exceed the budget of %d", sinks, recent, budget);
    if (num_seqs > 65535)
        return fail(KV_EUNSUPPORTED, "%d sequences in one call (at most 65,535)", num_seqs);
    if (max_len > INT32_MAX - (1 << 20))
        return fail(KV_EUNSUPPORTED, "sequences of up to %d tokens (at most 2^31 - 2^20)", max_len);
    return KV_OK;
}

kv_status keep(const float *weights, int64_t seq_stride, int64_t head_stride, const int32_t *lens, int32_t num_seqs,
               int32_t heads, int32_t max_len, int32_t budget, int32_t sinks, int32_t recent, int32_t *keep,
               int32_t *kept_lens, float *kept_weights, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    kv_status st = check_keep(num_seqs, heads, max_len, budget, sinks, recent);
    if (st != KV_OK)
        return st;
    if (seq_stride < 0 || head_stride < 0)
        return fail(KV_EINVAL, "strides must not be negative");
    if (num_seqs == 0)
        return KV_OK;
    if (!lens || !keep || !kept_lens || (!weights && max_len > 0))
        return fail(KV_EINVAL, "weights, lens, keep and kept_lens must not be NULL");
    const int pieces = pieces_of(num_seqs, heads, max_len, budget);
    const int64_t need = workspace_bytes_of(num_seqs, heads, pieces);
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(KV_EINVAL, "workspace of %lld bytes; %lld are needed", static_cast<long long>(workspace_bytes),
                    static_cast<long long>(need));
    if (reinterpret_cast<uintptr_t>(workspace) % 4 != 0)
        return fail(KV_EUNSUPPORTED, "workspace is not 4-byte aligned");
    int32_t *err = nullptr;
    st = error_word(&err);
    if (st != KV_OK)
        return st;
    int32_t *digits = static_cast<int32_t *>(workspace);
    const int64_t rows = static_cast<int64_t>(num_seqs) * heads, digit_words = rows * 3 * kBins;
    int32_t *states = need > 0 ? digits + digit_words : nullptr;
    const KeepArgs a{weights, seq_stride, head_stride, lens, heads, max_len, budget, sinks, recent, keep, kept_lens,
                     kept_weights, err, pieces, digits, states, states ? states + rows * 4 : nullptr};
    const dim3 grid(static_cast<uint32_t>(heads), static_cast<uint32_t>(num_seqs), static_cast<uint32_t>(pieces));
    const auto launch = [&](void (*kernel)(KeepArgs)) { return launch_kernel(kernel, grid, kKeepThreads, stream, a); };
    if (pieces > 1) {
        const uint32_t clear = static_cast<uint32_t>(std::min<int64_t>((digit_words + kThreads - 1) / kThreads, 1024));
        KVX_HIP(launch_kernel(clear_kernel, dim3(clear), kThreads, stream, digits, digit_words));
        KVX_HIP(launch(keep_kernel<2, 0>));
        KVX_HIP(launch(keep_kernel<2, 1>));
        KVX_HIP(launch(keep_kernel<2, 2>));
        KVX_HIP(launch(keep_kernel<2, kWrite>));
    } else {
        KVX_HIP(launch(max_len <= 2 * kRound ? keep_kernel<2, kWhole> : keep_kernel<0, kWhole>));
    }
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" {

int64_t kv_keep_workspace(int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget) {
    const kv_status st =
        kvx::guarded([&]() -> kv_status { return kvx::check_keep(num_seqs, heads, max_len, budget, 0, 0); });
    return st == KV_OK ? kvx::workspace_bytes_of(num_seqs, heads, kvx::pieces_of(num_seqs, heads, max_len, budget)) : st;
}

kv_status kv_keep(const float *weights, int64_t seq_stride, int64_t head_stride, const int32_t *lens, int32_t num_seqs,
                  int32_t heads, int32_t max_len, int32_t budget, int32_t sinks, int32_t recent, int32_t *keep,
                  int32_t *kept_lens, float *kept_weights, void *workspace, int64_t workspace_bytes, void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::keep(weights, seq_stride, head_stride, lens, num_seqs, heads, max_len, budget, sinks, recent, keep,
                         kept_lens, kept_weights, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
