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
// of up to 1,055 tokens, e4m3, D 256, a window of 4,096 and capped scores: 0.66 ms, 495 TFLOP/s; there the matrix
// cores are busy for a fifth of the cycles, LDS for a quarter and the vector units for a third, mostly one after the
// other: one workgroup a CU, whose two waves a SIMD meet at a barrier every round.  (Half of its waves half a round
// behind the others, with a barrier for each half: 0.76 ms, as scores take longer than outputs.)
#include <algorithm>
#include <type_traits>

#include "kvx_attend_kernels.h"

namespace kvx {

namespace {

constexpr int kRows = kTailRows;
constexpr int kWeighWaves = 4;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma_32x32x16(const u32x4 &a, const u32x4 &b, const f32x16 &c, Bf16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf16::frag, a), __builtin_bit_cast(Bf16::frag, b),
                                                   c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma_32x32x16(const u32x4 &a, const u32x4 &b, const f32x16 &c, F16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(F16::frag, a), __builtin_bit_cast(F16::frag, b), c,
                                                  0, 0, 0);
}

// A tile of RW x RW sums, and the product that adds to it.
template <int RW>
struct Tile;
template <>
struct Tile<32> {
    typedef f32x16 type;
};
template <>
struct Tile<16> {
    typedef f32x4 type;
};
template <class T>
__device__ __forceinline__ f32x16 product(const u32x4 &a, const u32x4 &b, const f32x16 &c, T) {
    return mfma_32x32x16(a, b, c, T{});
}
template <class T>
__device__ __forceinline__ f32x4 product(const u32x4 &a, const u32x4 &b, const f32x4 &c, T) {
    return mfma_16x16x32(a, b, c, T{});
}

typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef __attribute__((address_space(1))) const uint8_t global_byte;

// What takes the place of pieces that hold no element.
__device__ const __align__(16) uint8_t zeros[16] = {};

__device__ __forceinline__ u32x2 read_turned(lds_byte *p) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(p)));
}

// Asks the compiler to keep `AHEAD` sets of `READS` LDS reads in flight before the first of `SETS` sets of `PRODUCTS`
// products that take one each, and to issue one more after each.
template <int SETS, int PRODUCTS, int READS, int AHEAD>
__device__ __forceinline__ void interleave() {
    constexpr int kProduct = 0x8, kRead = 0x100;
    __builtin_amdgcn_sched_group_barrier(kRead, AHEAD * READS, 0);
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        __builtin_amdgcn_sched_group_barrier(kProduct, PRODUCTS, 0);
        if (i < SETS - AHEAD)
            __builtin_amdgcn_sched_group_barrier(kRead, READS, 0);
    }
}

// RW: rows of a wave, 32 (products of 32x32x16) or 16 (16x16x32).  PLAIN: neither a cap nor slopes.  FULL: weights
// meet V as two numbers of T, the second being what the first leaves, so that the output's rounding alone shows: off
// by 0.00166 of its norm (bf16).  Else one, rounded, since a second product and its operands cost 1.28 times the time
// for the turn above (2.00 ms instead of 1.57) and 1.18 for the ragged tails (0.78 instead of 0.66): 0.00225 and
// 0.00233.
template <class T, bool FP8, int DP, int TK, int RW, bool PLAIN, bool FULL>
__global__ __launch_bounds__(64 * kRows / RW, 2) void tail_kernel(const AttendArgs a, const Parts parts, const int tiles) {
    constexpr int E = FP8 ? 1 : 2;
    constexpr int ROW = 2 * DP;                     // bytes of a row in LDS
    constexpr int GC = DP * E / 16;                 // 16-byte pieces of a cached row
    constexpr int WAVES = kRows / RW, RP = 64 * WAVES / GC;  // rows that the workgroup loads at once
    constexpr int NP = TK / RP;                     // times
    constexpr bool WIDE = RW == 32;
    constexpr int TB = TK / 32, NS = RW / 2;        // rounds of 32 tokens; scores of a lane in one
    constexpr int KD = WIDE ? 16 : 32;              // columns of a product of scores
    constexpr int KS = DP / KD, DB = DP / RW;       // products of 32 tokens' scores, tiles of the output
    constexpr int SETS = WIDE ? 2 : 1;              // products of a tile of the output in 32 tokens
    typedef typename Tile<RW>::type Sums;
    // Permutations of a row's 16-byte pieces in LDS, so that the lanes that read together meet 256 different bytes of
    // the banks: 16 rows of one piece (K), 4 rows of 4 or 8 of 2 pieces (V).
    const auto k_permute = [](int t) { return (WIDE ? t : (t & 3) | (t >> 1 & 12)) & (DP / 8 < 16 ? DP / 8 - 1 : 15); };
    const auto v_permute = [](int t) {
        return (!WIDE ? 2 * ((t & 3) | (t >> 1 & 4)) : DP == 64 ? 4 * (t >> 1 & 1) : 4 * (t & 3)) | (t & 1);
    };
    // Token (of 32) of a lane's x-th score.
    const auto token_of = [](int x, int part) { return WIDE ? 8 * (x >> 2) + part * 4 + (x & 3) : part * 8 + x; };
    static_assert(TK % RP == 0, "whole rounds of loads");
    __shared__ __align__(16) uint8_t lds[2][2][TK * ROW];  // [K, V][round]

    const Pages &pg = a.pages;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & (RW - 1), part = lane / RW;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = a.num_seqs * pg.H, group = blockIdx.x % groups, item = blockIdx.x / groups;
    const int b = group / pg.H, h = group - b * pg.H;
    const int split = item % parts.splits, tile = tiles - 1 - item / parts.splits;  // the longest first
    Sequence seq;
    if (!sequence(a.batch, b, pg.err, seq))
        return;
    const int rows = seq.nq * a.group, row0 = tile * kRows;
    if (row0 >= rows || rows <= kStepRows)
        return;
    const int i0 = divide(row0, a.by_group), i1 = divide(min(row0 + kRows, rows) - 1, a.by_group) + 1;
    const Span span = span_of(seq.n, seq.nq, i0, i1, a.window);
    // (A part starts below 2^31, as the parts before it are shorter than the longest span, but may end beyond.)
    const int begin = span.start + split * parts.len;
    if (split > 0 && begin >= span.end)
        return;
    const uint32_t part_end = static_cast<uint32_t>(begin) + static_cast<uint32_t>(parts.len);
    const int stop = min(span.end, static_cast<int>(min(part_end, uint32_t{INT32_MAX})));
    const bool whole = span.end - span.start <= parts.len;

    // This lane's row: its query as the first product's operand, and what it sees.
    const int r = row0 + wave * RW + c;
    const bool row_ok = r < rows;
    const int row_i = divide(min(r, rows - 1), a.by_group), head = h * a.group + min(r, rows - 1) - row_i * a.group;
    const int p_row = row_ok ? seq.n - seq.nq + row_i : -1;
    const int wave_r0 = min(row0 + wave * RW, rows - 1), wave_r1 = min(row0 + wave * RW + RW - 1, rows - 1);
    const int p_first = seq.n - seq.nq + divide(wave_r0, a.by_group);
    const int p_last = seq.n - seq.nq + divide(wave_r1, a.by_group);
    const int low_last = a.window > 0 ? p_last + 1 - a.window : 0;
    const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.f;
    const float scale = a.scale * kLog2e;
    u32x4 qf[KS];
    {
        const uint8_t *q = a.q.data + (seq.q0 + row_i) * a.q.token_stride + head * a.q.head_stride;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int d = k * KD + part * 8;
            qf[k] = row_ok && d < pg.D ? *reinterpret_cast<const u32x4 *>(q + 2 * d) : u32x4{0, 0, 0, 0};
        }
    }

    const int32_t *table = a.batch.tables + b * a.batch.table_stride;
    const uint8_t *cache = pg.base + static_cast<uint32_t>(h) * pg.head_bytes;
    // (e4m3: a piece is two in LDS, so 8 lanes of a row would write every other one, and meet banks twice; 4 of the 8
    // take the next row, whose pairs are turned about: 0.658 ms instead of 0.667 for the ragged tails.)
    const int piece = FP8 ? (tid & 3) | (tid >> 1 & (GC - 4)) : tid % GC;
    const int first_row = FP8 && GC > 4 ? (tid >> 2 & 1) | tid / (2 * GC) * 2 : tid / GC;
    const bool piece_ok = piece * 16 < pg.row_bytes;

    // Lanes look up a round's tokens (lane % TK each): the page's block, then where the token's row is; -1 for a token
    // that takes part in nothing.  (No branch: beyond the part the last token's entry is read again, and waits are
    // counted, not emptied.)
    auto block_at = [&](int base) {
        const int t = base + (lane & (TK - 1));
        return table[divide(max(min(t, stop - 1), span.first), pg.by_bs)];
    };
    auto offset_at = [&](int base, int block) -> int64_t {
        const int t = base + (lane & (TK - 1));
        if (t >= stop || t < span.first || !in_cache(pg, block))
            return -1;
        return block * pg.block_stride + static_cast<uint32_t>(t - divide(t, pg.by_bs) * pg.BS) * pg.token_bytes;
    };
    // Requests K and V rows of a round: two-byte rows straight into LDS (a wave's 64 pieces of 16 bytes lie there as
    // its lanes do, so a lane fetches the piece that the permutation wants in its place), e4m3 into registers.  Slots
    // without a token and columns beyond D may hold anything, and 0 times it need not be 0: they become zeros.
    u32x4 next[2][FP8 ? NP : 1];
    // Of e4m3 rows a wave's WR rows of one load lie in one page where pages hold multiples of them (rounds begin at
    // multiples of 32).  If all of the round's tokens take part, the first row's address is the wave's, and the
    // lanes' distances from it are the same every round: 0.69 ms instead of 0.74 for the ragged tails above.  2-byte
    // rows do not gain (1.57 to 1.60 ms instead of 1.56): their pieces are permuted as well.
    constexpr int WR = 64 / GC;  // rows of a wave in one load
    const bool together = FP8 && pg.BS % WR == 0 && pg.D == DP;
    const uint32_t lane_row = static_cast<uint32_t>(first_row - wave * WR) * pg.token_bytes;
    auto request = [&](int64_t off, int buffer) {
        const bool all = __all(off >= 0);
        if constexpr (FP8) {
            if (together && all) {
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    const int first = n * RP + wave * WR;
                    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(off), first);
                    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(off >> 32), first);
                    const uint8_t *row = cache + static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv)
                        next[kv][n] = *reinterpret_cast<const u32x4 *>((kv ? row + pg.v_bytes : row) +
                                                                         (lane_row + piece * 16));
                }
                return;
            }
        }
        int64_t at[NP];
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int src = first_row + n * RP;
            const uint32_t lo = __shfl(static_cast<uint32_t>(off), src);
            const uint32_t hi = __shfl(static_cast<uint32_t>(off >> 32), src);
            at[n] = static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
        }
        if constexpr (FP8) {
#pragma unroll
            for (int n = 0; n < NP; ++n)
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>((kv ? cache + pg.v_bytes : cache) +
                                                                     max(at[n], int64_t{0}) + (piece_ok ? piece * 16 : 0));
                    next[kv][n] = at[n] < 0 || !piece_ok ? u32x4{0, 0, 0, 0} : x;
                }
        } else {
            const auto fetch = [&](auto every) {
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    const int src = first_row + n * RP;
                    const int to = (n * RP + wave * (64 / GC)) * ROW;  // the wave's first row
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        const int from = piece ^ (kv ? v_permute(src) : k_permute(src));
                        const uint8_t *x = (kv ? cache + pg.v_bytes : cache) + from * 16 + at[n];
                        if (!every && (at[n] < 0 || from * 16 >= pg.row_bytes))
                            x = zeros;
                        __builtin_amdgcn_global_load_lds((global_byte *)x, (lds_byte *)(lds[kv][buffer] + to), 16, 0, 0);
                    }
                }
            };
            if (pg.D == DP && all)
                fetch(std::true_type{});
            else
                fetch(std::false_type{});
        }
    };
    // What request() fetched is in LDS when every wave has done this and met at a barrier.
    auto deposit = [&](int kv, int buffer) {
        if constexpr (FP8) {
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                const int t = first_row + n * RP, permute = kv ? v_permute(t) : k_permute(t);
                uint8_t *to = lds[kv][buffer] + t * ROW;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t x0 = next[kv][n][2 * j], x1 = next[kv][n][2 * j + 1];
                    *reinterpret_cast<u32x4 *>(to + ((2 * piece + j) ^ permute) * 16) =
                        u32x4{T::from_e4m3(x0, false), T::from_e4m3(x0, true), T::from_e4m3(x1, false),
                              T::from_e4m3(x1, true)};
                }
            }
        } else {
            __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
        }
    };

    constexpr int AN = RW * RW / 64;  // elements of a tile of the output in a lane
    Sums acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int x = 0; x < AN; ++x)
            acc[d][x] = 0.f;
    float m = kLowest, l = 0.f;

    // Where this lane reads.  K: 16 bytes of a token's row per product, the token c of 32, or for the two products of
    // 16 tokens (c / 4) * 8 + c % 4 and that + 4.  V: 8 bytes, of one of 4 tokens' rows for the 16 lanes that turn
    // them, and of the one 8 (or 4) on.  Rows start at multiples of their length, so a permuted piece's address is
    // the first one's with bits of the product's (or the tile's) number turned over.
    const int k_row = WIDE ? c : (c >> 2) * 8 + (c & 3), v_row = part * (WIDE ? 4 : 8) + (lane >> 2 & 3);
    const int v_piece = (WIDE ? (lane >> 4 & 1) * 2 : 0) + (lane >> 1 & 1);
    int k_at = k_row * ROW + (part ^ k_permute(k_row)) * 16;
    int v_at = v_row * ROW + (v_piece ^ v_permute(v_row)) * 16 + (lane & 1) * 8;

    auto take_scores = [&](int buffer, float (&s)[TB][NS]) {
        const uint8_t *k_lds = lds[0][buffer];
        constexpr int SETS_K = WIDE ? 1 : 2;  // products side by side of 32 tokens
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            Sums sum[SETS_K];
#pragma unroll
            for (int j = 0; j < SETS_K; ++j) {
#pragma unroll
                for (int x = 0; x < AN; ++x)
                    sum[j][x] = 0.f;
                // (The permutation does not see the 4 tokens between the two products' rows.)
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    sum[j] = product(
                        *reinterpret_cast<const u32x4 *>(k_lds + (t * 32 + j * 4) * ROW + (k_at ^ k * 2 * KD)), qf[k],
                        sum[j], T{});
            }
#pragma unroll
            for (int x = 0; x < NS; ++x)
                s[t][x] = sum[x / AN][x % AN];
        }
        interleave<TB * SETS_K * KS, 1, 1, 6>();
    };
    // The largest over the lanes that share a row.
    const auto over_parts = [](float x) {
        x = fmaxf(x, __shfl_xor(x, 32));
        return WIDE ? x : fmaxf(x, __shfl_xor(x, 16));
    };

    if (begin < stop) {
        int buffer = 0;
        int64_t off = offset_at(begin, block_at(begin));
        int next_block = block_at(begin + TK);
        request(off, 0);
        deposit(0, 0);
        deposit(1, 0);
        __syncthreads();
        for (int base = begin;; base += TK, buffer ^= 1) {
            const bool more = stop - base > TK;
            const uint64_t usable = __ballot(off >= 0);
            if (more) {
                off = offset_at(base + TK, next_block);
                next_block = block_at(base + 2 * TK);
                request(off, buffer ^ 1);
            }
            // (Addresses are worked out where they are used: kept, they would cost registers.)
            asm volatile("" : "+v"(k_at), "+v"(v_at));
            // (The products go first: the other wave of the SIMD has its exponentials for the time between them.)
            __builtin_amdgcn_s_setprio(1);
            float s[TB][NS];
            take_scores(buffer, s);
            __builtin_amdgcn_s_setprio(0);
            const bool edge = usable != ~uint64_t{0} || p_first - base < TK - 1 || base < low_last;
            // Scores in powers of 2; in the plain case the factor is left to the exponent's argument.
            const float factor = PLAIN ? scale : 1.f;
            if constexpr (!PLAIN) {
                const auto each = [&](auto &&f) {
#pragma unroll
                    for (int t = 0; t < TB; ++t)
#pragma unroll
                        for (int x = 0; x < NS; ++x)
                            s[t][x] = f(s[t][x], t * 32 + token_of(x, part));
                };
                if (a.softcap > kSmallCap) {
                    const float inv = a.scale / a.softcap, cap = a.softcap * kLog2e;
                    each([&](float y, int) { return capped(y, inv, cap); });
                } else if (a.softcap > 0.f) {
                    const float twice = 2.f * kLog2e * a.scale / a.softcap, cap = a.softcap * kLog2e;
                    each([&](float y, int) { return small_capped(y, twice, cap); });
                } else {
                    each([&](float y, int) { return y * scale; });
                }
                if (a.slopes)
                    each([&](float y, int at) { return y - slope * static_cast<float>(p_row - (base + at)); });
            }
            if (edge) {
                // Tokens of this round that the row sees, counted from `base`: [from, to), and usable ones.
                const int to = p_row - base + 1, from = a.window > 0 ? to - a.window : INT32_MIN;
                const uint64_t mine = usable >> token_of(0, part);
#pragma unroll
                for (int t = 0; t < TB; ++t)
#pragma unroll
                    for (int x = 0; x < NS; ++x) {
                        const int bit = t * 32 + token_of(x, 0), at = t * 32 + token_of(x, part);
                        const bool sees = (mine >> bit & 1) && at < to && at >= from;
                        s[t][x] = sees ? s[t][x] : -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int x = 0; x < NS; x += 2)
                    top = fmaxf(fmaxf(top, s[t][x]), s[t][x + 1]);
            top *= factor;
            if (__any(top > m + 8.f)) {
                const float higher = fmaxf(m, over_parts(top)), f = __builtin_amdgcn_exp2f(m - higher);
                m = higher;
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int x = 0; x < AN; ++x)
                        acc[d][x] *= f;
            }
            const float zero = m - T::kShift;
            u32x4 p[TB][SETS], p_rest[TB][FULL ? SETS : 1];
            float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int x = 0; x < NS; x += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[t][x], factor, -zero));
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[t][x + 1], factor, -zero));
                    sums[x & 2] += e0;
                    sums[(x & 2) + 1] += e1;
                    const uint32_t w = T::pack(e0, e1);
                    p[t][x >> 3][x >> 1 & 3] = w;
                    if constexpr (FULL)
                        p_rest[t][x >> 3][x >> 1 & 3] = T::pack(e0 - T::low(w), e1 - T::high(w));
                }
            l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
            // (e4m3: K of the next round is widened beside the other wave's products, V after this one's; 0.665 ms
            // instead of 0.675 with both at the end.)
            if (FP8 && more)
                deposit(0, buffer ^ 1);
            asm volatile("" : "+v"(v_at));
            __builtin_amdgcn_s_setprio(1);
            lds_byte *v_lds = (lds_byte *)(lds[1][buffer]);  // (a cast between address spaces)
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int j = 0; j < SETS; ++j)
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        lds_byte *at = v_lds + (v_at ^ d * 2 * RW) + (t * 32 + j * 16) * ROW;
                        const u32x2 x = read_turned(at), y = read_turned(at + (WIDE ? 8 : 4) * ROW);
                        acc[d] = product(u32x4{x[0], x[1], y[0], y[1]}, p[t][j], acc[d], T{});
                        if constexpr (FULL)
                            acc[d] = product(u32x4{x[0], x[1], y[0], y[1]}, p_rest[t][j], acc[d], T{});
                    }
            interleave<TB * SETS * DB, FULL ? 2 : 1, 2, 3>();
            __builtin_amdgcn_s_setprio(0);
            if (!more)
                break;
            if (!FP8)
                deposit(0, buffer ^ 1);
            deposit(1, buffer ^ 1);
            __syncthreads();
        }
    }

    l += __shfl_xor(l, 32);
    if constexpr (!WIDE)
        l += __shfl_xor(l, 16);
    if (!row_ok)
        return;
    const float inv = l == 0.f ? 0.f : a.v_scale / l;
    const int64_t slot = (static_cast<int64_t>(seq.q0 + row_i) * a.heads + head) * parts.splits + split;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int x = 0; x < AN; x += 4) {
            const int col = d * RW + 2 * x + part * 4;
            if (col >= pg.D)
                continue;
            if (whole) {
                uint8_t *to = a.out.data + (seq.q0 + row_i) * a.out.token_stride + head * a.out.head_stride + 2 * col;
                *reinterpret_cast<u32x2 *>(to) = u32x2{T::pack(acc[d][x] * inv, acc[d][x + 1] * inv),
                                                        T::pack(acc[d][x + 2] * inv, acc[d][x + 3] * inv)};
            } else {
                *reinterpret_cast<f32x4 *>(parts.sums + slot * pg.D + col) =
                    f32x4{acc[d][x], acc[d][x + 1], acc[d][x + 2], acc[d][x + 3]};
            }
        }
    if (part == 0) {
        if (whole) {
            a.lse[static_cast<int64_t>(seq.q0 + row_i) * a.heads + head] =
                l == 0.f ? -INFINITY : (m - T::kShift + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
            parts.stats[slot * 2] = m - T::kShift;
            parts.stats[slot * 2 + 1] = l;
        }
    }
}

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

template <class T, bool FP8, int DP, int TK, int RW, bool PLAIN, bool FULL>
hipError_t launch(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    const int tiles = static_cast<int>(tail_tiles(max_queries, a.group));
    const uint32_t grid = static_cast<uint32_t>(tiles) * parts.splits * a.pages.H * a.num_seqs;
    return launch_kernel(tail_kernel<T, FP8, DP, TK, RW, PLAIN, FULL>, dim3(grid), 64 * kRows / RW, stream, a, parts,
                         tiles);
}

template <class T, bool FP8, bool PLAIN, bool FULL>
hipError_t launch(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    // (Wide rows: 32 of them would need more registers than two waves of a SIMD have, and one wave alone took 1.7
    // times as long.)
    if (a.pages.D > 128)
        return launch<T, FP8, 256, 64, 16, PLAIN, FULL>(a, parts, max_queries, stream);
    if (a.pages.D > 64)
        return launch<T, FP8, 128, 64, 32, PLAIN, FULL>(a, parts, max_queries, stream);
    return launch<T, FP8, 64, 64, 32, PLAIN, FULL>(a, parts, max_queries, stream);
}

template <class T, bool FP8>
hipError_t launch(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    if (a.softcap == 0.f && !a.slopes)
        return a.full_weights ? launch<T, FP8, true, true>(a, parts, max_queries, stream)
                              : launch<T, FP8, true, false>(a, parts, max_queries, stream);
    return a.full_weights ? launch<T, FP8, false, true>(a, parts, max_queries, stream)
                          : launch<T, FP8, false, false>(a, parts, max_queries, stream);
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
