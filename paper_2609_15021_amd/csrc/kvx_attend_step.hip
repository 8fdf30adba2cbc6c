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
// One sequence behind 131,077 tokens (8 heads of 5 rows, bf16, D 128): 95 us and 7 to join, 5.2 TB/s with both (a
// large reduction reads 6.1, a large copy moves 4.8).  16 sequences of up to 32,768 tokens in e4m3 (4 heads of 6
// rows, D 256): 117 us and 8 to join, 4.8 TB/s.  48 of up to 8,192 with weights (2 heads of 8 rows): 53 us (209 MB of
// K and V read, 13 MB of scores written), 8 to join, 7 for what each token received.
#include <algorithm>

#include "kvx_attend_kernels.h"

namespace kvx {

namespace {

constexpr int kWaves = 4;

template <int BYTES>
struct Vec;
template <>
struct Vec<4> {
    uint32_t w[1];
    __device__ __forceinline__ void load(const uint8_t *p) { w[0] = *reinterpret_cast<const uint32_t *>(p); }
};
template <>
struct Vec<8> {
    uint32_t w[2];
    __device__ __forceinline__ void load(const uint8_t *p) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
        w[0] = x[0];
        w[1] = x[1];
    }
};
template <>
struct Vec<16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint8_t *p) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
        w[0] = x[0];
        w[1] = x[1];
        w[2] = x[2];
        w[3] = x[3];
    }
};

// T: type of q, of the weights and of out; FP8: the cache holds e4m3; DP >= D columns; NT: tiles of 16 rows.
// (2 waves a SIMD; wide 2-byte rows would need to spill for that, and one wave runs them.)
template <class T, bool FP8, int DP, int NT>
__global__ __launch_bounds__(64 * kWaves, !FP8 && DP > 128 ? 1 : 2) void step_kernel(const AttendArgs a,
                                                                                     const Shares shares) {
    constexpr int E = FP8 ? 1 : 2;                       // bytes of a cached element
    constexpr int KC = DP * E / 64;                      // 16-byte pieces of a token's K in a lane
    constexpr int VE = DP / 16 * E > 16 ? 16 / E : DP / 16;  // V columns of a lane in a piece
    constexpr int NV = DP / (16 * VE);                   // such pieces
    constexpr int TILES = NV * VE;                       // 16-column tiles of the output
    const Pages &pg = a.pages;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.y / pg.H, h = blockIdx.y - tile * pg.H;
    Share share;
    if (!share_of(a, shares, blockIdx.x, false, share))
        return;
    const int b = share.b;
    Sequence seq;
    if (!sequence(a.batch, b, pg.err, seq))
        return;
    const int rows = seq.nq * a.group, row0 = tile * 16 * NT;
    if (row0 >= rows)
        return;
    const int i0 = divide(row0, a.by_group), i1 = divide(min(row0 + 16 * NT, rows) - 1, a.by_group) + 1;
    const Span span = span_of(seq.n, seq.nq, i0, i1, a.window);
    const int64_t part_at =
        span_of(seq.n, seq.nq, 0, seq.nq, a.window).start + static_cast<int64_t>(share.split) * share.len;
    const int begin = static_cast<int>(min(part_at, int64_t{INT32_MAX} - 1023));
    const int stop = static_cast<int>(min(part_at + share.len, static_cast<int64_t>(span.end)));
    const bool whole = share.parts == 1;
    const int p_first = seq.n - seq.nq + i0;
    const int low_last = a.window > 0 ? span.end - a.window : 0;  // from here on every row's window is open

    const int64_t slot0 = (static_cast<int64_t>(h) * shares.items + blockIdx.x) * shares.row_cap + row0;
    const int64_t score0 = (static_cast<int64_t>(b) * pg.H + h) * a.score_cap + row0;

    // Queries: a row's elements in the order in which K's pieces hold them.
    u32x4 qf[NT][KC * 2 / E];
    int p_of[NT];
    float slope[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = row0 + nt * 16 + c;
        const bool row = r < rows;
        const int i = divide(min(r, rows - 1), a.by_group), head = h * a.group + min(r, rows - 1) - i * a.group;
        p_of[nt] = row ? seq.n - seq.nq + i : -1;
        slope[nt] = a.slopes ? a.slopes[head] * kLog2e : 0.f;
        const uint8_t *q = a.q.data + (seq.q0 + i) * a.q.token_stride + head * a.q.head_stride;
#pragma unroll
        for (int k = 0; k < KC * 2 / E; ++k) {
            const int d = FP8 ? (k >> 1) * 64 + g * 16 + (k & 1) * 8 : k * 32 + g * 8;
            qf[nt][k] = row && d < pg.D ? *reinterpret_cast<const u32x4 *>(q + 2 * d) : u32x4{0, 0, 0, 0};
        }
    }

    // Where a lane's pieces start in a row (columns beyond D: the row's start, which Q's zeros or the output ignore).
    int k_at[KC], v_at[NV];
#pragma unroll
    for (int k = 0; k < KC; ++k)
        k_at[k] = k * 64 + g * 16 < pg.row_bytes ? k * 64 + g * 16 : 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int at = (v * 16 + c) * VE * E;
        v_at[v] = static_cast<int>(pg.v_bytes) + (at < pg.row_bytes ? at : 0);
    }
    const bool by_8 = pg.BS % 8 == 0;
    const int32_t *table = a.batch.tables + b * a.batch.table_stride;
    const uint8_t *cache = pg.base + static_cast<uint32_t>(h) * pg.head_bytes;

    // Page of token base + lane % 32, and where that token's row is (-1: none that a row sees).
    auto page_at = [&](int base, int &page, bool &shown) {
        const int t = base + (lane & 31);
        page = divide(t, pg.by_bs);
        shown = t < stop && (page + 1) * static_cast<int64_t>(pg.BS) > span.first;
        return shown ? table[page] : 0;
    };
    auto offset_at = [&](int base, int page, bool shown, int block) -> int64_t {
        if (!shown || !in_cache(pg, block))
            return -1;
        return block * pg.block_stride + static_cast<uint32_t>(base + (lane & 31) - page * pg.BS) * pg.token_bytes;
    };
    auto from_lane = [&](int64_t x, int src) -> int64_t {
        const uint32_t lo = __shfl(static_cast<uint32_t>(x), src), hi = __shfl(static_cast<uint32_t>(x >> 32), src);
        return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
    };

    Vec<16> k_reg[2][KC];
    Vec<VE * E> v_reg[8][NV];
    auto load_k = [&](int64_t off) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t at = max(from_lane(off, (c >> 2) * 8 + j * 4 + (c & 3)), int64_t{0});
#pragma unroll
            for (int k = 0; k < KC; ++k)
                k_reg[j][k].load(cache + at + k_at[k]);
        }
    };
    auto load_v = [&](int64_t off) {
        if (by_8) {
            int64_t at = max(from_lane(off, g * 8), int64_t{0});
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    v_reg[e][v].load(cache + at + v_at[v]);
                at += pg.token_bytes;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t at = max(from_lane(off, g * 8 + e), int64_t{0});
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    v_reg[e][v].load(cache + at + v_at[v]);
            }
        }
    };

    f32x4 acc[NT][TILES];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = kLowest;
        l[nt] = 0.f;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
            acc[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    constexpr int kStride = 32 * kWaves;
    int base = begin + wave * 32;
    if (base < stop) {
        int page, next_page = 0, next_block = 0;
        bool shown, next_shown = false;
        int block = page_at(base, page, shown);
        int64_t off = offset_at(base, page, shown, block);
        if (stop - base > kStride)
            next_block = page_at(base + kStride, next_page, next_shown);
        load_k(off);
        load_v(off);
        while (true) {
            const int t_lane = base + (lane & 31);
            const bool use = off >= 0 && t_lane >= span.first && t_lane < stop;
            const uint32_t usable = static_cast<uint32_t>(__ballot(use));
            const bool edge = usable != 0xffffffffu || p_first - base < 31 || base < low_last;
            const bool more = stop - base > kStride;

            f32x4 s[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[nt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < KC; ++k) {
                        const Vec<16> &x = k_reg[j][k];
                        if constexpr (FP8) {
                            s[nt][j] = mfma_16x16x32(u32x4{T::from_e4m3(x.w[0], false), T::from_e4m3(x.w[0], true),
                                                           T::from_e4m3(x.w[1], false), T::from_e4m3(x.w[1], true)},
                                                     qf[nt][2 * k], s[nt][j], T{});
                            s[nt][j] = mfma_16x16x32(u32x4{T::from_e4m3(x.w[2], false), T::from_e4m3(x.w[2], true),
                                                           T::from_e4m3(x.w[3], false), T::from_e4m3(x.w[3], true)},
                                                     qf[nt][2 * k + 1], s[nt][j], T{});
                        } else {
                            s[nt][j] = mfma_16x16x32(u32x4{x.w[0], x.w[1], x.w[2], x.w[3]}, qf[nt][k], s[nt][j], T{});
                        }
                    }
                }
            int64_t next_off = -1;
            if (more) {
                next_off = offset_at(base + kStride, next_page, next_shown, next_block);
                load_k(next_off);
                if (stop - base > 2 * kStride)
                    next_block = page_at(base + 2 * kStride, next_page, next_shown);
            }

            // Weights.  Everything from here on is in powers of 2.
            u32x4 p[NT], p_rest[NT];
            const uint32_t bits = usable >> (g * 8);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = s[nt][e >> 2][e & 3];
                if (a.softcap > 0.f) {
                    const float inv = a.scale / a.softcap, cap = a.softcap * kLog2e;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = capped(x[e], inv, cap);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] *= a.scale * kLog2e;
                }
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] -= slope[nt] * static_cast<float>(p_of[nt] - (base + g * 8 + e));
                }
                if (edge) {
                    const int to = p_of[nt] - (base + g * 8) + 1, from = a.window > 0 ? to - a.window : INT32_MIN;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (bits >> e & 1) && e < to && e >= from ? x[e] : -INFINITY;
                }
                if (a.scores && row0 + nt * 16 + c < rows) {
                    float *to = a.scores + (score0 + nt * 16 + c) * a.score_len + base + g * 8;
                    *reinterpret_cast<f32x4 *>(to) = f32x4{x[0], x[1], x[2], x[3]};
                    *reinterpret_cast<f32x4 *>(to + 4) = f32x4{x[4], x[5], x[6], x[7]};
                }
                float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                  fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
                // The sums are scaled down only when some score has outgrown them by 2^8.
                if (__any(top > m[nt] + 8.f)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float next = fmaxf(m[nt], top), f = __builtin_amdgcn_exp2f(m[nt] - next);
                    m[nt] = next;
                    l[nt] *= f;
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
                        acc[nt][t] *= f;
                }
                const float zero = m[nt] - T::kShift;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = __builtin_amdgcn_exp2f(x[e] - zero);
                l[nt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                // A weight is two numbers of the rows' type, so that its rounding does not add to the output's: the
                // products wait for memory anyway.
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const uint32_t w = T::pack(x[e], x[e + 1]);
                    p[nt][e / 2] = w;
                    p_rest[nt][e / 2] = T::pack(x[e] - T::low(w), x[e + 1] - T::high(w));
                }
            }

            // A slot without a token may hold anything, and 0 times it need not be 0.
            if (usable != 0xffffffffu) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(bits >> e & 1)) {
#pragma unroll
                        for (int v = 0; v < NV; ++v)
#pragma unroll
                            for (int w = 0; w < VE * E / 4; ++w)
                                v_reg[e][v].w[w] = 0;
                    }
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int w = 0; w < VE * E / 4; ++w) {
                    constexpr int kEach = 4 / E;  // columns in 4 bytes
                    u32x4 turned[kEach];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t x = v_reg[2 * e][v].w[w], y = v_reg[2 * e + 1][v].w[w];
                        if constexpr (FP8) {
                            const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x05010400);
                            const uint32_t hi = __builtin_amdgcn_perm(y, x, 0x07030602);
                            turned[0][e] = T::from_e4m3(lo, false);
                            turned[1][e] = T::from_e4m3(lo, true);
                            turned[2][e] = T::from_e4m3(hi, false);
                            turned[3][e] = T::from_e4m3(hi, true);
                        } else {
                            turned[0][e] = __builtin_amdgcn_perm(y, x, 0x05040100);
                            turned[1][e] = __builtin_amdgcn_perm(y, x, 0x07060302);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            f32x4 &x = acc[nt][v * VE + w * kEach + j];
                            x = mfma_16x16x32(turned[j], p[nt], x, T{});
                            x = mfma_16x16x32(turned[j], p_rest[nt], x, T{});
                        }
                }
            if (!more)
                break;
            load_v(next_off);
            off = next_off;
            base += kStride;
        }
    }

    // Join the waves: every wave's largest score and sum, then wave w collects component w of every tile, which are VE
    // consecutive columns per lane.
    __shared__ float stats[kWaves][NT * 16][2];
    __shared__ float parts[kWaves][kWaves - 1][NT * TILES][64];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        l[nt] += __shfl_xor(l[nt], 16);
        l[nt] += __shfl_xor(l[nt], 32);
        if (g == 0) {
            stats[wave][nt * 16 + c][0] = m[nt];
            stats[wave][nt * 16 + c][1] = l[nt];
        }
    }
    __syncthreads();
    float most[NT], total[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int col = nt * 16 + c;
        most[nt] = fmaxf(fmaxf(stats[0][col][0], stats[1][col][0]), fmaxf(stats[2][col][0], stats[3][col][0]));
        total[nt] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            total[nt] += stats[w][col][1] * __builtin_amdgcn_exp2f(stats[w][col][0] - most[nt]);
        const float f = __builtin_amdgcn_exp2f(m[nt] - most[nt]);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            acc[nt][t] *= f;
#pragma unroll
            for (int r = 0; r < kWaves; ++r)
                if (r != wave)
                    parts[r][wave - (wave > r)][nt * TILES + t][lane] = acc[nt][t][r];
        }
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = row0 + nt * 16 + c;
        if (r >= rows)
            continue;
        const int i = divide(r, a.by_group), head = h * a.group + r - i * a.group, row = seq.q0 + i;
        const int64_t slot = slot0 + nt * 16 + c;
        const float inv = total[nt] == 0.f ? 0.f : a.v_scale / total[nt];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int d = v * 16 * VE + (g * 4 + wave) * VE;
            float x[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const f32x4 &own = acc[nt][v * VE + j];
                x[j] = wave == 0 ? own[0] : wave == 1 ? own[1] : wave == 2 ? own[2] : own[3];
#pragma unroll
                for (int k = 0; k < kWaves - 1; ++k)
                    x[j] += parts[wave][k][nt * TILES + v * VE + j][lane];
            }
            if (d >= pg.D)
                continue;
            if (whole) {
                uint8_t *to = a.out.data + row * a.out.token_stride + head * a.out.head_stride + 2 * d;
#pragma unroll
                for (int j = 0; j < VE; j += 4)
                    *reinterpret_cast<u32x2 *>(to + 2 * j) = u32x2{T::pack(x[j] * inv, x[j + 1] * inv),
                                                                    T::pack(x[j + 2] * inv, x[j + 3] * inv)};
            } else {
                float *to = shares.sums + slot * pg.D + d;
#pragma unroll
                for (int j = 0; j < VE; j += 4)
                    *reinterpret_cast<f32x4 *>(to + j) = f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
            }
        }
        if (wave == 0 && g == 0) {
            if (whole) {
                a.lse[static_cast<int64_t>(row) * a.heads + head] =
                    total[nt] == 0.f ? -INFINITY : (most[nt] - T::kShift + __builtin_amdgcn_logf(total[nt])) * kLn2;
            } else {
                shares.stats[slot * 2] = most[nt] - T::kShift;
                shares.stats[slot * 2 + 1] = total[nt];
            }
        }
    }
}

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
    const int64_t len = share_len(a, shares, tid, 1024, true, sum);
    int32_t *seqs = shares.items_of + 2, *items = seqs + 2 * static_cast<int64_t>(shares.num_seqs);
    int base = 0;
    for (int b0 = 0; b0 < shares.num_seqs; b0 += 1024) {
        const int b = b0 + tid, mine = b < shares.num_seqs ? share_parts(a, b, len) : 0, upto = sum_up_to_lane(mine);
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
        shares.items_of[0] = static_cast<int>(len);
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
    if (rows <= kStepRows)
        return Row{0, 0, 0};
    const Span span = span_of(seq.n, seq.nq, divide(row0, a.by_group),
                              divide(min(row0 + kTailRows, rows) - 1, a.by_group) + 1, a.window);
    const int i = divide(r, a.by_group), head = h * a.group + r - i * a.group;
    return Row{(static_cast<int64_t>(seq.q0 + i) * a.heads + head) * from.splits, 1, parts_of(span, from.len)};
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
    // (The first parts' sums are on their way while the row's largest score is looked for.)
    constexpr int EARLY = SPREAD ? 8 : 4;
    const int s0 = SPREAD ? mine : 0, ds = SPREAD ? groups : 1;
    f32x4 early[EARLY];
    float early_most[EARLY];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) {
        const int s = s0 + k * ds;
        const bool is = row && s < parts;
        early[k] = is ? *reinterpret_cast<const f32x4 *>(from.sums + (row_at.slot + s * step) * D + d)
                      : f32x4{0.f, 0.f, 0.f, 0.f};
        early_most[k] = is ? stats[2 * s * step] : kLowest;
    }
    if constexpr (SPREAD) {  // every wave for itself
        const int lane = tid & 63;
        for (int s = lane; s < parts; s += 64)
            most = fmaxf(most, stats[2 * s * step]);
        for (int o = 32; o; o >>= 1)
            most = fmaxf(most, __shfl_xor(most, o));
        for (int s = lane; s < parts; s += 64)
            total += stats[2 * s * step + 1] * __builtin_amdgcn_exp2f(stats[2 * s * step] - most);
        for (int o = 32; o; o >>= 1)
            total += __shfl_xor(total, o);
    } else {
        for (int s = 0; s < parts; ++s)
            most = fmaxf(most, stats[2 * s * step]);
        for (int s = 0; s < parts; ++s)
            total += stats[2 * s * step + 1] * __builtin_amdgcn_exp2f(stats[2 * s * step] - most);
    }
    f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < EARLY; ++k)
        x += early[k] * __builtin_amdgcn_exp2f(early_most[k] - most);
    if (row)
        for (int s = s0 + EARLY * ds; s < parts; s += ds)
            x += *reinterpret_cast<const f32x4 *>(from.sums + (row_at.slot + s * step) * D + d) *
                 __builtin_amdgcn_exp2f(stats[2 * s * step] - most);
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

template <class T, bool FP8, int DP, int NT>
hipError_t launch(const AttendArgs &a, const Shares &shares, int max_rows, hipStream_t stream) {
    const int tiles = (max_rows + 16 * NT - 1) / (16 * NT);
    return launch_kernel(step_kernel<T, FP8, DP, NT>, dim3(shares.items, tiles * a.pages.H), 64 * kWaves, stream, a,
                         shares);
}

template <class T, bool FP8>
hipError_t launch(const AttendArgs &a, const Shares &shares, int max_rows, hipStream_t stream) {
    const bool two = step_tile_rows(max_rows, a.pages.D) == 32;
    if (a.pages.D > 128)
        return launch<T, FP8, 256, 1>(a, shares, max_rows, stream);
    if (a.pages.D > 64)
        return two ? launch<T, FP8, 128, 2>(a, shares, max_rows, stream)
                   : launch<T, FP8, 128, 1>(a, shares, max_rows, stream);
    return two ? launch<T, FP8, 64, 2>(a, shares, max_rows, stream)
               : launch<T, FP8, 64, 1>(a, shares, max_rows, stream);
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
    const int max_rows = static_cast<int>(std::min<int64_t>(kStepRows, static_cast<int64_t>(max_queries) * a.group));
    const bool fp8 = a.cache_type == KV_DTYPE_E4M3;
    if (a.q_type == KV_DTYPE_BF16)
        return fp8 ? launch<Bf16, true>(a, shares, max_rows, stream) : launch<Bf16, false>(a, shares, max_rows, stream);
    return fp8 ? launch<F16, true>(a, shares, max_rows, stream) : launch<F16, false>(a, shares, max_rows, stream);
}

hipError_t launch_join_step(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream) {
    return launch_join<true>(a, shares, std::min(max_queries, std::max(kStepRows / a.group, 1)), stream);
}

hipError_t launch_join_tail(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    // (8 parts one after the other take about as long as one row's launch.)
    return parts.splits > 8 ? launch_join<true>(a, parts, max_queries, stream)
                            : launch_join<false>(a, parts, max_queries, stream);
}

hipError_t launch_weigh_step(const AttendArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>((a.batch.max_len + 1023) / 1024), static_cast<uint32_t>(a.pages.H),
                    static_cast<uint32_t>(a.num_seqs));
    return launch_kernel(weigh_step_kernel, grid, 256, stream, a);
}

}  // namespace kvx
