// The kernel of kv_attend and kv_attend_pages for few new tokens per sequence; kvx_attend_step.hip says how it works.
#pragma once

#include <algorithm>
#include <type_traits>

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

// Where this workgroup leaves row r of its sequence and KV head h, which is `row_head` of all (row, query head) pairs.
__device__ __forceinline__ int64_t slot_in(const Shares &shares, int h, int r, int64_t, int) {
    return (static_cast<int64_t>(h) * shares.items + blockIdx.x) * shares.row_cap + r;
}
__device__ __forceinline__ int64_t slot_in(const Chosen &chosen, int, int, int64_t row_head, int split) {
    return row_head * chosen.splits + split;
}

// T: type of q, of the weights and of out; FP8: the cache holds e4m3; DP >= D columns; NT: tiles of 16 rows.
// (2 waves a SIMD; wide 2-byte rows would need to spill for that, and one wave runs them.  Two tiles of up to 128
// columns spill 3 to 18 registers in some variants, chosen pages of e4m3 with up to 256 columns 5.)
//
// SCALED: pages have scales (or where a.scales has none, scales of 1): K's multiply the scores, V's the weights, which
// then meet V in bfloat16: float16's range would not hold the products.  They are loaded with K, a lane a token.
//
// From: Shares, or Chosen: each new token is a sequence of its own, of the pages that it chose, one after the other.  A
// page's place in the list says where its tokens are, and which: the list is read a round before the table.  Or Alone:
// the same where there are rows enough for every wave to have one for itself, and nothing to join: 111 new tokens of
// each of 17 sequences over one page of 32 (3 heads of 12 rows, D 256) take 30 us instead of 103.  Heads run fastest in
// their grid, so that a head's workgroups come 8 apart where there are 8 heads, and so on one XCD, whose L2 then has
// that head's pages alone: 512 new tokens over 64 of 2,048 pages each take 160 us instead of 204.
template <class T, bool FP8, int DP, int NT, bool SCALED, class From>
__global__ __launch_bounds__(64 * kWaves, !FP8 && DP > 128 ? 1 : 2) void step_kernel(const AttendArgs a,
                                                                                     const From shares) {
    constexpr bool LISTED = std::is_base_of_v<Chosen, From>, ALONE = std::is_same_v<From, Alone>;
    constexpr int TEAM = ALONE ? 1 : kWaves;             // waves of a row
    typedef std::conditional_t<SCALED, Bf16, T> W;       // type of the weights
    constexpr int E = FP8 ? 1 : 2;                       // bytes of a cached element
    constexpr int KC = DP * E / 64;                      // 16-byte pieces of a token's K in a lane
    constexpr int VE = DP / 16 * E > 16 ? 16 / E : DP / 16;  // V columns of a lane in a piece
    constexpr int NV = DP / (16 * VE);                   // such pieces
    constexpr int TILES = NV * VE;                       // 16-column tiles of the output
    const Pages &pg = a.pages;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int across = LISTED ? blockIdx.x : blockIdx.y, place = across / pg.H, h = across - place * pg.H;
    const int tile = LISTED ? blockIdx.y : place;
    Share share;
    Sequence seq;
    [[maybe_unused]] int count = 0;                          // LISTED: pages of the list
    [[maybe_unused]] const int32_t *list = nullptr;
    [[maybe_unused]] int first_entry = 0;
    if constexpr (LISTED) {
        const int item = ALONE ? place * kWaves + wave : place, row = ALONE ? item : item / shares.splits;
        if (ALONE && row >= a.batch.num_queries)
            return;
        share.split = ALONE ? 0 : item - row * shares.splits;
        list = shares.pages + row * shares.token_stride + h * shares.head_stride;
        // (The list's first entry for the wave's tokens is on its way while the row is looked up.)
        const int64_t first = static_cast<int64_t>(share.split) * shares.len + (ALONE ? 0 : wave * 32) + (lane & 31);
        first_entry = list[min(divide(static_cast<int>(min(first, int64_t{INT32_MAX})), pg.by_bs), shares.budget - 1)];
        if (!chosen_of(a, shares, row, share, seq, count))
            return;
    } else {
        if (!share_of(a, shares, blockIdx.x, false, share) || !sequence(a.batch, share.b, pg.err, seq))
            return;
    }
    const int b = share.b;
    const int rows = seq.nq * a.group, row0 = tile * 16 * NT;
    if (row0 >= rows)
        return;
    const int i0 = divide(row0, a.by_group), i1 = divide(min(row0 + 16 * NT, rows) - 1, a.by_group) + 1;
    const Span span = LISTED ? Span{0, 0, count * pg.BS} : span_of(seq.n, seq.nq, i0, i1, a.window);
    const int64_t part_at = (LISTED ? 0 : span_of(seq.n, seq.nq, 0, seq.nq, a.window).start) +
                            static_cast<int64_t>(share.split) * share.len;
    const int begin = static_cast<int>(min(part_at, int64_t{INT32_MAX} - 1023));
    const int stop = static_cast<int>(min(part_at + share.len, static_cast<int64_t>(span.end)));
    const bool whole = share.parts == 1;
    const int p_first = seq.n - seq.nq + i0;
    const int low_last = a.window > 0 ? span.end - a.window : 0;  // from here on every row's window is open

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

    // Page of token base + lane % 32, and where that token's row is (-1: none that a row sees).  LISTED: tokens are
    // counted along the list, and `entry` is the list's page for that one.
    auto entry_at = [&](int base) {
        if constexpr (LISTED)
            return list[min(divide(min(base + (lane & 31), stop - 1), pg.by_bs), count - 1)];
        else
            return 0;
    };
    auto page_at = [&](int base, int entry, int &page, bool &shown) {
        const int t = base + (lane & 31);
        if constexpr (LISTED) {
            page = entry;
            shown = t < stop && entry >= 0 && entry < a.batch.table_len;
            if (t < stop && !shown)
                report(pg.err, KV_ASYNC_BAD_BATCH);
            // (A page that lies before the window may have no block, or one without a scale.)
            const int64_t start = static_cast<int64_t>(entry) * pg.BS;
            shown = shown && start <= p_first && (a.window == 0 || p_first - (start + pg.BS - 1) < a.window);
        } else {
            page = divide(t, pg.by_bs);
            shown = t < stop && (page + 1) * static_cast<int64_t>(pg.BS) > span.first;
        }
        return shown ? table[page] : 0;
    };
    auto slot_of = [&](int t, int page) { return t - (LISTED ? divide(t, pg.by_bs) : page) * pg.BS; };
    auto offset_at = [&](int base, int page, bool shown, int block) -> int64_t {
        if (!shown || !in_cache(pg, block))
            return -1;
        return block * pg.block_stride + static_cast<uint32_t>(slot_of(base + (lane & 31), page)) * pg.token_bytes;
    };
    // The exponents of a token's scales, K's and V's; 0 (a factor of 0) for none.
    auto exponents_at = [&](int64_t off, int block, int &k_exponent, int &v_exponent) {
        if constexpr (SCALED) {
            const bool has = a.scales.data != nullptr;
            k_exponent = off < 0 ? 0 : has ? *scale_at(a.scales, block, 0, h) : 127;
            v_exponent = off < 0 ? 0 : has ? *scale_at(a.scales, block, 1, h) : 127;
        }
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

    constexpr int kStride = 32 * TEAM;
    int base = begin + (ALONE ? 0 : wave * 32);
    if (base < stop) {
        int page, next_page = 0, next_block = 0, next_entry = 0;
        [[maybe_unused]] int k_exponent = 0, v_exponent = 0;
        bool shown, next_shown = false;
        int block = page_at(base, first_entry, page, shown);
        int64_t off = offset_at(base, page, shown, block);
        if (stop - base > kStride) {
            next_block = page_at(base + kStride, entry_at(base + kStride), next_page, next_shown);
            if (LISTED && stop - base > 2 * kStride)
                next_entry = entry_at(base + 2 * kStride);
        }
        load_k(off);
        exponents_at(off, block, k_exponent, v_exponent);
        load_v(off);
        while (true) {
            const int t_lane = base + (lane & 31);
            [[maybe_unused]] const int real = LISTED && off >= 0 ? page * pg.BS + slot_of(t_lane, page) : t_lane;
            const bool use = LISTED ? off >= 0 && t_lane < stop && real <= p_first &&
                                          (a.window == 0 || p_first - real < a.window)
                                    : off >= 0 && t_lane >= span.first && t_lane < stop;
            const uint32_t usable = static_cast<uint32_t>(__ballot(use));
            const bool edge = usable != 0xffffffffu || (!LISTED && (p_first - base < 31 || base < low_last));
            const bool more = stop - base > kStride;
            // The scales of the tokens of this lane's scores.
            [[maybe_unused]] float k_by[8], v_by[8];
            if constexpr (SCALED) {
                if (by_8) {
                    k_by[0] = power_of(__shfl(k_exponent, g * 8));
                    v_by[0] = power_of(__shfl(v_exponent, g * 8));
#pragma unroll
                    for (int e = 1; e < 8; ++e) {
                        k_by[e] = k_by[0];
                        v_by[e] = v_by[0];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        k_by[e] = power_of(__shfl(k_exponent, g * 8 + e));
                        v_by[e] = power_of(__shfl(v_exponent, g * 8 + e));
                    }
                }
            }
            // Their distances from the query's token, where slopes need them.
            [[maybe_unused]] int far[8];
            if constexpr (LISTED)
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        far[e] = p_first - __shfl(real, g * 8 + e);
                }

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
                exponents_at(next_off, next_block, k_exponent, v_exponent);
                page = next_page;
                if (stop - base > 2 * kStride) {
                    next_block = page_at(base + 2 * kStride, next_entry, next_page, next_shown);
                    if (LISTED && stop - base > 3 * kStride)
                        next_entry = entry_at(base + 3 * kStride);
                }
            }

            // Weights.  Everything from here on is in powers of 2.
            u32x4 p[NT], p_rest[NT];
            const uint32_t bits = usable >> (g * 8);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = SCALED ? s[nt][e >> 2][e & 3] * k_by[e] : s[nt][e >> 2][e & 3];
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
                        x[e] -= slope[nt] * static_cast<float>(LISTED ? far[e] : p_of[nt] - (base + g * 8 + e));
                }
                if (edge) {
                    const int to = p_of[nt] - (base + g * 8) + 1, from = a.window > 0 ? to - a.window : INT32_MIN;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (bits >> e & 1) && (LISTED || (e < to && e >= from)) ? x[e] : -INFINITY;
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
                const float zero = m[nt] - W::kShift;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = __builtin_amdgcn_exp2f(x[e] - zero);
                l[nt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                if constexpr (SCALED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] *= v_by[e];
                }
                // A weight is two numbers of the rows' type, so that its rounding does not add to the output's: the
                // products wait for memory anyway.
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const uint32_t w = W::pack(x[e], x[e + 1]);
                    p[nt][e / 2] = w;
                    p_rest[nt][e / 2] = W::pack(x[e] - W::low(w), x[e + 1] - W::high(w));
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
                            turned[0][e] = W::from_e4m3(lo, false);
                            turned[1][e] = W::from_e4m3(lo, true);
                            turned[2][e] = W::from_e4m3(hi, false);
                            turned[3][e] = W::from_e4m3(hi, true);
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
                            x = mfma_16x16x32(turned[j], p[nt], x, W{});
                            x = mfma_16x16x32(turned[j], p_rest[nt], x, W{});
                        }
                }
            if (!more)
                break;
            load_v(next_off);
            off = next_off;
            base += kStride;
        }
    }

    if constexpr (ALONE) {
        // (A row's columns are in the lanes of its column, 4 times VE of each 64 in each.)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            l[nt] += __shfl_xor(l[nt], 16);
            l[nt] += __shfl_xor(l[nt], 32);
            const int r = row0 + nt * 16 + c;
            if (r >= rows)
                continue;
            const int head = h * a.group + r, row = seq.q0;
            const float inv = l[nt] == 0.f ? 0.f : a.v_scale / l[nt];
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int d = v * 16 * VE + (g * 4 + k) * VE;
                    if (d >= pg.D)
                        continue;
                    uint8_t *to = a.out.data + row * a.out.token_stride + head * a.out.head_stride + 2 * d;
#pragma unroll
                    for (int j = 0; j < VE; j += 4) {
                        const f32x4 *x = acc[nt] + v * VE + j;
                        *reinterpret_cast<u32x2 *>(to + 2 * j) =
                            u32x2{T::pack(x[0][k] * inv, x[1][k] * inv), T::pack(x[2][k] * inv, x[3][k] * inv)};
                    }
                }
            if (g == 0)
                a.lse[static_cast<int64_t>(row) * a.heads + head] =
                    l[nt] == 0.f ? -INFINITY : (m[nt] - W::kShift + __builtin_amdgcn_logf(l[nt])) * kLn2;
        }
        return;
    } else {
        // Join the waves: every wave's largest score and sum, then wave w collects component w of every tile, which are
        // VE consecutive columns per lane.
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
            const int64_t slot = slot_in(shares, h, r, static_cast<int64_t>(row) * a.heads + head, share.split);
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
                        total[nt] == 0.f ? -INFINITY : (most[nt] - W::kShift + __builtin_amdgcn_logf(total[nt])) * kLn2;
                } else {
                    shares.stats[slot * 2] = most[nt] - W::kShift;
                    shares.stats[slot * 2 + 1] = total[nt];
                }
            }
        }
    }
}

template <class T, bool FP8, int DP, int NT, bool SCALED, class From>
hipError_t launch_tiles(const AttendArgs &a, const From &from, int items, int max_rows, hipStream_t stream) {
    const int tiles = (max_rows + 16 * NT - 1) / (16 * NT);
    const int groups = std::is_same_v<From, Alone> ? (items + kWaves - 1) / kWaves : items;
    const dim3 grid = std::is_base_of_v<Chosen, From> ? dim3(groups * a.pages.H, tiles) : dim3(groups, tiles * a.pages.H);
    return launch_kernel(step_kernel<T, FP8, DP, NT, SCALED, From>, grid, 64 * kWaves, stream, a, from);
}

// `items` workgroups (Alone: waves) for each KV head and tile of up to max_rows rows.
template <class T, bool FP8, bool SCALED, class From>
hipError_t launch_rows(const AttendArgs &a, const From &from, int items, int max_rows, hipStream_t stream) {
    const bool two = step_tile_rows(max_rows, a.pages.D) == 32;
    if (a.pages.D > 128)
        return launch_tiles<T, FP8, 256, 1, SCALED>(a, from, items, max_rows, stream);
    if (a.pages.D > 64)
        return two ? launch_tiles<T, FP8, 128, 2, SCALED>(a, from, items, max_rows, stream)
                   : launch_tiles<T, FP8, 128, 1, SCALED>(a, from, items, max_rows, stream);
    return two ? launch_tiles<T, FP8, 64, 2, SCALED>(a, from, items, max_rows, stream)
               : launch_tiles<T, FP8, 64, 1, SCALED>(a, from, items, max_rows, stream);
}

}  // namespace

}  // namespace kvx
