// Rows of 2-byte elements, 8 to a lane: as numbers, normed and rotated, and as e4m3.
#pragma once

#include <type_traits>

#include "kvx_paged.h"

namespace kvx {

typedef uint32_t vec16 __attribute__((ext_vector_type(4)));
typedef uint32_t vec8 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_float(uint32_t bits, int dtype) {
    return dtype == KV_DTYPE_BF16 ? __builtin_bit_cast(float, bits << 16)
                                  : static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}

// Clamped to e4m3's largest value; NaN stays.
__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }

template <int DTYPE>
__device__ __forceinline__ void to_floats(const vec16 &x, float *y) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        y[2 * w] = to_float(x[w] & 0xffff, DTYPE);
        y[2 * w + 1] = to_float(x[w] >> 16, DTYPE);
    }
}

// Two numbers, rounded to nearest even.
template <int DTYPE>
__device__ __forceinline__ uint32_t pack_two(float low, float high) {
    if constexpr (DTYPE == KV_DTYPE_BF16) {
        typedef __bf16 pair __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, pair{static_cast<__bf16>(low), static_cast<__bf16>(high)});
    } else {
        typedef _Float16 pair __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, pair{static_cast<_Float16>(low), static_cast<_Float16>(high)});
    }
}

template <int DTYPE>
__device__ __forceinline__ vec16 from_floats(const float *y) {
    return vec16{pack_two<DTYPE>(y[0], y[1]), pack_two<DTYPE>(y[2], y[3]), pack_two<DTYPE>(y[4], y[5]),
                 pack_two<DTYPE>(y[6], y[7])};
}

// Of 8 numbers, each rounded once.
__device__ __forceinline__ vec8 to_e4m3(const float *y) {
    vec8 x;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int packed = 0;
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * w]), clamp_e4m3(y[4 * w + 1]), packed, false);
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * w + 2]), clamp_e4m3(y[4 * w + 3]), packed, true);
        x[w] = static_cast<uint32_t>(packed);
    }
    return x;
}

// How kv_rotate norms and rotates a row of q or k.
struct Turn {
    const double *freqs;
    const int32_t *positions;
    const void *weight;  // NULL: not normed
    int32_t weight_f32;
    float eps, offset, magnitude, mean;  // mean: 1 / D
    int32_t rotary, half;
};

// Which columns are turned with each other, where a lane has 8 consecutive ones.
enum Pairs {
    kAsIs,        // none, and no norm
    kNeighbours,  // (2i, 2i + 1)
    kHalves,      // (i, i + half), half a multiple of 8: a lane's partners are another lane's columns, one for one
    kAnyHalves,   // (i, i + half), any half: the lane loads them too
};

// Weight d of a norm, which is there.
template <int DTYPE>
__device__ __forceinline__ float norm_weight(const Turn &t, int d) {
    const float w = t.weight_f32 ? static_cast<const float *>(t.weight)[d]
                                 : to_float(static_cast<const uint16_t *>(t.weight)[d], DTYPE);
    return w + t.offset;
}

// Cosine and sine of position * freq radians.  The angle is taken in turns and in 64 bits, and what is left of it
// without the whole turns is small, so far positions lose nothing: it is off by 2^-52 of the turns.
__device__ __forceinline__ void turn_by(int position, double freq, float magnitude, float &cosine, float &sine) {
    const double turns = position * (freq * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    cosine = c * magnitude;
    sine = s * magnitude;
}

// Sum over a group of LPR lanes (lanes of 16 by moves inside the vector unit, which cost nothing beside an LDS
// shuffle).
template <int LPR>
__device__ __forceinline__ float sum_over(float x) {
    const auto moved = [](float y, auto control) {
        constexpr int kControl = decltype(control)::value;
        return __builtin_bit_cast(
            float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), kControl, 0xf, 0xf, true));
    };
    x += moved(x, std::integral_constant<int, 0xb1>{});   // lane ^ 1
    x += moved(x, std::integral_constant<int, 0x4e>{});   // lane ^ 2
    x += moved(x, std::integral_constant<int, 0x141>{});  // 7 - lane, of 8
    if constexpr (LPR >= 16)
        x += moved(x, std::integral_constant<int, 0x140>{});  // 15 - lane, of 16
    if constexpr (LPR >= 32)
        x += __shfl_xor(x, 16);
    return x;
}

// 1 / sqrt(x), off by a unit of the last place, also where x is so small that the instruction takes it for 0.
__device__ __forceinline__ float inverse_root(float x) {
    return x < 0x1p-96f ? 0x1p32f * __builtin_amdgcn_rsqf(x * 0x1p64f) : __builtin_amdgcn_rsqf(x);
}

// Lane `vec` of LPR has columns d0 = 8 * vec on (none if `any` is not set).
template <int DTYPE, Pairs PAIRS, int LPR>
struct Turner {
    int d0;
    bool any, turned;
    int other;  // kHalves: the lane that has the partners

    __device__ __forceinline__ Turner(const Turn &t, int vec, int D) {
        d0 = vec * 8;
        any = d0 < D;
        turned = any && d0 < t.rotary;
        const int lane = static_cast<int>(threadIdx.x & 63);
        other = !turned ? lane : d0 < t.half ? lane + t.half / 8 : lane - t.half / 8;
    }

    // A column's partner under kAnyHalves, itself beyond the rotated ones.
    static __device__ __forceinline__ int partner(const Turn &t, int d) {
        return d >= t.rotary ? d : d < t.half ? d + t.half : d - t.half;
    }

    struct Vec {
        vec16 own, other;  // other: kAnyHalves alone
    };

    __device__ __forceinline__ Vec load(const Turn &t, const uint8_t *row) const {
        Vec v;
        v.own = any ? *reinterpret_cast<const vec16 *>(row + 2 * d0) : vec16{0, 0, 0, 0};
        if constexpr (PAIRS == kAnyHalves) {
            v.other = v.own;
            if (turned) {
                const uint16_t *x = reinterpret_cast<const uint16_t *>(row);
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    v.other[w] = x[partner(t, d0 + 2 * w)] | static_cast<uint32_t>(x[partner(t, d0 + 2 * w + 1)]) << 16;
            }
        }
        return v;
    }

    // The norm's weights of the lane's columns, and under kAnyHalves of their partners.  weight(column)
    struct Weights {
        float own[8], other[PAIRS == kAnyHalves ? 8 : 1];
    };
    template <class Weight>
    __device__ __forceinline__ Weights weights(const Turn &t, Weight &&weight) const {
        Weights w;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w.own[j] = weight(any ? d0 + j : 0);
            if constexpr (PAIRS == kAnyHalves)
                w.other[j] = weight(turned ? partner(t, d0 + j) : 0);
        }
        return w;
    }

    // The pair that the lane's column d0 + j belongs to.
    __device__ __forceinline__ int pair(const Turn &t, int j) const {
        const int d = d0 + j;
        return PAIRS == kNeighbours ? d >> 1 : d < t.half ? d : d - t.half;
    }

    // Cosines and sines of the lane's columns, of which kNeighbours has every other one.  (Of halves, a first column's
    // sine is negative: it loses what its partner gains.)
    static constexpr int kAngles = PAIRS == kNeighbours ? 4 : 8;
    struct Angles {
        float cosine[kAngles], sine[kAngles];
    };

    // angle(pair, cosine, sine)
    template <class Angle>
    __device__ __forceinline__ Angles angles(const Turn &t, Angle &&angle) const {
        Angles a;
#pragma unroll
        for (int j = 0; j < kAngles; ++j) {
            const int at = PAIRS == kNeighbours ? 2 * j : j;
            a.cosine[j] = 1.f;
            a.sine[j] = 0.f;
            if (turned && d0 + at < t.rotary)
                angle(pair(t, at), a.cosine[j], a.sine[j]);
            if (PAIRS != kNeighbours && d0 + at < t.half)
                a.sine[j] = -a.sine[j];
        }
        return a;
    }

    // kHalves: of cosines and sines of the lane's pairs, whatever they are where it is not turned, its columns'.
    __device__ __forceinline__ void settle(const Turn &t, Angles &a) const {
#pragma unroll
        for (int j = 0; j < kAngles; ++j) {
            a.cosine[j] = turned ? a.cosine[j] : 1.f;
            a.sine[j] = !turned ? 0.f : d0 < t.half ? -a.sine[j] : a.sine[j];
        }
    }

    // The lane's columns of a row, normed if `norm` (else all weights are 1), and turned.  All lanes of a row take
    // part.
    __device__ __forceinline__ void finish(const Turn &t, const Vec &v, bool norm, const Weights &w, const Angles &a,
                                           float *y) const {
        to_floats<DTYPE>(v.own, y);
        if constexpr (PAIRS == kAsIs)
            return;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum = fmaf(y[j], y[j], sum);
        const float inv = norm ? inverse_root(fmaf(sum_over<LPR>(sum), t.mean, t.eps)) : 1.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = y[j] * inv * w.own[j];
        float z[8];
        if constexpr (PAIRS == kNeighbours) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float p = y[j], q = y[j + 1], c = a.cosine[j / 2], s = a.sine[j / 2];
                z[j] = p * c - q * s;
                z[j + 1] = q * c + p * s;
            }
        } else {
            if constexpr (PAIRS == kAnyHalves) {
                to_floats<DTYPE>(v.other, z);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    z[j] = z[j] * inv * w.other[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    z[j] = __shfl(y[j], other);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                z[j] = y[j] * a.cosine[j] + z[j] * a.sine[j];
        }
        // (Columns that are not turned stay what they are, infinities too.)
        if (t.rotary < 8 * LPR) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                z[j] = d0 + j < t.rotary ? z[j] : y[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = z[j];
    }
};

// Lanes of a row of D columns, as a power of two.
inline int lanes_of(int D) { return D > 128 ? 32 : D > 64 ? 16 : 8; }

// What it takes of a batch: refused before anything is enqueued.
kv_status check_append_scaled(const kv_cache *cache, const kv_batch *batch);
// kv_append_scaled's kernel, with K normed and rotated where `turn` is given (and pairs are not kAsIs).
hipError_t launch_append_scaled(const Pages &pages, const Batch &batch, int32_t num_seqs, const Rows &k, const Rows &v,
                                int32_t dtype, const Scales &scales, const Turn &turn, Pairs pairs, hipStream_t stream);
// Checks that kv_append and kv_append_scaled share: the sizes and types of k and v.
kv_status check_append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k, const kv_rows *v,
                       int32_t cache_dtype);
kv_status check_factors(int32_t cache_dtype, float k_scale, float v_scale);

}  // namespace kvx
