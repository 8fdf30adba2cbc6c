// Rows of 2-byte elements, 8 to a lane: as numbers, normed and rotated, and as e4m3.
#pragma once

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

// Rounded to nearest even.
template <int DTYPE>
__device__ __forceinline__ uint32_t two_bytes(float x) {
    if constexpr (DTYPE == KV_DTYPE_BF16)
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    else
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
}

template <int DTYPE>
__device__ __forceinline__ vec16 from_floats(const float *y) {
    vec16 x;
#pragma unroll
    for (int w = 0; w < 4; ++w)
        x[w] = two_bytes<DTYPE>(y[2 * w]) | two_bytes<DTYPE>(y[2 * w + 1]) << 16;
    return x;
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
    kHalves,      // (i, i + half), half a multiple of 8: a lane's partners are 8 consecutive columns too
    kAnyHalves,   // (i, i + half), any half
};

// Cosine and sine of position * freq radians.  The angle is taken in turns and in 64 bits, and what is left of it
// without the whole turns is small, so far positions lose nothing: it is off by 2^-52 of the turns.
__device__ __forceinline__ void turn_by(int position, double freq, float magnitude, float &cosine, float &sine) {
    const double turns = position * (freq * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    cosine = c * magnitude;
    sine = s * magnitude;
}

// Lane `vec` of LPR has columns d0 = 8 * vec on (none if `any` is not set).
template <int DTYPE, Pairs PAIRS, int LPR>
struct Turner {
    int d0, other0;  // columns: the lane's first, and of kHalves its partners' first
    bool any, turned;

    __device__ __forceinline__ Turner(const Turn &t, int vec, int D) {
        d0 = vec * 8;
        any = d0 < D;
        turned = any && d0 < t.rotary;
        other0 = d0 < t.half ? d0 + t.half : d0 - t.half;
    }

    // A column's partner under kAnyHalves, itself beyond the rotated ones.
    static __device__ __forceinline__ int partner(const Turn &t, int d) {
        return d >= t.rotary ? d : d < t.half ? d + t.half : d - t.half;
    }

    struct Vec {
        vec16 own, other;
    };

    __device__ __forceinline__ Vec load(const Turn &t, const uint8_t *row) const {
        Vec v{vec16{0, 0, 0, 0}, vec16{0, 0, 0, 0}};
        if (any)
            v.own = *reinterpret_cast<const vec16 *>(row + 2 * d0);
        if constexpr (PAIRS == kHalves) {
            if (turned)
                v.other = *reinterpret_cast<const vec16 *>(row + 2 * other0);
        } else if constexpr (PAIRS == kAnyHalves) {
            if (turned) {
                const uint16_t *x = reinterpret_cast<const uint16_t *>(row);
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    v.other[w] = x[partner(t, d0 + 2 * w)] | static_cast<uint32_t>(x[partner(t, d0 + 2 * w + 1)]) << 16;
            }
        }
        return v;
    }

    // The norm's weights of the lane's columns and of their partners.
    struct Weights {
        float own[8], other[8];
    };

    static __device__ __forceinline__ float weight(const Turn &t, int d) {
        const float w = t.weight_f32 ? static_cast<const float *>(t.weight)[d]
                                     : to_float(static_cast<const uint16_t *>(t.weight)[d], DTYPE);
        return w + t.offset;
    }

    __device__ __forceinline__ Weights weights(const Turn &t) const {
        Weights w;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w.own[j] = t.weight && any ? weight(t, d0 + j) : 1.f;
            w.other[j] = 1.f;
            if (PAIRS == kHalves || PAIRS == kAnyHalves)
                w.other[j] = t.weight && turned ? weight(t, PAIRS == kHalves ? other0 + j : partner(t, d0 + j)) : 1.f;
        }
        return w;
    }

    // The pair that the lane's column d0 + j belongs to.
    __device__ __forceinline__ int pair(const Turn &t, int j) const {
        const int d = d0 + j;
        return PAIRS == kNeighbours ? d >> 1 : d < t.half ? d : d - t.half;
    }

    // angle(j, cosine, sine): of pair(j), asked for where the column is turned.  All lanes of a row take part.
    template <class Angle>
    __device__ __forceinline__ void finish(const Turn &t, const Vec &v, const Weights &w, Angle &&angle, float *y) const {
        to_floats<DTYPE>(v.own, y);
        if constexpr (PAIRS == kAsIs)
            return;
        float z[8];
        to_floats<DTYPE>(v.other, z);
        if (t.weight) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                sum = fmaf(y[j], y[j], sum);
#pragma unroll
            for (int o = LPR / 2; o; o >>= 1)
                sum += __shfl_xor(sum, o);
            const float inv = 1.f / sqrtf(fmaf(sum, t.mean, t.eps));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = y[j] * inv * w.own[j];
                z[j] = z[j] * inv * w.other[j];
            }
        }
        if (!turned)
            return;
        if constexpr (PAIRS == kNeighbours) {
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                if (d0 + j < t.rotary) {
                    float c, s;
                    angle(j, c, s);
                    const float a = y[j], b = y[j + 1];
                    y[j] = a * c - b * s;
                    y[j + 1] = b * c + a * s;
                }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (PAIRS == kHalves || d0 + j < t.rotary) {
                    float c, s;
                    angle(j, c, s);
                    y[j] = y[j] * c + (d0 + j < t.half ? -z[j] : z[j]) * s;
                }
        }
    }
};

// Lanes of a row of D columns, as a power of two.
inline int lanes_of(int D) { return D > 128 ? 32 : D > 64 ? 16 : 8; }

// kv_append_scaled's kernel, with K normed and rotated where `turn` is given (and pairs are not kAsIs).
kv_status launch_append_scaled(const Pages &pages, const Batch &batch, int32_t num_seqs, const Rows &k, const Rows &v,
                               int32_t dtype, const Scales &scales, const Turn &turn, Pairs pairs, hipStream_t stream);
// Checks that kv_append and kv_append_scaled share: the sizes and types of k and v.
kv_status check_append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k, const kv_rows *v,
                       int32_t cache_dtype);
kv_status check_factors(int32_t cache_dtype, float k_scale, float v_scale);

}  // namespace kvx
