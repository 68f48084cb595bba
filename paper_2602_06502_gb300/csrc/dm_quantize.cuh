// dm_quantize.cuh -- a row's values in 8 bits.
//
// The product with 127 / top is off by less than 2^-16 and gives a step r.  What
// is left, 127 x - r top, is exact in 32 bits (x and top have up to 11 bits), and
// where it is about half of top or more it corrects r: q is what the formula
// says to the last case.
#pragma once

#include "dm_cache.cuh"

namespace dm {

template <class T>
struct Two;
template <>
struct Two<__nv_bfloat16> {
    using type = __nv_bfloat162;
    static __device__ __forceinline__ float2 up(type x) { return __bfloat1622float2(x); }
    static __device__ __forceinline__ type down(float a, float b) { return __floats2bfloat162_rn(a, b); }
};
template <>
struct Two<__half> {
    using type = __half2;
    static __device__ __forceinline__ float2 up(type x) { return __half22float2(x); }
    static __device__ __forceinline__ type down(float a, float b) { return __floats2half2_rn(a, b); }
};

template <class T>
__device__ __forceinline__ void unpack(const uint4 &x, float *f) {
    const auto *p = reinterpret_cast<const typename Two<T>::type *>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = Two<T>::up(p[i]);
        f[2 * i] = y.x;
        f[2 * i + 1] = y.y;
    }
}

__device__ __forceinline__ float score_at(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float score_at(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ float score_at(const float *p) { return *p; }

// The largest of the sizes in a and b, two 16-bit values each: without their
// signs the bits of floating-point numbers are in their order, and what is not
// finite is above the rest.
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) { return __vmaxu2(a, b & 0x7FFF7FFFu); }

// Added to a number below 2^22 it leaves that number, rounded to even, in the low bits.
constexpr float kRound = 12582912.f;

// What a row's steps need of its largest size.
struct RowStep {
    float by, shift, big;   // 127 / top; a power of two that keeps that and 127 x in range; top, so shifted
    uint32_t keep;          // 0 where a value is not finite: all steps are zero then
};

// bits: of the row's largest size; the scale is NaN where a value is not finite.
template <class T>
__device__ __forceinline__ RowStep row_step(uint32_t bits, float &scale) {
    constexpr uint32_t kFinite = std::is_same_v<T, __half> ? 0x7C00 : 0x7F80;
    const uint16_t low = (uint16_t)bits;
    const bool finite = bits < kFinite;
    const float top = score_at(reinterpret_cast<const T *>(&low));
    scale = finite ? __fdiv_rn(top, 127.f) : __int_as_float(0x7FC00000);
    RowStep s;
    s.shift = top > 1e30f ? 0x1p-64f : top < 1e-30f ? 0x1p64f : 1.f;
    s.big = top * s.shift;
    s.by = bits == 0 || !finite ? 0.f : __fdiv_rn(127.f, s.big);
    s.keep = finite ? ~0u : 0u;
    return s;
}

// Whether a row's squares add up as they are: where its largest value is between
// 2^-48 and 2^50, up to 2^24 of them neither overflow nor lose what counts.  So for
// every half, and for nearly every row.
template <class T>
__device__ __forceinline__ bool plain_squares(uint32_t bits) {
    return std::is_same_v<T, __half> ? bits != 0 : bits - 0x2780u <= 0x5880u - 0x2780u;
}
// Whether they add up after a shift: else the row is zeros or not finite, and its
// scale, 0 or NaN, is the same with any norm.
template <class T>
__device__ __forceinline__ bool far_squares(uint32_t bits) {
    return !std::is_same_v<T, __half> && bits != 0 && bits < 0x7F80;
}
// By what its values are multiplied then, and its scale: `mean` is that of the
// squares so shifted.
__device__ __forceinline__ float far_shift(uint32_t bits) { return bits > 0x5880 ? 0x1p-100f : 0x1p96f; }
__device__ __forceinline__ float far_scale(uint32_t bits, float mean, float eps) {
    const float shift = far_shift(bits), top = __fdiv_rn(__uint_as_float(bits << 16) * shift, 127.f), more = eps * shift * shift;
    // the mean is at most 2^96, so it does not count beside 2^124
    return more < 0x1p124f ? top * rsqrtf(mean + more) : top * rsqrtf(eps) * 0x1p-96f;
}

// kRound + the steps of eight values, as bits.
template <class T>
__device__ __forceinline__ void steps8(uint4 v, const RowStep &s, uint32_t *n) {
    float f[8], far = 0.f;
    v.x &= s.keep, v.y &= s.keep, v.z &= s.keep, v.w &= s.keep;
    unpack<T>(v, f);
    if (s.shift != 1.f)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= s.shift;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __fmaf_rn(f[i], s.by, kRound);
        n[i] = __float_as_uint(y);
        far = fmaxf(far, fabsf(__fmaf_rn(f[i], s.by, kRound - y)));
    }
    if (far > 0.5f - 0x1p-15f) {
        const float half = 0.5f * s.big;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __fmaf_rn(kRound - __uint_as_float(n[i]), s.big, 127.f * f[i]);
            const uint32_t odd = n[i] & 1;   // ties to even
            if (e > half || (e == half && odd)) ++n[i];
            else if (e < -half || (e == -half && odd)) --n[i];
        }
    }
}

// Those steps as halves: 1536 + a step is a half with the step in its low bits.
__device__ __forceinline__ uint4 halves8(const uint32_t *n) {
    const __half2 minus = __half2half2(__ushort_as_half(0x6600));
    uint4 y;
    uint32_t *w = reinterpret_cast<uint32_t *>(&y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (n[2 * i] + 0x6600u & 0xFFFFu) | (n[2 * i + 1] + 0x6600u) << 16;
        const __half2 z = __hsub2(*reinterpret_cast<const __half2 *>(&two), minus);
        w[i] = *reinterpret_cast<const uint32_t *>(&z);
    }
    return y;
}

}  // namespace dm
