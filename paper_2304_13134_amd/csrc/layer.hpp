// Helpers of the layer between an encoder's frames and the lattice: element types, activations, values in 8 bits in
// blocks of 32 columns, and which frames exist.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/last.h"
#include "common.hpp"

namespace last {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// Rows begin wherever an element may, e.g. those of 257 columns: memory takes vectors at any address, and what is aligned is
// no slower for it (one instruction either way).
typedef f4 f4_any __attribute__((aligned(4)));
typedef u4 u4_any __attribute__((aligned(2)));
typedef h8 h8_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(1)));
typedef u4 u4_byte __attribute__((aligned(1)));

struct bf16_t { uint16_t bits; };
struct f16_t { _Float16 v; };
struct i8_t { int8_t v; };
struct e4m3_t { uint8_t bits; };

constexpr int kBlock = 32;           // columns that share a scale

// n / d for n < 2^31 as n m 2^-(31 + s) with s = ceil(log2 d), m = ceil(2^(31 + s) / d): m d passes 2^(31 + s) by less than d <= 2^s,
// so the quotient is off by less than n 2^-31 / d < 1 / d and its integer part is right.  (A division takes some 20 instructions, a
// quarter of them at a quarter of the rate: as much as the rest of what eight values kept in 8 bits take.)
struct Divisor {
    unsigned m, s;
};

inline Divisor divisor_of(unsigned d)
{
    unsigned s = 0;
    while ((1ull << s) < d) ++s;
    return Divisor{d ? (unsigned)(((1ull << (31 + s)) + d - 1) / d) : 0u, s};
}

__device__ __forceinline__ unsigned quotient(unsigned n, const Divisor& d) { return __umulhi(n + n, d.m) >> d.s; }

// rows b T + t of frames; those with t >= len[b] do not exist (lengths below 0 count as 0)
struct Frames {
    const int* len;                  // null: all exist
    int T;
    Divisor by;                      // T
};

__device__ __forceinline__ bool frame_exists(const Frames& f, int row)
{
    if (!f.len) return true;
    const int b = (int)quotient((unsigned)row, f.by);
    return row - b * f.T < f.len[b];
}

__device__ __forceinline__ float bf16_to_float(unsigned bits) { return __uint_as_float(bits << 16); }

// two float32 to bfloat16, to nearest even, NaN stays NaN
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(unsigned, r);
}

__device__ __forceinline__ unsigned f16_pair(float lo, float hi)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 r = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(unsigned, r);
}

// ---- scales of 8-bit values: byte = exponent + 127, 255 = the block holds a value that is not finite

__device__ __forceinline__ float scale_value(unsigned byte)
{
    const unsigned bits = byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23;
    return __uint_as_float(bits);
}

// the smallest exponent (from -127) at which the largest magnitude, given as its bits, does not pass the largest code:
// 127 = 1.984375 2^6, 448 = 1.75 2^8
template <bool E4M3>
__device__ __forceinline__ unsigned scale_byte(unsigned top)
{
    if (top >= 0x7f800000u) return 255u;
    const int b = (int)(top >> 23) - (E4M3 ? 8 : 6) + ((top & 0x7fffffu) > (E4M3 ? 0x600000u : 0x7e0000u) ? 1 : 0);
    return b < 0 ? 0u : (unsigned)b;
}

// four values times 1 / scale to four codes, to nearest even; 0 where the block holds a value that is not finite
template <bool E4M3>
__device__ __forceinline__ unsigned encode4(const float* v, unsigned byte)
{
    const float m = __uint_as_float((254u - byte) << 23);
    unsigned r;
    if constexpr (E4M3) {
        r = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[0] * m, v[1] * m, 0, false);
        r = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * m, v[3] * m, (int)r, true);
    } else {
        // v m is exact and at most 127; added to 1.5 2^23, whose neighbours are 1 apart, it is rounded to an integer, whose last eight
        // bits are the sum's
        unsigned c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(__builtin_fmaf(v[i], m, 12582912.f));
        r = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
    }
    return byte == 255u ? 0u : r;
}

template <bool E4M3>
__device__ __forceinline__ void decode4(unsigned q, float scale, float* v)
{
    if constexpr (E4M3) {
        v[0] = __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * scale;
        v[1] = __builtin_amdgcn_cvt_f32_fp8((int)q, 1) * scale;
        v[2] = __builtin_amdgcn_cvt_f32_fp8((int)q, 2) * scale;
        v[3] = __builtin_amdgcn_cvt_f32_fp8((int)q, 3) * scale;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(q >> (8 * i)) * scale;
    }
}

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ unsigned umax(unsigned a, unsigned b) { return a > b ? a : b; }

// ---- eight consecutive elements of a row; n of them exist (the others read as 0 and are not written)

template <typename E> struct Elt;
template <> struct Elt<float> {
    static constexpr int type = LAST_F32, size = 4;
    static __device__ void put(void* p, size_t i, float v) { ((float*)p)[i] = v; }
    static __device__ void put8(void* p, size_t i, const float* v)
    {
        *(f4_any*)((float*)p + i) = f4{v[0], v[1], v[2], v[3]};
        *(f4_any*)((float*)p + i + 4) = f4{v[4], v[5], v[6], v[7]};
    }
};
template <> struct Elt<bf16_t> {
    static constexpr int type = LAST_BF16, size = 2;
    static __device__ void put(void* p, size_t i, float v) { ((uint16_t*)p)[i] = (uint16_t)bf16_pair(v, 0.f); }
    static __device__ void put8(void* p, size_t i, const float* v)
    {
        *(u4_any*)((uint16_t*)p + i) = u4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    }
};
template <> struct Elt<f16_t> {
    static constexpr int type = LAST_F16, size = 2;
    static __device__ void put(void* p, size_t i, float v) { ((_Float16*)p)[i] = (_Float16)v; }
    static __device__ void put8(void* p, size_t i, const float* v)
    {
        *(u4_any*)((_Float16*)p + i) = u4{f16_pair(v[0], v[1]), f16_pair(v[2], v[3]), f16_pair(v[4], v[5]), f16_pair(v[6], v[7])};
    }
};
// codes of 8-bit values; the caller brings the scale of their block
template <bool E4M3> struct EltCodes {
    static constexpr int type = E4M3 ? LAST_E4M3 : LAST_I8, size = 1;
};
template <> struct Elt<i8_t> : EltCodes<false> {};
template <> struct Elt<e4m3_t> : EltCodes<true> {};

// as they stand in memory: to be sent for ahead of their use
template <typename E> struct Raw {
    u4 a;
};
template <> struct Raw<float> {
    u4 a, b;
};
template <> struct Raw<i8_t> {
    u2 a;
};
template <> struct Raw<e4m3_t> {
    u2 a;
};

template <typename E>
__device__ __forceinline__ Raw<E> raw8(const void* p, size_t i, int n)
{
    Raw<E> r{};
    if (n >= 8) {
        if constexpr (Elt<E>::size == 1) {
            r.a = *(const u2_any*)((const uint8_t*)p + i);
        } else {
            r.a = *(const u4_any*)((const char*)p + i * Elt<E>::size);
            if constexpr (Elt<E>::size == 4) r.b = *(const u4_any*)((const char*)p + i * 4 + 16);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k) {
            if (k >= n) continue;
            if constexpr (Elt<E>::size == 4) {
                const unsigned w = ((const unsigned*)p)[i + k];
                if (k < 4) r.a[k] = w;
                else r.b[k & 3] = w;
            } else if constexpr (Elt<E>::size == 2) {
                r.a[k >> 1] |= (unsigned)((const uint16_t*)p)[i + k] << (16 * (k & 1));
            } else {
                r.a[k >> 2] |= (unsigned)((const uint8_t*)p)[i + k] << (8 * (k & 3));
            }
        }
    }
    return r;
}

// (8-bit values: codes, the caller brings the scale of their block)
template <typename E>
__device__ __forceinline__ void unpack(const Raw<E>& r, float* v)
{
    if constexpr (Elt<E>::type == LAST_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[k] = __uint_as_float(r.a[k]); v[4 + k] = __uint_as_float(r.b[k]); }
    } else if constexpr (Elt<E>::type == LAST_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[2 * k] = bf16_to_float(r.a[k] & 0xffffu); v[2 * k + 1] = __uint_as_float(r.a[k] & 0xffff0000u); }
    } else if constexpr (Elt<E>::type == LAST_F16) {
        const h8 h = __builtin_bit_cast(h8, r.a);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)h[k];
    } else {
        decode4<Elt<E>::type == LAST_E4M3>(r.a[0], 1.f, v);
        decode4<Elt<E>::type == LAST_E4M3>(r.a[1], 1.f, v + 4);
    }
}

template <typename E>
__device__ __forceinline__ void load8(const void* p, size_t i, int n, float* v) { unpack<E>(raw8<E>(p, i, n), v); }

template <typename E>
__device__ __forceinline__ void store8(void* p, size_t i, int n, const float* v)
{
    if (n >= 8) {
        Elt<E>::put8(p, i, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) Elt<E>::put(p, i + k, v[k]);
    }
}

// the same with the type given at run time, the same for all lanes
__device__ __forceinline__ void store8_as(int type, void* p, size_t i, int n, const float* v)
{
    if (type == LAST_BF16) store8<bf16_t>(p, i, n, v);
    else if (type == LAST_F16) store8<f16_t>(p, i, n, v);
    else store8<float>(p, i, n, v);
}

// eight codes of a row, n of which exist
__device__ __forceinline__ void store_codes(uint8_t* p, size_t i, int n, unsigned lo, unsigned hi)
{
    if (n >= 8) {
        *(u2_any*)(p + i) = u2{lo, hi};
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[i + k] = (uint8_t)((k < 4 ? lo : hi) >> (8 * (k & 3)));
    }
}

__device__ __forceinline__ void load_codes(const uint8_t* p, size_t i, int n, unsigned* lo, unsigned* hi)
{
    if (n >= 8) {
        const u2 a = *(const u2_any*)(p + i);
        *lo = a[0];
        *hi = a[1];
    } else {
        unsigned r[2] = {0u, 0u};
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) r[k >> 2] |= (unsigned)p[i + k] << (8 * (k & 3));
        *lo = r[0];
        *hi = r[1];
    }
}

// ---- a matrix of 8-bit values with its scales
struct Eight {
    uint8_t* q;                      // null: there is none
    uint8_t* scales;
    long long pitch, scale_pitch;
    int e4m3;
};

// Eight columns c.. of a row, in each of four lanes that hold a block of 32 columns between them; `top`: the largest
// magnitude of the block.  One of them (first) writes the scale.
__device__ __forceinline__ void store_eight(const Eight& k, size_t row, int c, int n, bool first, unsigned top, const float* v)
{
    const unsigned byte = k.e4m3 ? scale_byte<true>(top) : scale_byte<false>(top);
    const unsigned lo = k.e4m3 ? encode4<true>(v, byte) : encode4<false>(v, byte);
    const unsigned hi = k.e4m3 ? encode4<true>(v + 4, byte) : encode4<false>(v + 4, byte);
    if (n > 0) {
        store_codes(k.q + row * k.pitch, c, n, lo, hi);
        if (first) k.scales[row * k.scale_pitch + c / kBlock] = (uint8_t)byte;
    }
}

__device__ __forceinline__ unsigned top8(const float* v)
{
    unsigned t = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) t = umax(t, magnitude_bits(v[k]));
    return t;
}

// largest of four neighbouring lanes, which hold a block between them
__device__ __forceinline__ unsigned quad_max(unsigned t)
{
    t = umax(t, (unsigned)__shfl_xor((int)t, 1, kWave));
    return umax(t, (unsigned)__shfl_xor((int)t, 2, kWave));
}

// ---- activations and their derivatives, in 32 bits, to a few 1e-7 of their result (exp(-v) and exp(-v^2 / 2) to about 1e-7
// times their exponent, where they are small)

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

// Q(v) = erfc(v / sqrt 2) / 2 for v >= 0, the upper tail of the normal distribution, given g = exp(-v^2 / 2).  erfc(z) e^(z^2) is
// t times a polynomial in t = 1 / (1 + 0.42 z), fitted for least relative error over z up to 9.5 (1.7e-7; 5e-7 in float32), so
// that the tail keeps its digits where 1 - erf has none.
__device__ __forceinline__ float normal_tail(float v, float g)
{
    const float t = __builtin_amdgcn_rcpf(1.f + 0.42f * 0.70710678f * v);
    float p = 0.07021627f;
    p = p * t - 0.32019392f;
    p = p * t + 0.44056344f;
    p = p * t - 0.13042411f;
    p = p * t + 0.26868749f;
    p = p * t + 0.19474322f;
    p = p * t + 0.23958302f;
    p = p * t + 0.23682442f;
    return 0.5f * p * t * g;
}

// the normal distribution function
__device__ __forceinline__ float normal_cdf(float v, float g)
{
    const float q = normal_tail(fabsf(v), g);
    return v < 0.f ? q : 1.f - q;
}

// from the exponential, and near 0, where that loses digits, from the series (to v^9: 3e-8 at 0.3)
__device__ __forceinline__ float tanh_of(float v)
{
    const float u = fabsf(v), s = v * v;
    const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __expf(2.f * u));
    const float near = u * (1.f + s * (-0.33333333f + s * (0.13333333f + s * (-0.053968254f + s * 0.021869489f))));
    return copysignf(u < 0.3f ? near : far, v);
}

__device__ __forceinline__ float activate(int act, float v)
{
    switch (act) {
    case LAST_ACT_RELU: return v < 0.f ? 0.f : v;
    case LAST_ACT_SILU: return v * sigmoid(v);
    case LAST_ACT_GELU: return v * normal_cdf(v, __expf(-0.5f * v * v));
    case LAST_ACT_TANH: return tanh_of(v);
    default: return v;
    }
}

__device__ __forceinline__ float slope(int act, float v)
{
    switch (act) {
    case LAST_ACT_RELU: return v > 0.f ? 1.f : v <= 0.f ? 0.f : v;
    case LAST_ACT_SILU: {
        const float p = sigmoid(v);
        return p * (1.f + v * (1.f - p));
    }
    case LAST_ACT_GELU: {
        const float g = __expf(-0.5f * v * v);
        return normal_cdf(v, g) + v * 0.39894228f * g;
    }
    case LAST_ACT_TANH: {
        // 1 - tanh^2 = 4 e^(-2|v|) / (1 + e^(-2|v|))^2, without the difference
        const float g = __expf(-2.f * fabsf(v)), r = __builtin_amdgcn_rcpf(1.f + g);
        return 4.f * g * r * r;
    }
    default: return 1.f;
    }
}

// eight at a time, the choice of the activation outside
__device__ __forceinline__ void activate8(int act, float* v)
{
    if (act == LAST_ACT_NONE) return;
    if (act == LAST_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate(LAST_ACT_RELU, v[k]);
    } else if (act == LAST_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate(LAST_ACT_SILU, v[k]);
    } else if (act == LAST_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate(LAST_ACT_GELU, v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate(LAST_ACT_TANH, v[k]);
    }
}

__device__ __forceinline__ void times_slope(int act, const float* h, float* v)
{
    if (act == LAST_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= slope(LAST_ACT_RELU, h[k]);
    } else if (act == LAST_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= slope(LAST_ACT_SILU, h[k]);
    } else if (act == LAST_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= slope(LAST_ACT_GELU, h[k]);
    } else if (act == LAST_ACT_TANH) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= slope(LAST_ACT_TANH, h[k]);
    }
}

}  // namespace last
