// Rounding to 8-bit integers, shared by the key/value store and the 8-bit linear layers.
//
// A group of values x_i (a token's head in the store, a token's row or a weight column in a layer) is held as whole numbers
// q_i = 127 x_i / amax, amax = max |x_i|, and one fp32 scale amax / 127.  q_i is the exact quotient rounded to the nearest
// number, halves to the even one: the fp32 product below decides it unless it lies next to a border of two numbers, which is
// then decided in exact arithmetic.  So every implementation of the definition holds the same numbers, whatever it rounds
// on the way.  A group with an infinity or a NaN gets a NaN scale (it reads back as NaN throughout), a group of zeros scale 0.
#pragma once

#include "mfma_util.h"

namespace pserve {

typedef __attribute__((ext_vector_type(2))) uint32_t q8_u32x2;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((ext_vector_type(4))) int i32x4;

// A launch has fewer than 2^32 threads in a dimension, and whole blocks count: numbers of blocks that may come near that are laid out in lines
// of equal length.  The blocks of the last line that are too many find no row of theirs.
inline dim3 block_lines(int64_t blocks, unsigned z = 1) {
    const int64_t lines = cdiv(blocks, 1 << 20);
    return dim3((unsigned)cdiv(blocks, lines), (unsigned)lines, z);
}
__device__ __forceinline__ int64_t block_of_lines() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

struct Quant8 {
    float mul, amax, inv, scale;                    // x * mul: groups of tiny values are read 2^64 times as large (exact)
    // amax_bits: the largest |x| as its bit pattern (so infinities and NaN come out on top)
    __device__ __forceinline__ explicit Quant8(uint32_t amax_bits) {
        const float a = __uint_as_float(amax_bits);
        mul = a < 0x1p-60f ? 0x1p64f : 1.f;
        amax = a * mul;
        // a / 127, correctly rounded: the quotient by the rounded reciprocal and one correction from its exact rest (Markstein 1990; the same
        // as the division for all 2^23 mantissas at the ends of the exponents taken here), a third of a division's instructions
        const float by = 1.f / 127.f, q = a * by;
        scale = a < 0x1p-100f ? a / 127.f : fmaf(fmaf(-127.f, q, a), by, q);
        scale = fminf(scale, 0x1.0204060000000p+121f);             // 127 times the scale of the largest number rounds to infinity, one step below it does not
        inv = a > 0.f ? __builtin_amdgcn_rcpf(amax * 0x1p-7f) * (127.f / 128.f) : 0.f;     // to 1.5 steps; the argument keeps off the subnormal results
        if (amax_bits >= 0x7f800000u) { scale = __uint_as_float(0x7fc00000u); mul = 0.f; inv = 0.f; amax = 1.f; }
    }
    __device__ __forceinline__ int operator()(float x) const {
        const float y = x * mul, t = y * inv;       // |error of t| < 127 * (1.5 * 2^-23 + 2^-24) < 2^-15
        float r = rintf(t);
        if (fabsf(fabsf(t - r) - 0.5f) < 0x1p-14f) {
            const double k = floorf(fabsf(t)), twice = 254.0 * fabs((double)y), border = (2.0 * k + 1.0) * (double)amax;  // exact: 32 bits each
            const double up = twice > border ? 1.0 : twice < border ? 0.0 : fmod(k, 2.0);
            r = copysignf((float)(k + up), t);
        }
        return scale == scale ? (int)r : 0;         // (inf * 0 is NaN)
    }
};

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// eight consecutive values as fp32
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
    const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r[i] << 16); v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = to_bf16(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (uint32_t)to_bf16(v[2 * i]) | ((uint32_t)to_bf16(v[2 * i + 1]) << 16);
    *reinterpret_cast<u32x4*>(p) = o;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
// Eight values as they lie in memory, their largest magnitude as a bit pattern (bf16: two at a time, whole numbers of 16 bits), the values
template <typename T> struct Raw8 { u32x4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ void load_raw(const T* p, Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = *reinterpret_cast<const u32x4*>(p + i * (16 / sizeof(T)));
}
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
__device__ __forceinline__ uint32_t largest8(uint32_t m, const Raw8<uint16_t>& r) {
    u16x2 p = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_elementwise_max(p, __builtin_bit_cast(u16x2, r.w[0][i] & 0x7fff7fffu));
    return max(m, (uint32_t)max(p[0], p[1]) << 16);
}
__device__ __forceinline__ uint32_t largest8(uint32_t m, const Raw8<float>& r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, r.w[i / 4][i % 4] & 0x7fffffffu);
    return m;
}
template <typename T>
__device__ __forceinline__ void values8(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = __uint_as_float(i & 1 ? r.w[0][i / 2] & 0xffff0000u : r.w[0][i / 2] << 16);
        else v[i] = __uint_as_float(r.w[i / 4][i % 4]);
    }
}
// The largest of L neighbouring lanes (8, 16 or 64) in all of them: within 16 lanes by operands that come from other lanes
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
#define PS_LANE(ctrl) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, ctrl, 0xf, 0xf, true))
    PS_LANE(0xb1);                              // lane ^ 1
    PS_LANE(0x4e);                              // lane ^ 2
    PS_LANE(0x141);                             // the other four of eight
    if (L >= 16) PS_LANE(0x140);                // the other eight of sixteen
#undef PS_LANE
    if (L == 64) {
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    }
    return m;
}

// Eight whole numbers as bytes.  t + 1.5 * 2^23 is rounded to a whole number, whose low byte is the two's complement form; only where
// one of the eight is next to a border (or the group is one of tiny values) does the exact form above decide.
__device__ __forceinline__ q8_u32x2 pack8(const Quant8& z, const float (&v)[8]) {
    constexpr float MAGIC = 12582912.f;
    uint32_t s[8];
    float far = 0.f;                                            // largest distance to the whole number
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float r = fmaf(v[i], z.inv, MAGIC);
        s[i] = __float_as_uint(r);
        far = fmaxf(far, fabsf(fmaf(v[i], z.inv, MAGIC - r)));
    }
    if (far > 0.5f - 0x1p-14f || z.mul > 1.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = (uint32_t)z(v[i]);
    }
    q8_u32x2 o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(s[4 * h + 1], s[4 * h], 0x0c0c0400), hi = __builtin_amdgcn_perm(s[4 * h + 3], s[4 * h + 2], 0x04000c0c);
        o[h] = lo | hi;
    }
    return o;
}

}  // namespace pserve
