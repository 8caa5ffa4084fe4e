// Rounding to 8-bit floating point (e4m3: sign, four exponent bits, three fraction bits, largest number 448), shared by the rows that the
// norms write and the 8-bit floating-point layers.
//
// A block of 128 consecutive values x_i is held as numbers v_i = e4m3(x_i 2^-e) and one power of two 2^e, e the smallest whole number of
// -100 .. 119 with max |x_i| <= 448 * 2^e, so e = 119 where none is (what lies beyond 448 * 2^119 = 2.98e38 is held as that; what the block stands
// for, v_i 2^e, is a normal bf16 number or zero in all cases, which the layers of fp32 tensors use).  A power of two
// and not amax / 448: multiplying by it does not round, so the one rounding of a value (to the nearest, halves to the even fraction) is that
// of the conversion instruction; the relative error is the same 2^-4 at most, as the format's numbers lie as dense at both ends of a factor of
// two; and the matrix instruction takes powers of two (scale byte e + 127) for nothing.  A block with an infinity or a NaN is held as NaN.
#pragma once

#include "quant8.h"

namespace pserve {

constexpr int F8_BLOCK = 128;
constexpr uint32_t F8_NAN4 = 0x7f7f7f7fu;
constexpr uint32_t F8_LARGEST_BITS = 0x7f600000u;      // 448 * 2^119
constexpr uint32_t F8_FIRST_BYTE = 127 - 100, F8_LAST_BYTE = 127 + 119;

// rows of K values: [rows][f8_width(K)] numbers, then the scale bytes in words of four blocks, [f8_scales(K) / 4][rows]: what neighbouring lanes read for neighbouring
// rows is in one line (with a row's bytes side by side, lanes 32 or 64 bytes apart, 16 x 8192 x 8192 took 20 us for 17.5, 8192^3 450 for 439)
__host__ __device__ inline int32_t f8_width(int32_t K) { return (K + 127) / 128 * 128; }
__host__ __device__ inline int32_t f8_scales(int32_t K) { return (K + 511) / 512 * 4; }
__device__ __forceinline__ int64_t f8_scale_at(int64_t rows, int64_t row, int b) { return 4 * ((b >> 2) * rows + row) + (b & 3); }
inline size_t f8_bytes(int64_t rows, int32_t K) { return (size_t)rows * (size_t)(f8_width(K) + f8_scales(K)); }

// four numbers of a word: x / 2^e for two values of each pair, as the scaled conversion rounds them (the same as a multiplication and a conversion)
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

struct F8Scale {
    uint32_t amax, byte;
    float scale;                                        // 2^e
    __device__ __forceinline__ explicit F8Scale(uint32_t amax_bits) : amax(amax_bits) {
        // the exponent field counts up where the fraction passes 0.75 (448 = 1.75 * 2^8)
        const uint32_t up = (amax_bits + 0x1fffffu) >> 23;
        byte = min(max(up, F8_FIRST_BYTE + 8u) - 8u, F8_LAST_BYTE);
        if (amax_bits >= 0x7f800000u) byte = 127;
        scale = __uint_as_float(byte << 23);
    }
    __device__ __forceinline__ uint32_t word(float a, float b, float c, float d) const {
        s16x2 o = {0, 0};
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, a, b, scale, false);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, c, d, scale, true);
        return __builtin_bit_cast(uint32_t, o);
    }
    // N values as bytes
    template <int N>
    __device__ __forceinline__ void words(const float (&v)[N], uint32_t (&o)[N / 4]) const {
        if (amax <= F8_LARGEST_BITS) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) o[i] = word(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {                                        // what is too large is cut off; a block that is not finite is NaN
            const float most = 448.f * 0x1p119f;
            float s[N];
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = fminf(fmaxf(v[i], -most), most);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) o[i] = amax >= 0x7f800000u ? F8_NAN4 : word(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
        }
    }
    // Eight values as they lie in memory
    __device__ __forceinline__ q8_u32x2 pack8(const Raw8<float>& r) const {
        float v[8];
        uint32_t o[2];
        values8(r, v);
        words(v, o);
        return q8_u32x2{o[0], o[1]};
    }
    __device__ __forceinline__ q8_u32x2 pack8(const Raw8<uint16_t>& r) const {
        if (amax > F8_LARGEST_BITS) {
            float v[8];
            uint32_t o[2];
            values8(r, v);
            words(v, o);
            return q8_u32x2{o[0], o[1]};
        }
        q8_u32x2 o;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s16x2 w = {0, 0};
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, (uint32_t)r.w[0][2 * h]), scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, (uint32_t)r.w[0][2 * h + 1]), scale, true);
            o[h] = __builtin_bit_cast(uint32_t, w);
        }
        return o;
    }
    __device__ __forceinline__ void pack(const float (&v)[8], uint8_t* o) const {
        uint32_t w[2];
        words(v, w);
        *reinterpret_cast<q8_u32x2*>(o) = q8_u32x2{w[0], w[1]};
    }
    __device__ __forceinline__ void pack(const float (&v)[4], uint8_t* o) const {
        uint32_t w[1];
        words(v, w);
        *reinterpret_cast<uint32_t*>(o) = w[0];
    }
};

__device__ __forceinline__ float f8_scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Over neighbouring lanes (8, 16, 32 or 64), in all of them, by operands that come from other lanes: within sixteen as in lanes_max, then
// lane ^ 16 and lane ^ 32 by swapping rows of sixteen and halves (both results together are the lane's own and the other value)
__device__ __forceinline__ uint32_t max_16_apart(uint32_t m) {
    const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t max_32_apart(uint32_t m) {
    const auto r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max(r[0], r[1]);
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#define PS_LANE(ctrl) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, 0xf, 0xf, true))
    PS_LANE(0xb1);
    PS_LANE(0x4e);
    PS_LANE(0x141);
    if (L >= 16) PS_LANE(0x140);
#undef PS_LANE
    if (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (L == 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// 16 bytes at any element's address
template <typename T> struct AnyPiece;
template <> struct AnyPiece<uint16_t> { typedef u32x4 __attribute__((aligned(2))) type; };
template <> struct AnyPiece<float> { typedef u32x4 __attribute__((aligned(4))) type; };

// 16 bytes from or to any element's address, past the caches where `past` says so.  (The empty statements keep the compiler from making one of the two.)
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* at, bool past) {
    const auto* p = reinterpret_cast<const typename AnyPiece<T>::type*>(at);
    u32x4 v;
    if (past) {
        asm volatile("");
        v = __builtin_nontemporal_load(p);
        asm volatile("");
    } else {
        v = *p;
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* at, const u32x4& v, bool past) {
    auto* p = reinterpret_cast<typename AnyPiece<T>::type*>(at);
    if (past) {
        asm volatile("");
        __builtin_nontemporal_store(v, p);
        asm volatile("");
    } else {
        *p = v;
    }
}

// the largest |v| of N values as a bit pattern (infinities and NaN come out on top)
template <int N>
__device__ __forceinline__ uint32_t f8_largest(const float (&v)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

}  // namespace pserve
