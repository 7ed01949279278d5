// The quantised K/V cache: records of codes and block scales, and their conversions.
//
// A row of 128 float16 values is 4 blocks of 32.  A block stores a scale 2^s and a code a
// value, e4m3 (8 bits, largest value 448) or e2m1 (4 bits, largest value 6):
//   s    = the smallest integer >= s_min with max |x| <= largest 2^s,
//   code = the nearest code value to x 2^-s, ties to the even code.
// s_min is -15 (-23): the code values' spacing times 2^s is then at least 2^-24, the spacing
// of float16's smallest values, so nothing below it is worth representing and every stored
// value is a float16 value.  Only s = 8 (14) reaches past 65504, the largest float16 value;
// there the codes stop at 240 (3).  A power-of-two scale makes x 2^-s exact, and gfx950
// scales and converts two values in one instruction either way.
//
// Record of one token and KV head, quant_record_bytes() long: the K codes in order of their
// dims (two 4-bit codes a byte, the even dim low), the V codes, 4 bytes s + 127 of K's
// blocks, 4 of V's, zeros up to a multiple of 16 bytes.  A gathered record touches 3 cache lines of
// 128 bytes (8/8 bits: 272 bytes at any multiple of 16 end within three), 2.5 on average (8/4: 208)
// or 2 (4/4: 144).  With the 8 scale bytes of a row in an array of their own it would be as many, 3
// (8/8) and 2 (4/4), or more, 3 (8/4); one record keeps a range of rows one stretch of memory, to
// write, to stream and to move between HBM and the host.  What it costs: 16 of its bytes hold 8 of
// scales, and over the host link, with the scales left in HBM, the codes alone would be 1 line
// instead of 2 (4/4) or 2 instead of 3 (8/8).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.hpp"

namespace pariskv {

typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));
// Loaded words, as a vector type that arrays of stay in registers (HIP's uint4 is a class).
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef short s2v __attribute__((ext_vector_type(2)));

// Bytes of the codes of one row.
__host__ __device__ constexpr int quant_code_bytes(int bits) { return kD * bits / 8; }
__host__ __device__ constexpr int quant_record_bytes(int k_bits, int v_bits) {
    return (quant_code_bytes(k_bits) + quant_code_bytes(v_bits) + 8 + 15) / 16 * 16;
}

template <int BITS>
struct QuantFormat;
template <>
struct QuantFormat<8> {
    static constexpr int kEmax = 8;                // 448 = 1.75 * 2^8
    static constexpr uint32_t kTopMant = 0x600000; // .75 as a float32 mantissa
    static constexpr int kSmin = -15, kSmax = 8;
    static constexpr uint32_t kLimit = 0x7b807b80; // 240 * 2^8 = 61440, twice
};
template <>
struct QuantFormat<4> {
    static constexpr int kEmax = 2;                // 6 = 1.5 * 2^2
    static constexpr uint32_t kTopMant = 0x400000;
    static constexpr int kSmin = -23, kSmax = 14;
    static constexpr uint32_t kLimit = 0x7a007a00; // 3 * 2^14 = 49152, twice
};

// s + 127 of a block with this largest magnitude.
template <int BITS>
__device__ __forceinline__ uint32_t quant_scale(float amax) {
    using F = QuantFormat<BITS>;
    const uint32_t b = __float_as_uint(amax);
    const int s = (int)(b >> 23) - F::kEmax + ((b & 0x7fffffu) > F::kTopMant ? 1 : 0);
    return (uint32_t)max(s, F::kSmin + 127);
}

// The float32 2^s of a stored scale byte (bits 23..30 hold s + 127).
__device__ __forceinline__ float quant_scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// 8 float16 values (4 words) to codes: 2 words of e4m3, or 1 word of e2m1 in .x.
template <int BITS>
__device__ __forceinline__ uint2 quant_encode8(uint4 v, uint32_t scale) {
    using F = QuantFormat<BITS>;
    const float sf = quant_scale_value(scale);
    h2v x[4];
    __builtin_memcpy(x, &v, 16);
    if (scale == (uint32_t)(F::kSmax + 127)) {
        h2v lim;
        const uint32_t lw = F::kLimit;
        __builtin_memcpy(&lim, &lw, 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_elementwise_max(__builtin_elementwise_min(x[i], lim), -lim);
    }
    uint2 r{0u, 0u};
    if constexpr (BITS == 8) {
        s2v lo{0, 0}, hi{0, 0};
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, x[0], sf, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, x[1], sf, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, x[2], sf, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, x[3], sf, true);
        __builtin_memcpy(&r.x, &lo, 4);
        __builtin_memcpy(&r.y, &hi, 4);
    } else {
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.x, x[0], sf, 0);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.x, x[1], sf, 1);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.x, x[2], sf, 2);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.x, x[3], sf, 3);
    }
    return r;
}

// 8 codes back to float16 values (exact): word x (and y with 8 bits).
template <int BITS>
__device__ __forceinline__ h8v quant_decode8(uint32_t x, uint32_t y, float scale) {
    h2v a, b, c, d;
    if constexpr (BITS == 8) {
        a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, scale, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, scale, true);
        c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, scale, false);
        d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, scale, true);
    } else {
        a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 0);
        b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 2);
        d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 3);
    }
    return h8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 8 codes at `p`: two words of 8-bit codes, one of 4-bit codes.
template <int BITS>
__device__ __forceinline__ u2v quant_load8(const uint8_t* p) {
    if constexpr (BITS == 8) return *reinterpret_cast<const u2v*>(p);
    return u2v{*reinterpret_cast<const uint32_t*>(p), 0u};
}

}  // namespace pariskv
