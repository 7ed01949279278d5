// Device code that the few-token and the prompt form of chunk_attend.hpp share.
#pragma once

#include "chunk_attend.hpp"
#include "quant.hpp"

namespace pariskv {

typedef short s4v __attribute__((ext_vector_type(4)));

// Orders this wave's LDS accesses as written (the lanes read what other lanes wrote).
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Maximum (sum) of x over the lanes l, l ^ 16, l ^ 32, l ^ 48: the four lanes of a row.
__device__ __forceinline__ float rows_max(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

__device__ __forceinline__ h8v as_h8(u4v v) { return __builtin_bit_cast(h8v, v); }

// The 8 values of two transposing reads.
__device__ __forceinline__ h8v join_h4(s4v a, s4v b) {
    return __builtin_bit_cast(h8v, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// 16 bytes of float16 query; negated for a negative scale, so that the kernels' scale is positive
// and the largest score has the largest weight.
__device__ __forceinline__ h8v query_part(u4v v, uint32_t flip) {
    return as_h8(v ^ flip);
}
// A score's factor in powers of two.  A scale of 0 weighs every score alike, as this does.
__device__ __forceinline__ float score_factor(float scale) {
    return fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-37f);
}

// Bits 0..x of a word (none for x < 0).
__device__ __forceinline__ uint32_t bits_to(int x) { return x < 0 ? 0u : x >= 31 ? ~0u : (2u << x) - 1u; }

// Which of 32 keys at cache rows base, base + 1, ... the token at position p sees.
__device__ __forceinline__ uint32_t window_bits(int p, int base, int sink, int window) {
    return bits_to(p - base) & (bits_to(sink - 1 - base) | ~bits_to(p - window - base));
}

// The cache rows that some tokens of a sequence see: [0, sink_end) and [lo, hi), with the first
// token's position (sliding window; sink_end = lo = 0 in a tree).
struct KeySpan {
    int sink_end, lo, hi;
    int start;
    int tokens;  // new tokens
};

// Of tokens [i0, i1) of sequence seq, at most the tokens there are.
__device__ __forceinline__ KeySpan key_span(const ChunkArgs& a, int seq, int i0, int i1) {
    KeySpan s;
    const int n = (int)a.n;
    const int len = a.lens ? min(max(a.lens[seq], 0), n) : n;
    s.tokens = a.counts ? min(max(a.counts[seq], 0), a.t) : a.t;
    s.start = len;
    s.sink_end = s.lo = 0;
    s.hi = len;
    if (a.window > 0) {
        i1 = min(i1, s.tokens);
        if (i0 >= i1) {
            s.hi = 0;
        } else {
            s.hi = len + i1;
            s.lo = max(0, len + i0 - (int)a.window + 1);
            s.sink_end = min((int)a.sink, s.lo);
        }
    }
    return s;
}

}  // namespace pariskv
