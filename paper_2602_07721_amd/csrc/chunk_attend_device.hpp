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

// Keys of one (sequence, KV head), as the kernel walks them.
struct KeySpan {
    int64_t sink_end, lo, keys;  // cached key v: row v below sink_end, else v - sink_end + lo
    int64_t start;               // position of new token 0 (sliding window)
    int32_t tokens;              // new tokens
};

__device__ __forceinline__ KeySpan key_span(const ChunkArgs& a, int seq) {
    KeySpan s;
    int64_t len = a.n;
    if (a.lens) {
        const int64_t v = a.lens[seq];
        len = v < 0 ? 0 : v < a.n ? v : a.n;
    }
    s.tokens = a.t;
    if (a.counts) {
        const int32_t v = a.counts[seq];
        s.tokens = v < 0 ? 0 : v < a.t ? v : a.t;
    }
    s.start = len;
    s.sink_end = s.lo = 0;
    s.keys = len;
    if (a.window > 0) {
        const int64_t hi = s.tokens > 0 ? len + s.tokens : 0;
        s.lo = len - a.window + 1 > 0 ? len - a.window + 1 : 0;
        if (s.lo > hi) s.lo = hi;
        s.sink_end = a.sink < s.lo ? a.sink : s.lo;
        s.keys = s.sink_end + hi - s.lo;
    }
    return s;
}

}  // namespace pariskv
