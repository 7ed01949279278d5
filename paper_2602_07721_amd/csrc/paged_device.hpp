// Device code that both forms of the attention over pages share.
#pragma once

#include "chunk_attend_device.hpp"
#include "pages.hpp"

namespace pariskv {

// One sequence's new tokens [begin, begin + count) of q and its cached rows, as the call's arrays say
// and its sizes allow.
struct PagedSeq {
    int begin, count, len;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int b) {
    PagedSeq s;
    s.begin = min(max(a.offsets[b], 0), a.t);
    const int end = min(max(a.offsets[b + 1], s.begin), a.t);
    s.count = min(end - s.begin, a.most);
    if (a.counts) s.count = min(s.count, max(a.counts[b], 0));
    const int64_t room = min(a.width * (int64_t)a.page.d, kMaxKvRows);
    s.len = (int)min((int64_t)max(a.lens[b], 0), room);
    return s;
}

// Where a key's row lies in K and V: its page's entry, and whether there is such a page.
__device__ __forceinline__ int page_entry(const PagedArgs& a, int b, int row) {
    return a.table[b * a.width + a.page((uint32_t)row)];
}
__device__ __forceinline__ int page_row(const PagedArgs& a, int entry, int head, int row) {
    const int size = (int)a.page.d;
    return (entry * a.hkv + head) * size + (row - (int)a.page((uint32_t)row) * size);
}

// What is done to scores before their softmax.
enum { kPlainScores = 0, kCappedScores = 1, kBiasedScores = 2 };

// With a shape, scores are in powers of two: s' = cap log2(e) tanh(scale s / cap), or the plain
// product, plus slope log2(e) times the distance.  tanh(u) = 1 - 2 / (2^(2 log2(e) u) + 1) is off by
// 2^-23 at most; where u is small, a series in u keeps that relative to u (the next term is 2^-24 of
// it at 0.2).
template <int SHAPE>
struct ScoreShape {
    float unit, cap, slope;  // s times unit is u (capped) or the score in powers of two
    __device__ __forceinline__ ScoreShape(const PagedArgs& a, int head) {
        constexpr float kLog2e = 1.4426950408889634f;
        const float scale = fabsf(a.scale);
        unit = SHAPE & kCappedScores ? scale / a.cap : scale * kLog2e;
        cap = SHAPE & kCappedScores ? a.cap * kLog2e : 0.f;
        slope = SHAPE & kBiasedScores ? a.slopes[head] * kLog2e : 0.f;
    }
    // Of the key `distance` behind the token (negative: how far behind).
    __device__ __forceinline__ float operator()(float s, float distance) const {
        float x = s * unit;
        if constexpr ((SHAPE & kCappedScores) != 0) {
            const float u = x, u2 = u * u;
            const float e = __builtin_amdgcn_exp2f(u * 2.8853900817779268f);
            const float far = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f);
            float near = __builtin_fmaf(u2, -0.053968254f, 0.13333334f);
            near = __builtin_fmaf(u2, near, -0.33333334f);
            near = __builtin_fmaf(u2 * u, near, u);
            x = cap * (u2 < 0.04f ? near : far);
        }
        if constexpr ((SHAPE & kBiasedScores) != 0) x = __builtin_fmaf(slope, distance, x);
        return x;
    }
};

// Values of V that are not finite, of the keys that a row at position p sees, dims 4 d4 on.
__device__ __forceinline__ f4v paged_odd_part(const PagedArgs& a, int b, int head, int p, int len, int d4) {
    f4v sum{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j <= min(p, len - 1); ++j) {
        const int entry = page_entry(a, b, j);
        if ((uint32_t)entry >= (uint32_t)a.n_pages) continue;
        add_odd(sum, static_cast<const h4v*>(a.V)[(int64_t)page_row(a, entry, head, j) * (kD / 4) + d4]);
    }
    return sum;
}

// Sum over the lanes before this one, 64 bits.
__device__ __forceinline__ int64_t wave_sum_before(int64_t v, int64_t* all) {
    const int lane = threadIdx.x & 63;
    int64_t in = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t x = __shfl_up((long long)in, d, 64);
        if (lane >= d) in += x;
    }
    *all = __shfl((long long)in, 63, 64);
    return in - v;
}

hipError_t launch_paged_prompt(const PagedArgs& a, hipStream_t s);
size_t paged_prompt_bytes(const PagedArgs& a);

}  // namespace pariskv
