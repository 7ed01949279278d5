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
// A score's factor in powers of two.  A scale of 0 weighs every score alike, as this does.  Scores times the
// largest finite factor are alike, or so far apart that a larger one weighs them no other way; an infinite
// one would make NaNs of products that are 0.
constexpr float kMostFactor = 0x1.fffffep127f;
__device__ __forceinline__ float score_factor(float scale) {
    return fminf(fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-37f), kMostFactor);
}

// A row's weights are P = 2^(c2 (s - r) + kUp): s its scores, c2 their factor, and r one of them, near
// the largest so far (-infinity before the first).  r is raised only when a weight would pass 2^kSlack
// times that of r, so P stays below 2^16.  P is taken as 2^(c2 s + nm) with nm = kUp - c2 r, one
// instruction a score.  Where nm is so large that its rounding would show, r is subtracted from the
// scores first: nm is a NaN there, which sends every step through the path that raises r.  So the
// differences of finite scores decide, however large both are.
constexpr float kUp = 8.f;
constexpr float kSlack = 7.f;
constexpr float kLargeNm = 8388608.f;  // 2^23: float32 has steps of 1/2 to 1 there
__device__ __forceinline__ float nm_of(float r, float c2) { return __builtin_fmaf(-r, c2, kUp); }
// What sums and outputs of a state at r are multiplied by when they move to `to` >= r.
__device__ __forceinline__ float rescale(float r, float to, float c2) { return __builtin_amdgcn_exp2f((r - to) * c2); }
// Sums and outputs taken with nm are 2^(c2 r + nm - kUp) of those at r: what they are multiplied by
// for that (1 where nm is not what they were taken with, or nothing was).
__device__ __forceinline__ float at_r(float r, float nm, float c2) {
    const float x = __builtin_fmaf(-r, c2, kUp - nm);
    return __builtin_fabsf(nm) < kLargeNm ? __builtin_amdgcn_exp2f(x) : 1.f;
}
// Raises a row's r to m, the largest score it has met, and gives what its state is multiplied by.
__device__ __forceinline__ float raise(float m, float c2, float& r, float& nm) {
    const float to = nm_of(m, c2);
    const bool small = __builtin_fabsf(nm) < kLargeNm && __builtin_fabsf(to) < kLargeNm;
    const float c = small ? __builtin_amdgcn_exp2f(to - nm) : rescale(r, m, c2);
    r = m;
    nm = __builtin_fabsf(to) < kLargeNm ? to : __builtin_nanf("");
    return c;
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

// ---- few new tokens: a wave's 16 or 32 rows over steps of 32 keys

constexpr int kCaKeys = 32;      // keys of a step
constexpr int kCaRow = kD + 4;   // floats of an output row in LDS (spreads the rows over the banks)
// LDS of a wave's outputs [row][kCaRow], references r and sums.
constexpr int ca_state_bytes(int rows) { return rows * (kCaRow + 2) * 4; }

// What a block works on: tile `tile` of the rows of (sequence, KV head) grp, share `split` of its keys.
struct ChunkPlace {
    int64_t grp;
    int split, seq, tile;
};
// Consecutive blocks go to the 8 XCDs in turn: the row tiles of one share of the keys are 8
// apart, so that one XCD's L2 serves them all.  (The host keeps the number of blocks below 2^31.)
__device__ __forceinline__ ChunkPlace chunk_place(const ChunkArgs& a, uint32_t row_tiles, uint32_t groups) {
    ChunkPlace p;
    uint32_t id = blockIdx.x, share = id;
    p.tile = 0;
    if (row_tiles > 1) {
        const uint32_t full = groups * (uint32_t)a.splits / 8 * 8 * row_tiles;
        if (id < full) {
            share = id / (8 * row_tiles) * 8 + id % 8;
            p.tile = (int)(id / 8 % row_tiles);
        } else {
            id -= full;
            share = full / row_tiles + id / row_tiles;
            p.tile = (int)(id % row_tiles);
        }
    }
    const uint32_t grp = share / (uint32_t)a.splits;
    p.grp = grp;
    p.split = (int)(share % (uint32_t)a.splits);
    p.seq = (int)(grp / (uint32_t)a.hkv);
    return p;
}

// The reference r and the sum of a row's part in the workspace (behind all rows' outputs).
__device__ __forceinline__ float2* part_state(const ChunkArgs& a, int64_t groups, int64_t row) {
    return reinterpret_cast<float2*>(a.part + groups * a.g * a.t * a.splits * kD) + row * a.splits;
}
// A share without keys: its rows' states say so (their outputs are not read).
__device__ __forceinline__ void leave_idle(const ChunkArgs& a, const ChunkPlace& pl, int64_t groups, int row0, int rows) {
    const int M = a.g * a.t;
    for (int r = row0 + (int)threadIdx.x; r < min(row0 + rows, M); r += (int)blockDim.x)
        part_state(a, groups, pl.grp * M + r)[pl.split] = float2{-__builtin_huge_valf(), 0.f};
}

// Which of the drafts first, first + 1, ... (valid of them) token tok sees.
__device__ __forceinline__ uint32_t draft_bits(const ChunkArgs& a, int seq, int tok, int first, int valid) {
    const uint64_t m = a.mask ? (uint64_t)a.mask[(int64_t)seq * a.t + tok] : ~0ull >> (63 - tok);
    return first > 63 ? 0u : (uint32_t)(m >> first) & bits_to(valid - 1);
}

// Values of V that are not finite.  A key that a token does not see has a weight of 0 there, but 0
// times infinity is not 0, and a draft or a row that overflowed must not spoil tokens that do not
// see it.  So where not every token sees every key (drafts; the ends of windows) the products get
// such values as 0, and the rows that see them have them added at the end, if there were any.
// Where every token sees the key the products take them as they are, and an infinity may come out
// as NaN (a weight's second part may be 0 or negative): either way the dim is not finite for the
// tokens that see the key, and for no others.
//
// Sets bits of kOddBits in m if one of v's 8 values is such a value (all ones in its exponent).
constexpr uint32_t kOddBits = 0x80008000u;
__device__ __forceinline__ void note_odd(u4v v, uint32_t& m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= (v[i] & 0x7c007c00u) + 0x04000400u;
}
__device__ __forceinline__ u4v finite_part(u4v v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7c00u) == 0x7c00u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7c000000u) == 0x7c000000u) v[i] &= 0xffffu;
    }
    return v;
}
// Adds x's values that are not finite to sum.
__device__ __forceinline__ void add_odd(f4v& sum, h4v x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_isfinite((float)x[i]) ? 0.f : (float)x[i];
}
// Such values of the keys that row `row` sees, dims 4 d4 on: of all its drafts, or of the cache
// rows of its window and sinks.
template <bool WINDOW>
__device__ __forceinline__ f4v odd_part(const ChunkArgs& a, int64_t row, int d4) {
    const int64_t M = (int64_t)a.g * a.t, grp = row / M;
    const int tok = (int)(row % M) % a.t, seq = (int)(grp / a.hkv);
    f4v sum{0.f, 0.f, 0.f, 0.f};
    if constexpr (WINDOW) {
        const h4v* v = static_cast<const h4v*>(a.V) + grp * a.capacity * (kD / 4) + d4;
        const int p = key_span(a, seq, 0, a.t).start + tok;
        const int lo = max(0, p - (int)a.window + 1), sinks = min((int)a.sink, lo);
        for (int j = 0; j < sinks; ++j) add_odd(sum, v[(int64_t)j * (kD / 4)]);
        for (int j = lo; j <= p; ++j) add_odd(sum, v[(int64_t)j * (kD / 4)]);
    } else {
        const uint64_t m = a.mask ? (uint64_t)a.mask[(int64_t)seq * a.t + tok] : ~0ull >> (63 - tok);
        const h4v* v = static_cast<const h4v*>(a.Vt) + grp * a.t * (kD / 4) + d4;
        for (int j = 0; j < a.t; ++j)
            if ((m >> j) & 1) add_odd(sum, v[j * (kD / 4)]);
    }
    return sum;
}

// 16 bytes of key `key`'s V (chunk `chunk` of 16) in a tile of V in LDS.  The XOR spreads the 16
// rows of a transposing read over all banks.
__device__ __forceinline__ void put_v(unsigned char* vt, int key, int chunk, h8v v) {
    *reinterpret_cast<h8v*>(vt + key * 256 + ((chunk ^ (2 * (key & 7))) << 4)) = v;
}

// The finite parts of a step's V that this wave has put into LDS.
__device__ __forceinline__ void clean_v(unsigned char* vt, int lane) {
    wave_lds_order();
    u4v* at = reinterpret_cast<u4v*>(vt) + lane;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) at[64 * i] = finite_part(at[64 * i]);
}

typedef float f16v __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s4v* lds_s4v;

// A wave's rows: their softmax, and how matrix instructions split them over the lanes.  R rows
// and 32 keys a step: S^T = K Q^T in kHalves blocks of keys and kSteps steps of dims, O^T +=
// V^T P^T with the scores' registers as the second operand.  32 rows take instructions of 32 x
// 32, which occupy the issue of the vector units half as long as those of 16 x 16.
template <int R>
struct ChunkRows;

// P of two neighbouring scores of a row as two float16 values each: hi, and what hi leaves.
__device__ __forceinline__ void split_p(float s0, float s1, float c2, float base, float& sum, h8v& hi, h8v& lo, int at) {
    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s0, c2, base));
    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1, c2, base));
    sum += p0 + p1;
    // Two values an instruction; p - hi is exact.
    const h2v ph = __builtin_convertvector((f2v{p0, p1}), h2v);
    const h2v pl = __builtin_convertvector((f2v{__builtin_fmaf((float)ph[0], -1.f, p0),
                                                __builtin_fmaf((float)ph[1], -1.f, p1)}), h2v);
    hi[at] = ph[0];
    hi[at + 1] = ph[1];
    lo[at] = pl[0];
    lo[at + 1] = pl[1];
}

// The r that a row's state is left with.  Maxima pass NaNs over, sums and outputs do not: a row whose
// scores are all NaN has the r of one that saw no key, but a sum that is NaN.  Any finite r keeps
// such a state in the joins, which then hand the NaNs on.
__device__ __forceinline__ float left_r(float r, float sum) {
    return sum != sum && r == -__builtin_huge_valf() ? 0.f : r;
}

// 16 rows.  Lane l = col + 16 lg: row col, keys 16 h + 4 lg + i, outputs of dims 16 d + 4 lg + i.
template <>
struct ChunkRows<16> {
    static constexpr int kHalves = 2, kSteps = 4;
    // The reference score, nm (infinite before the first key), the sum over this lane's keys.
    float r = -__builtin_huge_valf(), nm = __builtin_huge_valf(), sum = 0.f, c2;
    f4v o[8], s[2];
    int lg, tkey;

    __device__ __forceinline__ ChunkRows(float factor, int lane)
        : c2(factor), lg(lane >> 4), tkey(4 * (lane >> 4) + ((lane & 15) >> 2)) {
#pragma unroll
        for (int d = 0; d < 8; ++d) o[d] = f4v{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ static int row(int lane) { return lane & 15; }
    // This lane's part of step c of a key (of the row's query): key(lane) of half h, 8 dims from
    // dim() on.  BLOCKS: as a quantised key's lane group likes it, one block of 32 dims each.
    template <bool BLOCKS>
    __device__ __forceinline__ static int dim(int c, int lane) {
        return BLOCKS ? 32 * (lane >> 4) + 8 * c : 32 * c + 8 * (lane >> 4);
    }
    __device__ __forceinline__ static int key(int h, int lane) { return 16 * h + (lane & 15); }

    template <class F>
    __device__ __forceinline__ void scores(const h8v (&qf)[kSteps], F&& kpart) {
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kpart(h, c), qf[c],
                                                              c == 0 ? f4v{0.f, 0.f, 0.f, 0.f} : s[h], 0, 0, 0);
    }

    // With the step's V in LDS at vt; bits of w: the keys that the row sees.
    __device__ __forceinline__ void accumulate(uint32_t w, const unsigned char* vt, int lane) {
        if (__builtin_expect(!__all(w == ~0u), 0)) {
            const uint32_t b = w >> (4 * lg);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(b & (1u << (16 * h + i)))) s[h][i] = -__builtin_huge_valf();
        }
        float top = -__builtin_huge_valf();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[h][i]);
        float base = nm < __builtin_huge_valf() ? nm : 0.f;
        if (__builtin_expect(__any(top > -__builtin_huge_valf() && !(__builtin_fmaf(top, c2, nm) <= kUp + kSlack)), 0)) {
            const float m = rows_max(top);  // -inf where the row saw nothing in this step
            if (m > r) {
                const float c = raise(m, c2, r, nm);  // 0 before the first key
                sum *= c;
#pragma unroll
                for (int d = 0; d < 8; ++d) o[d] *= c;
                base = nm;
            }
            if (__builtin_expect(__any(nm != nm), 0)) {
                const float off = nm != nm ? r : 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) s[h] -= off;
                base = nm != nm ? kUp : base;
            }
        }
        h8v hi, lo;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; i += 2) split_p(s[h][i], s[h][i + 1], c2, base, sum, hi, lo, 4 * h + i);
        const int col = lane & 15;
        const unsigned char* tr = vt + tkey * 256 + ((col & 3) >> 1) * 16 + (col & 1) * 8;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const unsigned char* at = tr + ((d ^ (tkey & 7)) << 5);
            const h8v vf = join_h4(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(at)),
                                   __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(at + 16 * 256)));
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, hi, o[d], 0, 0, 0);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, lo, o[d], 0, 0, 0);
        }
    }

    // Adds the values of a row of V that are not finite to this lane's outputs.
    __device__ __forceinline__ void add_odd_values(const h4v* v) {
#pragma unroll
        for (int d = 0; d < 8; ++d) add_odd(o[d], v[4 * d + lg]);
    }

    // Leaves the state in ca_state_bytes(16) of LDS; the sums' signs say `odd`.
    __device__ __forceinline__ void leave(unsigned char* to, int lane, bool odd) const {
        float* so = reinterpret_cast<float*>(to);
        const float fix = at_r(r, nm, c2), l = __builtin_fabsf(rows_sum(sum)) * fix;
        const int row = lane & 15;
        if (lg == 0) {
            so[16 * kCaRow + row] = left_r(r, l);
            so[16 * (kCaRow + 1) + row] = odd ? -l : l;
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) *reinterpret_cast<f4v*>(so + row * kCaRow + 16 * d + 4 * lg) = o[d] * fix;
    }
};

// 32 rows.  Lane l = col + 32 half: row col, keys 8 (i / 4) + 4 half + i % 4, outputs of dims
// 32 d + 8 (i / 4) + 4 half + i % 4.
template <>
struct ChunkRows<32> {
    static constexpr int kHalves = 1, kSteps = 8;
    float r = -__builtin_huge_valf(), nm = __builtin_huge_valf(), sum = 0.f, c2;
    f16v o[4], s;
    int half, tkey, tchunk;

    __device__ __forceinline__ ChunkRows(float factor, int lane)
        : c2(factor), half(lane >> 5), tkey(4 * (lane >> 5) + ((lane & 15) >> 2)),
          tchunk(2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
    __device__ __forceinline__ static int row(int lane) { return lane & 31; }
    template <bool BLOCKS>
    __device__ __forceinline__ static int dim(int c, int lane) {
        return BLOCKS ? 64 * (lane >> 5) + 8 * c : 16 * c + 8 * (lane >> 5);
    }
    __device__ __forceinline__ static int key(int, int lane) { return lane & 31; }

    template <class F>
    __device__ __forceinline__ void scores(const h8v (&qf)[kSteps], F&& kpart) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kSteps; ++c) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kpart(0, c), qf[c], s, 0, 0, 0);
    }

    __device__ __forceinline__ void accumulate(uint32_t w, const unsigned char* vt, int lane) {
        if (__builtin_expect(!__all(w == ~0u), 0)) {
            const uint32_t b = w >> (4 * half);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(b & (1u << (8 * (i / 4) + i % 4)))) s[i] = -__builtin_huge_valf();
        }
        float top = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
        float base = nm < __builtin_huge_valf() ? nm : 0.f;
        if (__builtin_expect(__any(top > -__builtin_huge_valf() && !(__builtin_fmaf(top, c2, nm) <= kUp + kSlack)), 0)) {
            const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            const float m = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
            if (m > r) {
                const float c = raise(m, c2, r, nm);
                sum *= c;
#pragma unroll
                for (int d = 0; d < 4; ++d) o[d] *= c;
                base = nm;
            }
            if (__builtin_expect(__any(nm != nm), 0)) {
                const float off = nm != nm ? r : 0.f;
                s -= off;
                base = nm != nm ? kUp : base;
            }
        }
        const unsigned char* tr = vt + tkey * 256 + (lane & 1) * 8;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            h8v hi, lo;
#pragma unroll
            for (int i = 0; i < 8; i += 2) split_p(s[8 * k + i], s[8 * k + i + 1], c2, base, sum, hi, lo, i);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const unsigned char* at = tr + 16 * k * 256 + (((4 * d + tchunk) ^ (2 * tkey)) << 4);
                const h8v vf = join_h4(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(at)),
                                       __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(at + 8 * 256)));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, hi, o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, lo, o[d], 0, 0, 0);
            }
        }
    }

    __device__ __forceinline__ void add_odd_values(const h4v* v) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f4v part{0.f, 0.f, 0.f, 0.f};
                add_odd(part, v[8 * d + 2 * j + half]);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][4 * j + i] += part[i];
            }
    }

    __device__ __forceinline__ void leave(unsigned char* to, int lane, bool odd) const {
        float* so = reinterpret_cast<float*>(to);
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        const int row = lane & 31;
        const float fix = at_r(r, nm, c2);
        if (half == 0) {
            const float l = __builtin_fabsf(__uint_as_float(x[0]) + __uint_as_float(x[1])) * fix;
            so[32 * kCaRow + row] = left_r(r, l);
            so[32 * (kCaRow + 1) + row] = odd ? -l : l;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<f4v*>(so + row * kCaRow + 32 * d + 8 * j + 4 * half) =
                    f4v{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]} * fix;
    }
};

// 4 dims of an output row: float32, or float16 where the prompt's next product reads it.  Rows of
// tokens that are not there are left as they were.
template <bool WINDOW>
__device__ __forceinline__ void store_row(const ChunkArgs& a, int64_t row, int d4, float inv, f4v acc, bool odd,
                                          bool real) {
    acc *= inv;
    if (odd && real) acc += odd_part<WINDOW>(a, row, d4);
    if constexpr (WINDOW) {
        const h4v h{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
        if (real) static_cast<h4v*>(a.out)[row * (kD / 4) + d4] = h;
    } else {
        static_cast<f4v*>(a.out)[row * (kD / 4) + d4] = acc;
    }
}

// Joins the states that WAVES waves left `stride` bytes apart for rows [row0, row0 + R) of
// group grp, and writes the rows, or the share's part of them.  32 lanes a row, 4 dims a lane;
// `sub` of `subs` such sets of lanes.  A negative sum says that odd_part has something
// to add, in a wave's state and in a share's part.
template <int R, int WAVES, bool WINDOW>
__device__ __forceinline__ void join_waves(const ChunkArgs& a, const ChunkPlace& pl, int64_t groups, int row0, int tokens,
                                           const unsigned char* states, int stride, int sub, int subs) {
    const int M = a.g * a.t, d4 = threadIdx.x & 31;
    const float* of = reinterpret_cast<const float*>(states);
    const float c2 = score_factor(a.scale);
    for (int r = sub; r < R; r += subs) {
        if (row0 + r >= M) break;
        float top = -__builtin_huge_valf();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, of[w * (stride / 4) + R * kCaRow + r]);
        float l = 0.f;
        bool odd = false;
        f4v acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) odd |= __builtin_signbit(of[w * (stride / 4) + R * (kCaRow + 1) + r]);
        if (top > -__builtin_huge_valf())
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float* ow = of + w * (stride / 4);
                const float c = rescale(ow[R * kCaRow + r], top, c2);
                l += c * __builtin_fabsf(ow[R * (kCaRow + 1) + r]);
                acc += c * *reinterpret_cast<const f4v*>(ow + r * kCaRow + 4 * d4);
            }
        const int64_t row = pl.grp * M + row0 + r;
        if (a.splits > 1) {
            const int64_t at = row * a.splits + pl.split;
            reinterpret_cast<f4v*>(a.part)[at * (kD / 4) + d4] = acc;
            if (d4 == 0) part_state(a, groups, row)[pl.split] = float2{top, odd ? -l : l};
        } else {
            store_row<WINDOW>(a, row, d4, l > 0.f ? 1.f / l : 0.f, acc, odd, (row0 + r) % a.t < tokens);
        }
    }
}

}  // namespace pariskv
