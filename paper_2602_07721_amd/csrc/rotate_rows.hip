// New rows on their way into a cache of pages: queries and keys are normalised for each head and
// rotated by their positions, keys and values written to their slots.
//
//   y = x w / sqrt(mean(x^2) + eps)
//   (a, b) -> (a cos - b sin, b cos + a sin)   for the pairs of the first `rot` dims
//
// Everything in float32, rounded once.  An angle is position * frequency in two numbers of 64 bits, less
// its whole turns, before it is rounded to float32: 4 million positions on, float32 would be off by a
// quarter radian; near 2^31 radians one number of 64 bits is off by up to 2^-21.9.
//
// Bound by HBM: 512 bytes a row of q, k and v.  16 lanes take some heads of one kind of a token, 16 bytes
// a lane, 4 rows at a time and the next 4 on their way: the norm's sum is four lane moves, a pair's other
// half comes from the lane that holds it.  The lanes' sines, cosines and weights, made while the first rows
// are on their way and folded into two factors a dim, serve all of them: 16384 tokens of 32 + 16 heads 84
// us, 4.8 TB/s (a copy: 5.2); 107 us with sines in LDS behind a barrier for a block of 4 tokens, and 94
// with cosines, sines and weights in registers of their own, which leave fewer waves.

#include <hip/hip_fp16.h>

#include "pages.hpp"

namespace pariskv {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));

constexpr int kRrThreads = 256, kRrGroups = kRrThreads / 16;
constexpr int kRrAhead = 4;       // rows whose loads a group has in flight
constexpr int kRrMostHeads = 8;   // heads of a group
constexpr int kRrFewGroups = 2048;

enum { kNoPairs = 0, kHalves = 1, kNeighbours = 2 };

// Groups of a token of up to n heads each: of q, of k, of v.  Those of a kind take heads in turn, so
// that a wave's read next to each other.
struct RowGroups {
    int q, kv;
    __host__ __device__ RowGroups(const RotateArgs& a, int n)
        : q((a.hkv * a.g + n - 1) / n), kv((a.hkv + n - 1) / n) {}
    __host__ __device__ int64_t all(const RotateArgs& a) const { return (int64_t)a.t * (q + 2 * kv); }
};

// p f / (2 pi) less the nearest whole number, from -1/2 to 1/2: what the product and 1 / (2 pi) leave in 64
// bits is added at the end.
__device__ __forceinline__ float turns_of(double p, double f) {
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
    const double angle = p * f, whole = rint(angle * kTurn);
    return (float)(fma(angle, kTurn, -whole) + fma(angle, kTurnRest, fma(p, f, -angle) * kTurn));
}

template <int PAIRS>
__global__ __launch_bounds__(kRrThreads) void rotate_rows_kernel(RotateArgs a, int heads) {
    const RowGroups gr(a, heads);
    const int c = threadIdx.x & 15;  // dims 8 c .. 8 c + 7 of a row
    // All of q's groups, then k's, then v's: a wave's are of one kind mostly.
    int64_t id = (int64_t)blockIdx.x * kRrGroups + (threadIdx.x >> 4);
    const int64_t nq = (int64_t)a.t * gr.q, nk = (int64_t)a.t * gr.kv;
    const int kind = id < nq ? 0 : id < nq + nk ? 1 : 2;
    id -= kind == 0 ? 0 : kind == 1 ? nq : nq + nk;
    const uint32_t per = (uint32_t)(kind == 0 ? gr.q : gr.kv);
    const int tok = (int)((uint32_t)id / per), first = (int)((uint32_t)id % per);
    if (tok >= a.t) return;
    const int slot = a.slots[tok];
    const int all = kind == 0 ? a.hkv * a.g : a.hkv;
    const __half* from = kind == 0 ? static_cast<const __half*>(a.q) + tok * a.q_stride
                       : kind == 1 ? static_cast<const __half*>(a.k) + tok * a.k_stride
                                   : static_cast<const __half*>(a.v) + tok * a.v_stride;
    int4v x[kRrAhead];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kRrAhead; ++u)
            x[u] = reinterpret_cast<const int4v*>(from + min(h0 + u * (int)per, all - 1) * kD)[c];
    };
    load(first);

    // The pairs' other halves, and which halves this lane's are.
    const int half = a.rot / 2;
    const bool turns = PAIRS != kNoPairs && kind < 2 && 8 * c < a.rot;
    const bool is_first = PAIRS != kHalves || 8 * c < half;
    const int other = PAIRS == kHalves && turns ? (is_first ? c + half / 8 : c - half / 8) : c;
    const int other_lane = (int)((threadIdx.x & 48) | other) << 2;
    // y = inv (x A + x' B), x' the pair's other half: weights, cosines and sines in two factors a dim.
    const float* weight = kind == 0 ? a.q_weight : a.k_weight;
    const bool norm = kind < 2 && weight;
    float fa[8], fb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        fa[i] = norm ? weight[8 * c + i] : 1.f;
        fb[i] = !norm ? 1.f : PAIRS == kHalves ? weight[8 * other + i] : weight[8 * c + (i ^ 1)];
    }
    if (PAIRS != kNoPairs && turns) {
        const double p = a.positions[tok];
        const int f0 = PAIRS == kHalves ? 8 * min(c, other) : 4 * c;
        float si = 0.f, co = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (PAIRS == kHalves || i % 2 == 0) {
                // In turns; within 2^-22.9 of sine and cosine over 2^24 values of half a turn either way.
                const float x = turns_of(p, a.freqs[f0 + (PAIRS == kHalves ? i : i / 2)]);
                si = __builtin_amdgcn_sinf(x);
                co = __builtin_amdgcn_cosf(x);
            }
            fa[i] *= co;
            fb[i] *= (PAIRS == kHalves ? is_first : i % 2 == 0) ? -si : si;
        }
    }
    if (slot < 0 || slot >= a.n_slots) return;
    const int page = (int)a.page((uint32_t)slot), size = (int)a.page.d;
    // Row 0 of the kind, and how far apart its heads' rows are.
    const int64_t to_row = kind == 0 ? (int64_t)tok * all : (int64_t)page * a.hkv * size + (slot - page * size);
    const int step = kind == 0 ? 1 : size;
    int4v* to = static_cast<int4v*>(kind == 0 ? a.q_out : kind == 1 ? a.K : a.V) + to_row * (kD / 8) + c;
    for (int h0 = first; h0 < all; h0 += kRrAhead * (int)per) {
        int4v y[kRrAhead];
#pragma unroll
        for (int u = 0; u < kRrAhead; ++u) y[u] = x[u];
        if (h0 + kRrAhead * (int)per < all) load(h0 + kRrAhead * (int)per);
#pragma unroll
        for (int u = 0; u < kRrAhead; ++u) {
            if (kind < 2) {
                const half8 in = __builtin_bit_cast(half8, y[u]);
                float inv = 1.f;
                if (norm) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)in[i], (float)in[i], s);
                    inv = rsqrtf(row_sum_f32(s) * (1.f / kD) + a.eps);
                }
                half8 pair = in;
                if constexpr (PAIRS == kHalves) {
                    int4v z;
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = __builtin_amdgcn_ds_bpermute(other_lane, y[u][i]);
                    pair = __builtin_bit_cast(half8, z);
                }
                half8 out;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float res = (float)in[i] * fa[i];
                    if constexpr (PAIRS != kNoPairs) {
                        const float both = __builtin_fmaf((float)(PAIRS == kHalves ? pair[i] : in[i ^ 1]), fb[i], res);
                        res = turns ? both : res;
                    }
                    out[i] = (_Float16)(res * inv);
                }
                y[u] = __builtin_bit_cast(int4v, out);
            }
            const int h = h0 + u * (int)per;
            if (h >= all) continue;
            to[(int64_t)h * step * (kD / 8)] = y[u];
        }
    }
}

}  // namespace

hipError_t launch_rotate_rows(const RotateArgs& a, hipStream_t s) {
    // 8 heads share a group's sines, in few groups 4, which one group loads at once: 4096 tokens of 32 + 16
    // heads take 21.0 us with 8 and 27.1 with 4, 32 tokens 7.4 and 6.4, 500 about the same.
    const int heads = RowGroups(a, kRrMostHeads).all(a) < kRrFewGroups ? kRrAhead : kRrMostHeads;
    const int64_t blocks = (RowGroups(a, heads).all(a) + kRrGroups - 1) / kRrGroups;
    const ProfEvents pe = prof_begin("rotate_rows");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRrThreads), 0, s, pe.start, pe.stop, 0, a, heads);
    };
    if (a.rot == 0) go(rotate_rows_kernel<kNoPairs>);
    else if (!a.pairs) go(rotate_rows_kernel<kHalves>);
    else go(rotate_rows_kernel<kNeighbours>);
    return hipGetLastError();
}

}  // namespace pariskv
