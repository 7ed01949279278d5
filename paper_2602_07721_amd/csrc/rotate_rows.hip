// New rows on their way into a cache of pages: queries and keys are normalised for each head and
// rotated by their positions, keys and values written to their slots.
//
//   y = x w / sqrt(mean(x^2) + eps)
//   (a, b) -> (a cos - b sin, b cos + a sin)   for the pairs of the first `rot` dims
//
// Everything in float32, rounded once.  An angle is position * frequency in 64 bits, less its whole
// turns, before it is rounded to float32: 4 million positions on, float32 would be off by a quarter
// radian.  Its sine and cosine are made once a token, in LDS, for all of its heads.
//
// Bound by HBM: 512 bytes a row of q, k and v.  16 lanes a row, 16 bytes a lane, so the norm's sum
// is four lane moves; a pair's other half comes from the lane that holds it.

#include <hip/hip_fp16.h>

#include "pages.hpp"

namespace pariskv {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));

constexpr int kRrThreads = 256, kRrGroups = kRrThreads / 16;
constexpr int kRrManyTokens = 4;  // tokens of a block in large calls
constexpr int kRrAhead = 4;       // rows whose loads a group has in flight

enum { kNoPairs = 0, kHalves = 1, kNeighbours = 2 };

template <int PAIRS, int TOKENS>
__global__ __launch_bounds__(kRrThreads) void rotate_rows_kernel(RotateArgs a) {
    __shared__ float2 turn[TOKENS][kD / 2];  // cosine, sine
    __shared__ int at[TOKENS];               // row of the slot's first head in the cache, -1: no slot
    const int tid = threadIdx.x, c = tid & 15, group = tid >> 4;
    const int t0 = blockIdx.x * TOKENS;
    const int hq = a.hkv * a.g, heads = hq + 2 * a.hkv;
    const int half = a.rot / 2;

    if (tid < TOKENS) {
        const int slot = t0 + tid < a.t ? a.slots[t0 + tid] : -1;
        int row = -1;
        if (slot >= 0 && slot < a.n_slots) {
            const int page = (int)a.page((uint32_t)slot), size = (int)a.page.d;
            row = page * a.hkv * size + (slot - page * size);
        }
        at[tid] = row;
    }
    if constexpr (PAIRS != kNoPairs) {
        for (int i = tid; i < TOKENS * half; i += kRrThreads) {
            const int tok = i / half, f = i % half;
            const double turns = (double)a.positions[min(t0 + tok, a.t - 1)] * (double)a.freqs[f] * 0.15915494309189535;
            float s, co;
            sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
            turn[tok][f] = float2{co, s};
        }
    }
    __syncthreads();

    // Dims 8 c .. 8 c + 7 of a row, those of the pairs' other halves, and which halves these are.
    const bool turns = 8 * c < a.rot, first = PAIRS != kHalves || 8 * c < half;
    const int other = PAIRS == kHalves && turns ? (first ? c + half / 8 : c - half / 8) : c;
    const int other_lane = (((tid & 48) | other) & 63) << 2;
    const int f0 = PAIRS == kHalves ? (turns ? 8 * min(c, other) : 0) : 4 * c;
    float w[2][8], wo[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[0][i] = a.q_weight ? a.q_weight[8 * c + i] : 1.f;
        w[1][i] = a.k_weight ? a.k_weight[8 * c + i] : 1.f;
        wo[0][i] = PAIRS == kHalves && a.q_weight ? a.q_weight[8 * other + i] : 1.f;
        wo[1][i] = PAIRS == kHalves && a.k_weight ? a.k_weight[8 * other + i] : 1.f;
    }

    const int rows = min(TOKENS, a.t - t0) * heads;
    auto source = [&](int r) {
        const int tok = r / heads, h = r % heads;
        const int64_t token = t0 + tok;
        const __half* p = h < hq            ? static_cast<const __half*>(a.q) + token * a.q_stride + h * kD
                          : h < hq + a.hkv ? static_cast<const __half*>(a.k) + token * a.k_stride + (h - hq) * kD
                                           : static_cast<const __half*>(a.v) + token * a.v_stride + (h - hq - a.hkv) * kD;
        return reinterpret_cast<const int4v*>(p) + c;
    };
    for (int r0 = group; r0 < rows; r0 += kRrGroups * kRrAhead) {
        int4v x[kRrAhead];
#pragma unroll
        for (int u = 0; u < kRrAhead; ++u) x[u] = *source(min(r0 + u * kRrGroups, rows - 1));
#pragma unroll
        for (int u = 0; u < kRrAhead; ++u) {
            const int r = min(r0 + u * kRrGroups, rows - 1);
            const int tok = r / heads, h = r % heads;
            const int kind = h < hq ? 0 : h < hq + a.hkv ? 1 : 2;
            int4v y = x[u];
            const half8 in = __builtin_bit_cast(half8, y);
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)in[i], (float)in[i], s);
            s = row_sum_f32(s);
            const bool norm = kind == 0 ? a.q_weight != nullptr : a.k_weight != nullptr;
            const float inv = norm ? rsqrtf(s * (1.f / kD) + a.eps) : 1.f;
            half8 pair = in;
            if constexpr (PAIRS == kHalves) {
                int4v z;
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = __builtin_amdgcn_ds_bpermute(other_lane, y[i]);
                pair = __builtin_bit_cast(half8, z);
            }
            if (kind < 2) {
                half8 out;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float own = (float)in[i] * inv * (kind == 0 ? w[0][i] : w[1][i]);
                    float res = own;
                    if constexpr (PAIRS == kHalves) {
                        const float2 cs = turn[tok][f0 + i];
                        const float oth = (float)pair[i] * inv * (kind == 0 ? wo[0][i] : wo[1][i]);
                        if (turns) res = first ? own * cs.x - oth * cs.y : own * cs.x + oth * cs.y;
                    } else if constexpr (PAIRS == kNeighbours) {
                        const float2 cs = turn[tok][f0 + i / 2];
                        const float oth = (float)in[i ^ 1] * inv * (kind == 0 ? w[0][i ^ 1] : w[1][i ^ 1]);
                        if (turns) res = i % 2 == 0 ? own * cs.x - oth * cs.y : own * cs.x + oth * cs.y;
                    }
                    out[i] = (_Float16)res;
                }
                y = __builtin_bit_cast(int4v, out);
            }
            if (r0 + u * kRrGroups >= rows || at[tok] < 0) continue;
            char* to;
            if (kind == 0)
                to = static_cast<char*>(a.q_out) + ((int64_t)(t0 + tok) * hq + h) * (2 * kD);
            else
                to = static_cast<char*>(kind == 1 ? a.K : a.V) +
                     ((int64_t)at[tok] + (int64_t)(h - hq - (kind - 1) * a.hkv) * a.page.d) * (2 * kD);
            reinterpret_cast<int4v*>(to)[c] = y;
        }
    }
}

}  // namespace

hipError_t launch_rotate_rows(const RotateArgs& a, hipStream_t s) {
    // One token a block leaves no CU idle in small calls; several share the weights' loads.
    const bool many = a.t >= 2048;
    const int per = many ? kRrManyTokens : 1;
    const ProfEvents pe = prof_begin("rotate_rows");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)((a.t + per - 1) / per)), dim3(kRrThreads), 0, s, pe.start, pe.stop,
                              0, a);
    };
    if (a.rot == 0)
        many ? go(rotate_rows_kernel<kNoPairs, kRrManyTokens>) : go(rotate_rows_kernel<kNoPairs, 1>);
    else if (!a.pairs)
        many ? go(rotate_rows_kernel<kHalves, kRrManyTokens>) : go(rotate_rows_kernel<kHalves, 1>);
    else
        many ? go(rotate_rows_kernel<kNeighbours, kRrManyTokens>) : go(rotate_rows_kernel<kNeighbours, 1>);
    return hipGetLastError();
}

}  // namespace pariskv
