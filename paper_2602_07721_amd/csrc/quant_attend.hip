// Attention of one decode step over retrieved rows of the quantised cache and, with a window,
// over Sink + Local + Update Buffer rows of the float16 window cache:
//   o = sum_{i in list} softmax_i(scale <k_i, q>) v_i,  codes or float16 in, float32 math.
//
// One block per query head, as the float16 attention (attend_row.hpp): 16 lanes a row, 8 dims
// a lane, so a row's 128 code bytes are one 128-byte read by 16 lanes and its 8 scale bytes
// one broadcast read; every lane keeps the codes of kQaUnroll rows in flight and a running
// maximum, sum and 8 accumulators in float32.  Codes become float16 in registers (one
// instruction for two values) and are multiplied in float32.  Bound by the latency of one
// round of gathered records (HBM) or by the host link, which moves whole lines of 128 bytes:
// 16384 records of 144 (272) bytes in pinned memory take 88 (123) us, 2 (3) lines each at 48
// GB/s, from 32 blocks as from 512, and the same when a record is loaded by one instruction.

#include <hip/hip_fp16.h>

#include "attend_row.hpp"
#include "quant.hpp"

namespace pariskv {

namespace {

constexpr int kQaThreads = 1024;
constexpr int kQaGroups = kQaThreads / 16;  // rows a block reads at once
constexpr int kQaWaves = kQaThreads / 64;
constexpr int kQaUnroll = 4;  // rows in flight a lane (8: 6.8 us where 4 take 5.9, 32 heads x 256 rows)

struct QaScratch {
    float m[kQaWaves], l[kQaWaves];
    float acc[kQaWaves][kD];
};

// Running softmax of a group of 16 lanes: maximum and sum, and the outputs of 8 dims a lane.
struct QaState {
    float m = -__builtin_huge_valf(), l = 0.f, acc[8] = {};

    // N rows, of which `there` exist: one rescaling.
    template <int N>
    __device__ __forceinline__ void add(const float (&s)[N], const float (&v)[N][8], const bool (&there)[N]) {
        float mn = m;
#pragma unroll
        for (int u = 0; u < N; ++u) mn = there[u] ? fmaxf(mn, s[u]) : mn;
        // m = -inf before the first row: c = 0.  Rows whose scores are NaN leave the maximum as it is,
        // and make the sum NaN.
        const float from = mn > -__builtin_huge_valf() ? mn : 0.f;
        const float c = __expf(m - from);
        l *= c;
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[d] *= c;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (!there[u]) continue;  // its values may be anything
            const float p = __expf(s[u] - from);
            l += p;
#pragma unroll
            for (int d = 0; d < 8; ++d) acc[d] += p * v[u][d];
        }
        m = mn;
    }
};

__device__ __forceinline__ float dot8(const float* a, const float* b) {
    float s = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) s += a[d] * b[d];
    return s;
}

__device__ __forceinline__ void to_float8(h8v h, float* f) {
#pragma unroll
    for (int d = 0; d < 8; ++d) f[d] = (float)h[d];
}

template <int KB, int VB>
__global__ __launch_bounds__(kQaThreads) void quant_attend_kernel(
    const __half* __restrict__ q, const uint8_t* __restrict__ rec, int64_t capacity, const int32_t* __restrict__ idx,
    int32_t k, int32_t hkv, int32_t g, float scale, float* __restrict__ out, AttendWindow win,
    const __half* __restrict__ Kw, const __half* __restrict__ Vw) {
    __shared__ QaScratch sm;
    constexpr int kRecord = quant_record_bytes(KB, VB);
    constexpr int kScales = quant_code_bytes(KB) + quant_code_bytes(VB);
    const int32_t hq = hkv * g;
    const int64_t row = blockIdx.x;
    const int64_t kvh = row / hq * hkv + row % hq / g;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, grp16 = tid >> 4, l16 = tid & 15;

    float qf[8];
    unpack8_half(reinterpret_cast<const uint4*>(q + row * kD)[l16], qf);
#pragma unroll
    for (int d = 0; d < 8; ++d) qf[d] *= scale;
    QaState st;

    const uint8_t* base = rec + kvh * capacity * kRecord;
    const int32_t* list = idx + row * k;
    const int shift = 8 * (l16 >> 2);
    for (int at = 0; at < k; at += kQaGroups * kQaUnroll) {
        int64_t r[kQaUnroll];
        u2v kc[kQaUnroll], vc[kQaUnroll], sc[kQaUnroll];
#pragma unroll
        for (int u = 0; u < kQaUnroll; ++u) {
            const int j = at + u * kQaGroups + grp16;
            const int32_t x = j < k ? list[j] : -1;
            r[u] = x < 0 ? -1 : win.retr_begin + x;
            if (r[u] >= capacity) r[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < kQaUnroll; ++u) {
            if (r[u] < 0) continue;
            const uint8_t* p = base + r[u] * kRecord;
            kc[u] = quant_load8<KB>(p + l16 * KB);
            vc[u] = quant_load8<VB>(p + quant_code_bytes(KB) + l16 * VB);
            sc[u] = *reinterpret_cast<const u2v*>(p + kScales);
        }
        float s[kQaUnroll], v[kQaUnroll][8];
        bool there[kQaUnroll];
#pragma unroll
        for (int u = 0; u < kQaUnroll; ++u) {
            there[u] = r[u] >= 0;
            float f[8];
            to_float8(quant_decode8<KB>(kc[u][0], kc[u][1], quant_scale_value((sc[u][0] >> shift) & 255u)), f);
            s[u] = sum16(dot8(qf, f));
            to_float8(quant_decode8<VB>(vc[u][0], vc[u][1], quant_scale_value((sc[u][1] >> shift) & 255u)), v[u]);
        }
        st.add(s, v, there);
    }
    const int nd = (int)win.dense_rows();
    for (int at = 0; at < nd; at += kQaGroups * kQaUnroll) {
        u4v kc[kQaUnroll], vc[kQaUnroll];
#pragma unroll
        for (int u = 0; u < kQaUnroll; ++u) {
            const int j = min(at + u * kQaGroups + grp16, nd - 1);
            const int64_t slot = kvh * win.win_capacity + (win.dense_entry(j) & ~kWinRow);
            kc[u] = reinterpret_cast<const u4v*>(Kw + slot * kD)[l16];
            vc[u] = reinterpret_cast<const u4v*>(Vw + slot * kD)[l16];
        }
        float s[kQaUnroll], v[kQaUnroll][8];
        bool there[kQaUnroll];
#pragma unroll
        for (int u = 0; u < kQaUnroll; ++u) {
            there[u] = at + u * kQaGroups + grp16 < nd;
            float f[8];
            to_float8(__builtin_bit_cast(h8v, kc[u]), f);
            s[u] = sum16(dot8(qf, f));
            to_float8(__builtin_bit_cast(h8v, vc[u]), v[u]);
        }
        st.add(s, v, there);
    }

    // The 4 rows of 16 lanes of a wave into one state, then the waves' states through LDS.
#pragma unroll
    for (int step = 16; step <= 32; step <<= 1) {
        const float mp = __uint_as_float(lane_xor(__float_as_uint(st.m), step, lane));
        const float lp = __uint_as_float(lane_xor(__float_as_uint(st.l), step, lane));
        const float mn = fmaxf(st.m, mp);
        const float safe = mn > -__builtin_huge_valf() ? mn : 0.f;
        const float c0 = __expf(st.m - safe), c1 = __expf(mp - safe);
        st.l = st.l * c0 + lp * c1;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const float ap = __uint_as_float(lane_xor(__float_as_uint(st.acc[d]), step, lane));
            st.acc[d] = st.acc[d] * c0 + ap * c1;
        }
        st.m = mn;
    }
    if (lane < 16) {
        if (l16 == 0) {
            sm.m[wave] = st.m;
            sm.l[wave] = st.l;
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) sm.acc[wave][8 * l16 + d] = st.acc[d];
    }
    __syncthreads();
    if (tid < kD) {
        float M = -__builtin_huge_valf(), L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < kQaWaves; ++w) M = fmaxf(M, sm.m[w]);
        const float from = M > -__builtin_huge_valf() ? M : 0.f;
#pragma unroll
        for (int w = 0; w < kQaWaves; ++w) {
            const float c = __expf(sm.m[w] - from);
            L += sm.l[w] * c;
            O += sm.acc[w][tid] * c;
        }
        out[row * kD + tid] = L == 0.f ? 0.f : O / L;  // NaN where some score was
    }
}

}  // namespace

hipError_t launch_quant_attend(const void* q, const uint8_t* rec, int64_t capacity, int32_t k_bits, int32_t v_bits,
                               const int32_t* idx, int32_t k, int32_t batch, int32_t hkv, int32_t g, float scale,
                               float* out, const AttendWindow& win, const void* Kw, const void* Vw, hipStream_t s) {
    const ProfEvents pe = prof_begin(win.dense_rows() > 0 ? "quant_tiered_attend" : "quant_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)(batch * hkv * g)), dim3(kQaThreads), 0, s, pe.start, pe.stop, 0,
                              static_cast<const __half*>(q), rec, capacity, idx, k, hkv, g, scale, out, win,
                              static_cast<const __half*>(Kw), static_cast<const __half*>(Vw));
    };
    if (k_bits == 8)
        v_bits == 8 ? go(quant_attend_kernel<8, 8>) : go(quant_attend_kernel<8, 4>);
    else
        v_bits == 8 ? go(quant_attend_kernel<4, 8>) : go(quant_attend_kernel<4, 4>);
    return hipGetLastError();
}

}  // namespace pariskv
