// Rows into the quantised cache as they are written, and back (format: quant.hpp).
//
// 16 lanes hold a row of K and the row of V of one token and KV head, 8 dims a lane; a block
// of 32 dims is then 4 lanes, whose largest magnitude two lane exchanges give.  Both
// directions are bound by HBM: 8 x 131072 rows and 8-bit codes, 822 MB, take 131 us to quantise
// (6.3 TB/s) and 147 us back (5.6 TB/s; a plain copy reaches 5.3).

#include "quant.hpp"

namespace pariskv {

namespace {

constexpr int kQuThreads = 256;
constexpr int kQuRows = kQuThreads / 16;  // rows a block takes at once

// First row of sequence `seq` in the cache.
__device__ __forceinline__ int64_t quant_first_row(const int32_t* rows, int64_t row, int seq) {
    return rows ? (int64_t)rows[seq] : row;
}

// s + 127 of the block that this lane's 8 values belong to.
template <int BITS>
__device__ __forceinline__ uint32_t block_scale(uint4 v) {
    // Magnitudes of float16 values order as their bits do.
    typedef unsigned short u2 __attribute__((ext_vector_type(2)));
    const uint32_t w[4] = {v.x & 0x7fff7fffu, v.y & 0x7fff7fffu, v.z & 0x7fff7fffu, v.w & 0x7fff7fffu};
    u2 a[4];
    __builtin_memcpy(a, w, 16);
    u2 m = __builtin_elementwise_max(__builtin_elementwise_max(a[0], a[1]), __builtin_elementwise_max(a[2], a[3]));
    uint32_t b = max((uint32_t)m[0], (uint32_t)m[1]);
    b = max(b, (uint32_t)__builtin_amdgcn_mov_dpp((int)b, 0xB1, 0xF, 0xF, true));
    b = max(b, (uint32_t)__builtin_amdgcn_mov_dpp((int)b, 0x4E, 0xF, 0xF, true));
    const unsigned short h = (unsigned short)b;
    _Float16 f;
    __builtin_memcpy(&f, &h, 2);
    return quant_scale<BITS>((float)f);
}

// The four block scales of a row as one word, in every lane of the row.
__device__ __forceinline__ uint32_t row_scales(uint32_t scale, int lane) {
    uint32_t w = scale << (8 * ((lane >> 2) & 3));
    w |= lane_xor(w, 4, lane);
    return w | lane_xor(w, 8, lane);
}

template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t* p, int l16, uint2 c) {
    if constexpr (BITS == 8)
        reinterpret_cast<uint2*>(p)[l16] = c;
    else
        reinterpret_cast<uint32_t*>(p)[l16] = c.x;
}

template <int KB, int VB>
__global__ __launch_bounds__(kQuThreads) void quantize_rows_kernel(const uint4* __restrict__ K,
                                                                   const uint4* __restrict__ V,
                                                                   int64_t src_capacity, uint8_t* __restrict__ rec,
                                                                   int64_t capacity, int64_t row,
                                                                   const int32_t* __restrict__ rows, int64_t t,
                                                                   int32_t hkv) {
    constexpr int kRecord = quant_record_bytes(KB, VB);
    const int64_t grp = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * kQuRows + (threadIdx.x >> 4);
    const int64_t r = quant_first_row(rows, row, (int)(grp / hkv)) + i;
    if (i >= t || r < 0 || r >= capacity) return;  // all 16 lanes of a row together
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    // Past the caches: the rows are not read again soon (8 x 131072 rows: 150 us without).
    const u4v k4 = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(K) + (grp * src_capacity + i) * 16 + l16);
    const u4v v4 = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(V) + (grp * src_capacity + i) * 16 + l16);
    const uint4 k{k4[0], k4[1], k4[2], k4[3]}, v{v4[0], v4[1], v4[2], v4[3]};
    const uint32_t sk = block_scale<KB>(k), sv = block_scale<VB>(v);
    uint8_t* out = rec + (grp * capacity + r) * kRecord;
    store_codes<KB>(out, l16, quant_encode8<KB>(k, sk));
    store_codes<VB>(out + quant_code_bytes(KB), l16, quant_encode8<VB>(v, sv));
    const uint32_t wk = row_scales(sk, lane), wv = row_scales(sv, lane);
    constexpr int kScales = quant_code_bytes(KB) + quant_code_bytes(VB);
    static_assert(kRecord == kScales + 16, "the scales and the zeros behind them are one store");
    if (l16 == 0) *reinterpret_cast<uint4*>(out + kScales) = uint4{wk, wv, 0u, 0u};
}

template <int KB, int VB>
__global__ __launch_bounds__(kQuThreads) void dequantize_rows_kernel(const uint8_t* __restrict__ rec,
                                                                     int64_t capacity, int64_t row,
                                                                     const int32_t* __restrict__ rows, int64_t t,
                                                                     int32_t hkv, uint4* __restrict__ K,
                                                                     uint4* __restrict__ V, int64_t dst_capacity) {
    constexpr int kRecord = quant_record_bytes(KB, VB);
    const int64_t grp = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * kQuRows + (threadIdx.x >> 4);
    const int64_t r = quant_first_row(rows, row, (int)(grp / hkv)) + i;
    if (i >= t || r < 0 || r >= capacity) return;
    const int l16 = threadIdx.x & 15;
    const uint8_t* in = rec + (grp * capacity + r) * kRecord;
    const u2v ck = quant_load8<KB>(in + l16 * KB);
    const u2v cv = quant_load8<VB>(in + quant_code_bytes(KB) + l16 * VB);
    const uint2 s = *reinterpret_cast<const uint2*>(in + quant_code_bytes(KB) + quant_code_bytes(VB));
    const int shift = 8 * (l16 >> 2);
    const h8v k = quant_decode8<KB>(ck.x, ck.y, quant_scale_value((s.x >> shift) & 255u));
    const h8v v = quant_decode8<VB>(cv.x, cv.y, quant_scale_value((s.y >> shift) & 255u));
    uint4 w;
    __builtin_memcpy(&w, &k, 16);
    K[(grp * dst_capacity + i) * 16 + l16] = w;
    __builtin_memcpy(&w, &v, 16);
    V[(grp * dst_capacity + i) * 16 + l16] = w;
}

}  // namespace

hipError_t launch_quantize_rows(const void* K, const void* V, int64_t src_capacity, uint8_t* rec, int64_t capacity,
                                int32_t k_bits, int32_t v_bits, int64_t row, const int32_t* rows, int64_t t,
                                int32_t batch, int32_t hkv, hipStream_t s) {
    const dim3 grid((unsigned)((t + kQuRows - 1) / kQuRows), (unsigned)(batch * hkv));
    const ProfEvents pe = prof_begin("quantize_rows");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, grid, dim3(kQuThreads), 0, s, pe.start, pe.stop, 0,
                              static_cast<const uint4*>(K), static_cast<const uint4*>(V), src_capacity, rec, capacity,
                              row, rows, t, hkv);
    };
    if (k_bits == 8)
        v_bits == 8 ? go(quantize_rows_kernel<8, 8>) : go(quantize_rows_kernel<8, 4>);
    else
        v_bits == 8 ? go(quantize_rows_kernel<4, 8>) : go(quantize_rows_kernel<4, 4>);
    return hipGetLastError();
}

hipError_t launch_dequantize_rows(const uint8_t* rec, int64_t capacity, int32_t k_bits, int32_t v_bits, int64_t row,
                                  const int32_t* rows, int64_t t, int32_t batch, int32_t hkv, void* K, void* V,
                                  int64_t dst_capacity, hipStream_t s) {
    const dim3 grid((unsigned)((t + kQuRows - 1) / kQuRows), (unsigned)(batch * hkv));
    const ProfEvents pe = prof_begin("dequantize_rows");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, grid, dim3(kQuThreads), 0, s, pe.start, pe.stop, 0, rec, capacity, row, rows, t,
                              hkv, static_cast<uint4*>(K), static_cast<uint4*>(V), dst_capacity);
    };
    if (k_bits == 8)
        v_bits == 8 ? go(dequantize_rows_kernel<8, 8>) : go(dequantize_rows_kernel<8, 4>);
    else
        v_bits == 8 ? go(dequantize_rows_kernel<4, 8>) : go(dequantize_rows_kernel<4, 4>);
    return hipGetLastError();
}

}  // namespace pariskv
