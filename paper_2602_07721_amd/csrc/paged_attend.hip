// Attention of new tokens over pages where a sequence and KV head has at most 32 rows: decode steps
// and a few drafted or chunked tokens.
//
// Bound by HBM, and every sequence has a length of its own: the work is one line of parts of 128
// keys -- all of a sequence's first KV head, of its second, ..., of the next sequence -- cut into as
// many equal stretches as the chip holds blocks, wherever the cuts fall.  Which sequence a block
// begins in follows from sums over the lengths, which every block makes for itself, so a captured
// call stays right when lengths change.  A block meets the ends of at most two heads that others
// share with it; their softmax states go through memory to a second kernel, all others' are whole.
//
// Per wave and 32 keys as in chunk_attend_device.hpp: S^T = K Q^T, P in two float16 parts, O^T +=
// V^T P^T.  A lane looks up one key's page a step ahead of the loads that need it, so page sizes and
// tiles need not fit each other; lanes get each other's rows by permutes.

#include <hip/hip_fp16.h>

#include "paged_device.hpp"

namespace pariskv {

namespace {

// 30 tokens over up to 20011 rows take 221 us with 16 rows and 227 with 32, 40 with biases over up to 4096,
// 7 heads on a KV head, 31 and 36.
__host__ __device__ inline int few_rows(int64_t rows) { return rows <= 16 ? 16 : 32; }

struct Everyone {
    __device__ __forceinline__ bool operator()(const PagedSeq&) const { return true; }
};

template <int R, int SHAPE>
__global__ __launch_bounds__(kPgThreads, 2) void paged_few_kernel(PagedArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[kPgWaves * few_wave_lds(R)];
    few_stretch<R, SHAPE>(a, a.blocks == kPgBlocks ? line_block(blockIdx.x, kPgBlocks) : (int)blockIdx.x, Everyone(),
                             [&](int w) { return lds + w * few_wave_lds(R); });
}

__global__ __launch_bounds__(32 * kPjGroups) void paged_few_join_kernel(PagedArgs a, int R, int shaped) {
    const int rows = a.most * a.g;
    few_join(a, R, shaped ? 1.f : score_factor(a.scale), (int)blockIdx.x / rows, (int)blockIdx.x % rows);
}

}  // namespace

size_t paged_plan(PagedArgs& a) {
    const int64_t rows = (int64_t)a.most * a.g;
    // No more blocks than parts of full tables.
    const int64_t parts = (a.width * a.page.d + kPfKeys - 1) / kPfKeys * a.batch * a.hkv;
    a.blocks = (int32_t)(parts < kPgBlocks ? (parts < 1 ? 1 : parts) : kPgBlocks);
    return rows <= 32 ? FewSpace::bytes(few_rows(rows)) : paged_prompt_bytes(a);
}

hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.most * a.g;
    // 8 tokens of 4 heads a KV head, here and as tiles of rows: of a sequence of 20011 rows 30 and 39 us, of 8
    // of 131072 651 and 800, of 30 of up to 2011 52 and 55, of up to 20011 285 and 266.
    if (rows > 32) return launch_paged_prompt(a, s);
    const int shape = score_shape(a);
    ProfEvents pe = prof_begin("paged_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)a.blocks), dim3(kPgThreads), 0, s, pe.start, pe.stop, 0, a);
    };
    by_shape(shape, [&](auto x) {
        constexpr int kShape = decltype(x)::value;
        few_rows(rows) == 16 ? go(paged_few_kernel<16, kShape>) : go(paged_few_kernel<32, kShape>);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.blocks == 1) return e;
    pe = prof_begin("paged_join");
    hipExtLaunchKernelGGL(paged_few_join_kernel, dim3((unsigned)(rows * a.blocks)), dim3(32 * kPjGroups), 0, s, pe.start,
                          pe.stop, 0, a, few_rows(rows), shape);
    return hipGetLastError();
}

}  // namespace pariskv
