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

constexpr int kPfWaves = 4, kPfThreads = 64 * kPfWaves;
constexpr int kPfKeys = kPfWaves * kCaKeys;  // keys of a part
constexpr int few_blocks(int rows) { return rows == 16 ? 768 : 512; }  // 3 or 2 a CU

__host__ __device__ inline int few_rows(int64_t rows) { return rows <= 16 ? 16 : 32; }

// Parts of a sequence's keys for one KV head; one also where there are tokens but no keys.
__device__ __forceinline__ int few_parts(const PagedSeq& s) {
    return s.count > 0 ? max(1, (s.len + kPfKeys - 1) / kPfKeys) : 0;
}

// Blocks that have work: each at least one of the line's parts.
__device__ __forceinline__ int64_t few_used(const PagedArgs& a, int64_t line) { return min(line, (int64_t)a.blocks); }

// The workspace: parts before each sequence (one KV head's) and of all; outputs and states of the
// heads that blocks share, two a block.
struct FewSpace {
    int64_t* before;  // [batch + 1]
    float* part;      // [2 blocks][R][D]
    float2* state;    // [2 blocks][R]
};
__host__ __device__ inline size_t few_line_bytes(int batch) { return ((size_t)batch + 1 + 31) / 32 * 256; }
template <int R>
__device__ __forceinline__ FewSpace few_space(const PagedArgs& a) {
    FewSpace w;
    char* p = static_cast<char*>(a.workspace);
    w.before = reinterpret_cast<int64_t*>(p);
    w.part = reinterpret_cast<float*>(p + few_line_bytes(a.batch));
    w.state = reinterpret_cast<float2*>(w.part + (int64_t)2 * a.blocks * R * kD);
    return w;
}

template <int R, int SHAPE>
__global__ __launch_bounds__(kPfThreads, R == 16 ? 3 : 2) void paged_few_kernel(PagedArgs a) {
    constexpr int kVBytes = kCaKeys * kD * 2;
    constexpr int kWaveLds = kVBytes > ca_state_bytes(R) ? kVBytes : ca_state_bytes(R);
    __shared__ __attribute__((aligned(16))) unsigned char lds[kPfWaves * kWaveLds];
    __shared__ int64_t wave_total[kPfWaves], found_before;
    __shared__ int found;
    using Rows = ChunkRows<R>;
    constexpr int kHalves = Rows::kHalves, kSteps = Rows::kSteps;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const FewSpace ws = few_space<R>(a);

    // Sums over the sequences: thread i has `each` neighbouring ones.
    const int each = (a.batch + kPfThreads - 1) / kPfThreads;
    const int mine0 = min(tid * each, a.batch), mine1 = min(mine0 + each, a.batch);
    int64_t sum = 0;
    for (int b = mine0; b < mine1; ++b) sum += few_parts(paged_seq(a, b));
    int64_t all;
    int64_t before = wave_sum_before(sum, &all);
    if (lane == 63) wave_total[wave] = all;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < kPfWaves; ++w) {
        before += w < wave ? wave_total[w] : 0;
        all += wave_total[w];
    }
    if (blockIdx.x == 0) {
        int64_t at = before;
        for (int b = mine0; b < mine1; ++b) {
            ws.before[b] = at;
            at += few_parts(paged_seq(a, b));
        }
        if (tid == kPfThreads - 1) ws.before[a.batch] = all;
    }
    const int64_t line = all * a.hkv;
    const int64_t blocks = few_used(a, line);
    if (blockIdx.x >= blocks) return;  // the whole block
    const int64_t x0 = blockIdx.x * line / blocks, x1 = (blockIdx.x + 1) * line / blocks;
    if (before * a.hkv <= x0 && x0 < (before + sum) * a.hkv) {  // one thread's
        int64_t at = before;
        int b = mine0;
        for (;; ++b) {
            const int n = few_parts(paged_seq(a, b));
            if (x0 < (at + n) * a.hkv) break;
            at += n;
        }
        found = b;
        found_before = at;
    }
    __syncthreads();

    int b = found;
    PagedSeq seq = paged_seq(a, b);
    int parts = few_parts(seq);
    int64_t skip = x0 - found_before * a.hkv;
    int head = (int)(skip / parts), part0 = (int)(skip % parts);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    unsigned char* vt = lds + wave * kWaveLds;
    const int vrow = lane >> 4, vchunk = lane & 15;  // of a load or a store of 4 rows of V

    for (int64_t x = x0; x < x1;) {
        const int part1 = (int)min((int64_t)parts, part0 + (x1 - x));
        const int M = seq.count * a.g, len = seq.len;
        const int first = part0 * kPfWaves, last = min(part1 * kPfWaves, (len + kCaKeys - 1) / kCaKeys);
        const int row = min(Rows::row(lane), M - 1), tok = row / a.g, qhead = head * a.g + row % a.g;
        const int p = len - seq.count + tok;
        const __half* qr = static_cast<const __half*>(a.q) + (int64_t)(seq.begin + tok) * a.q_stride + qhead * kD;
        h8v qf[kSteps];
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
            qf[c] = query_part(*reinterpret_cast<const u4v*>(qr + Rows::template dim<false>(c, lane)), flip);
        const ScoreShape<SHAPE> shape(a, qhead);
        Rows rows(SHAPE ? 1.f : score_factor(a.scale), lane);

        // A step's pages, one key a lane (and lane + 32): entries of the table, then rows of K and V
        // and which of them there are.  Keys behind the last repeat it, those without a page the
        // first that has one (there or not, row 0 of the pages is memory).
        auto key_row = [&](int st) { return min(st * kCaKeys + (lane & 31), len - 1); };
        auto entry_of = [&](int st) { return page_entry(a, b, key_row(st)); };
        int at = 0;          // this lane's key's row
        uint32_t there = 0;  // the step's keys that have pages
        auto place = [&](int st, int entry) {
            const bool good = (uint32_t)entry < (uint32_t)a.n_pages;
            there = (uint32_t)__ballot(good);
            at = good ? page_row(a, entry, head, key_row(st)) : 0;
            if (__builtin_expect(there != ~0u, 0)) {
                const int other = there ? __builtin_amdgcn_readlane(at, __builtin_ctz(there)) : 0;
                at = good ? at : other;
            }
        };
        u4v kreg[8], vreg[8];
        auto load = [&]() {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = __builtin_amdgcn_ds_bpermute((4 * i + vrow) << 2, at);
                vreg[i] = reinterpret_cast<const u4v*>(static_cast<const __half*>(a.V) + (int64_t)r * kD)[vchunk];
            }
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const int r = __builtin_amdgcn_ds_bpermute(Rows::key(h, lane) << 2, at);
                const __half* k = static_cast<const __half*>(a.K) + (int64_t)r * kD;
#pragma unroll
                for (int c = 0; c < kSteps; ++c)
                    kreg[h * kSteps + c] = *reinterpret_cast<const u4v*>(k + Rows::template dim<false>(c, lane));
            }
        };
        bool odd = false;  // whether some V there had values that are not finite
        int st = first + wave, entry = 0;
        if (st < last) {
            place(st, entry_of(st));
            load();
            if (st + kPfWaves < last) entry = entry_of(st + kPfWaves);
        }
        for (; st < last; st += kPfWaves) {
            const uint32_t w = bits_to(min(p, len - 1) - st * kCaKeys) & there;
            wave_lds_order();  // the step before has read its V
#pragma unroll
            for (int i = 0; i < 8; ++i) put_v(vt, 4 * i + vrow, vchunk, as_h8(vreg[i]));
            if (__builtin_expect(!__all(w == ~0u), 0)) {
                uint32_t m = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) note_odd(vreg[i], m);
                if (__any(m & kOddBits)) {
                    odd = true;
                    clean_v(vt, lane);
                }
            }
            wave_lds_order();
            rows.scores(qf, [&](int h, int c) { return as_h8(kreg[h * kSteps + c]); });
            if (st + kPfWaves < last) {
                place(st + kPfWaves, entry);
                load();
                if (st + 2 * kPfWaves < last) entry = entry_of(st + 2 * kPfWaves);
            }
            if constexpr (SHAPE != kPlainScores) {
                const float from = (float)(st * kCaKeys - p);
                if constexpr (R == 16) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            rows.s[h][i] = shape(rows.s[h][i], from + (float)(16 * h + 4 * rows.lg + i));
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        rows.s[i] = shape(rows.s[i], from + (float)(8 * (i / 4) + 4 * rows.half + i % 4));
                }
            }
            rows.accumulate(w, vt, lane);
        }

        wave_lds_order();
        rows.leave(vt, lane, odd);
        __syncthreads();
        // Joins the waves' states, 32 lanes a row, 4 dims a lane.
        const bool whole = part0 == 0 && part1 == parts;
        const int slot = 2 * (int)blockIdx.x + (x == x0 ? 0 : 1);
        const float* of = reinterpret_cast<const float*>(lds);
        const float c2 = rows.c2;
        const int d4 = tid & 31;
        for (int r = tid >> 5; r < M; r += kPfThreads / 32) {
            float top = -__builtin_huge_valf(), l = 0.f;
            bool some = false;
            f4v acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kPfWaves; ++w) {
                top = fmaxf(top, of[w * (kWaveLds / 4) + R * kCaRow + r]);
                some |= __builtin_signbit(of[w * (kWaveLds / 4) + R * (kCaRow + 1) + r]);
            }
            if (top > -__builtin_huge_valf())
#pragma unroll
                for (int w = 0; w < kPfWaves; ++w) {
                    const float* ow = of + w * (kWaveLds / 4);
                    const float c = rescale(ow[R * kCaRow + r], top, c2);
                    l += c * __builtin_fabsf(ow[R * (kCaRow + 1) + r]);
                    acc += c * *reinterpret_cast<const f4v*>(ow + r * kCaRow + 4 * d4);
                }
            if (whole) {
                acc *= l > 0.f ? 1.f / l : l;
                if (some) acc += paged_odd_part(a, b, head, len - seq.count + r / a.g, len, d4);
                static_cast<h4v*>(a.out)[((int64_t)(seq.begin + r / a.g) * a.hkv * a.g + head * a.g + r % a.g) * (kD / 4) + d4] =
                    h4v{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
            } else {
                reinterpret_cast<f4v*>(ws.part)[((int64_t)slot * R + r) * (kD / 4) + d4] = acc;
                if (d4 == 0) ws.state[slot * R + r] = float2{top, some ? -l : l};
            }
        }
        x += part1 - part0;
        part0 = 0;
        if (x < x1) {
            __syncthreads();  // the states are read
            if (++head == a.hkv) {
                head = 0;
                do {
                    if (++b >= a.batch) return;  // not with lengths that stay as they are
                    seq = paged_seq(a, b);
                } while (seq.count == 0);
                parts = few_parts(seq);
            }
        }
    }
}

// Joins the states of a row of a head that blocks share: 8 groups of 32 lanes take every eighth
// block, 4 dims a lane.
constexpr int kPcGroups = 8;
template <int R>
__global__ __launch_bounds__(32 * kPcGroups) void paged_few_join_kernel(PagedArgs a, int shaped) {
    __shared__ f4v so[kPcGroups][32];
    __shared__ float sr[kPcGroups], sl[kPcGroups];
    const FewSpace ws = few_space<R>(a);
    const uint32_t rows = (uint32_t)(a.most * a.g);
    const int r = (int)(blockIdx.x % rows), item = (int)(blockIdx.x / rows), b = item / a.hkv, head = item % a.hkv;
    const int64_t b0 = ws.before[b], parts = ws.before[b + 1] - b0, line = ws.before[a.batch] * a.hkv;
    if (parts < 2) return;
    // Block i has the line from i line / blocks on: the blocks of the head's first and last part.
    const int64_t x = b0 * a.hkv + head * parts, blocks = few_used(a, line);
    const int i0 = (int)(((x + 1) * blocks - 1) / line), i1 = (int)(((x + parts) * blocks - 1) / line);
    if (i0 == i1) return;
    const PagedSeq seq = paged_seq(a, b);
    if (r >= seq.count * a.g) return;
    const bool first = i0 * line / blocks == x;  // the head's first block begins with it
    const int d4 = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const float c2 = shaped ? 1.f : score_factor(a.scale);
    bool odd = false;
    float top = -__builtin_huge_valf(), l = 0.f;
    f4v acc{0.f, 0.f, 0.f, 0.f};
    for (int i = i0 + sub; i <= i1; i += kPcGroups) {
        const int64_t at = (int64_t)(2 * i + (i == i0 && !first ? 1 : 0)) * R + r;
        const float2 st = ws.state[at];
        const f4v v = reinterpret_cast<const f4v*>(ws.part)[at * (kD / 4) + d4];
        if (st.x == -__builtin_huge_valf()) continue;  // saw no key
        odd |= __builtin_signbit(st.y);
        const float to = fmaxf(top, st.x);
        const float c0 = rescale(top, to, c2), c1 = rescale(st.x, to, c2);
        l = l * c0 + __builtin_fabsf(st.y) * c1;
        acc = acc * c0 + v * c1;
        top = to;
    }
    so[sub][d4] = acc;
    if (d4 == 0) {
        sr[sub] = top;
        sl[sub] = odd ? -l : l;
    }
    __syncthreads();
    if (sub != 0) return;
    top = -__builtin_huge_valf();
    l = 0.f;
    acc = f4v{0.f, 0.f, 0.f, 0.f};
    odd = false;
#pragma unroll
    for (int i = 0; i < kPcGroups; ++i) {
        top = fmaxf(top, sr[i]);
        odd |= __builtin_signbit(sl[i]);
    }
    if (top > -__builtin_huge_valf())
#pragma unroll
        for (int i = 0; i < kPcGroups; ++i) {
            const float c = rescale(sr[i], top, c2);
            l += c * __builtin_fabsf(sl[i]);
            acc += c * so[i][d4];
        }
    acc *= l > 0.f ? 1.f / l : l;
    const int tok = r / a.g;
    if (odd) acc += paged_odd_part(a, b, head, seq.len - seq.count + tok, seq.len, d4);
    static_cast<h4v*>(a.out)[((int64_t)(seq.begin + tok) * a.hkv * a.g + head * a.g + r % a.g) * (kD / 4) + d4] =
        h4v{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
}

}  // namespace

size_t paged_plan(PagedArgs& a) {
    const int64_t rows = (int64_t)a.most * a.g;
    const int R = few_rows(rows);
    // No more blocks than parts of full tables.
    const int64_t parts = (a.width * a.page.d + kPfKeys - 1) / kPfKeys * a.batch * a.hkv;
    a.blocks = (int32_t)(parts < few_blocks(R) ? (parts < 1 ? 1 : parts) : few_blocks(R));
    auto few = [&](int r) { return few_line_bytes(a.batch) + (size_t)2 * few_blocks(r) * r * (kD + 2) * 4; };
    size_t bytes = few(16);
    if (rows > 16 && few(32) > bytes) bytes = few(32);
    if (rows > 32 && paged_prompt_bytes(a) > bytes) bytes = paged_prompt_bytes(a);
    return bytes;
}

hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.most * a.g;
    if (rows > 32) return launch_paged_prompt(a, s);
    const int shape = (a.cap > 0.f ? kCappedScores : 0) | (a.slopes ? kBiasedScores : 0);
    ProfEvents pe = prof_begin("paged_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)a.blocks), dim3(kPfThreads), 0, s, pe.start, pe.stop, 0, a);
    };
    auto by_rows = [&](auto k16, auto k32) { few_rows(rows) == 16 ? go(k16) : go(k32); };
    if (shape == kPlainScores) by_rows(paged_few_kernel<16, 0>, paged_few_kernel<32, 0>);
    else if (shape == kCappedScores) by_rows(paged_few_kernel<16, 1>, paged_few_kernel<32, 1>);
    else if (shape == kBiasedScores) by_rows(paged_few_kernel<16, 2>, paged_few_kernel<32, 2>);
    else by_rows(paged_few_kernel<16, 3>, paged_few_kernel<32, 3>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.blocks == 1) return e;
    pe = prof_begin("paged_join");
    auto join = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)(rows * a.batch * a.hkv)), dim3(32 * kPcGroups), 0, s, pe.start,
                              pe.stop, 0, a, shape);
    };
    few_rows(rows) == 16 ? join(paged_few_join_kernel<16>) : join(paged_few_join_kernel<32>);
    return hipGetLastError();
}

}  // namespace pariskv
