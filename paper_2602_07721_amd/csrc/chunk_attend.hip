// Attention of a few new tokens per sequence over a long cache, on matrix instructions.
//
// The g heads of a KV head times the t new tokens are M = g t rows over the same keys, so a
// key's row is read once for 16 NQ of them (NQ tiles of 16 rows a block).  Per wave and 32 keys:
//   S^T = K Q^T    a lane holds 8 keys' scores of one row per tile of 16 rows,
//   P              exp2 of the scores less the row's running maximum,
//   O^T += V^T P^T the scores' own registers are the second operand: matrix instructions sum
//                  over 32 keys in any order, as long as both operands agree on it.
// K goes from HBM to registers as the operand it is.  V^T needs a column's keys in one lane:
// V goes through 8 KB of LDS of the wave's own and a transposing read; chunks of 16 bytes are
// XORed with the key so that the 16 rows of such a read fall on all banks.  The next 32 keys'
// loads are in flight meanwhile.  Waves share nothing until the end, when their states
// (maximum, sum, outputs) are joined through LDS; blocks that share a sequence's keys leave
// theirs in the workspace for a second kernel.
//
// Float32 results from float16 instructions: products are exact and summed in float32; P is
// split into two float16 values (their sum is P to 2^-22 of it), two instructions instead of
// one.  The maximum is raised only when a score exceeds it by 2^7, so that P, scaled by 2^8,
// stays below 2^16 and small P lose nothing.

#include <hip/hip_fp16.h>

#include "chunk_attend_device.hpp"

namespace pariskv {

namespace {

constexpr int kCaThreads = 256;
constexpr int kCaWaves = kCaThreads / 64;
constexpr int kCaKeys = 32;            // keys of a wave's step
constexpr float kCaUp = 8.f;           // P is held scaled by 2^8 ...
constexpr float kCaSlack = 7.f;        // ... and grows by up to 2^7 before the maximum is raised
constexpr int64_t kCaBlocks = 1024;     // blocks that a call's keys are shared out to
constexpr int kCaRow = kD + 4;         // floats of an output row in LDS (spreads the rows over the banks)

constexpr size_t ca_lds_bytes(int nq) {
    const size_t v = (size_t)kCaWaves * kCaKeys * kD * 2;
    const size_t o = (size_t)kCaWaves * 16 * nq * (kCaRow + 2) * 4;
    return v > o ? v : o;
}

// 4 dims of an output row: float32, or float16 where the prompt's next product reads it.  Rows
// of tokens that are not there are left as they were.
template <bool WINDOW>
__device__ __forceinline__ void store_row(const ChunkArgs& a, int64_t row, int d4, float inv, f4v acc, bool real) {
    acc *= inv;
    if constexpr (WINDOW) {
        const h4v h{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
        if (real) static_cast<h4v*>(a.out)[row * (kD / 4) + d4] = h;
    } else {
        static_cast<f4v*>(a.out)[row * (kD / 4) + d4] = acc;
    }
}

// Registers of 32 keys of a wave, as loaded.  K: lane l holds key l % 16 of each half, of the
// dims that step_dim names; V: 8 loads of 4 whole rows.
template <int BITS>
struct KeyRegs {
    u4v k[2][BITS / 4];
    uint32_t scale[2];
};
template <int BITS>
struct ValueRegs {
    u2v v[8];
    uint32_t scale[8];
};
template <>
struct ValueRegs<16> {
    u4v v[8];
};

// Dims of matrix step c that lane group l / 16 holds start here.  A quantised key's lane group
// holds one whole block (one scale a lane); a float16 key's four lanes read 64 bytes in a row.
template <bool QUANT>
__device__ __forceinline__ int step_dim(int c, int grp) {
    return QUANT ? 32 * grp + 8 * c : 32 * c + 8 * grp;
}

// A step's 32 keys: rows of a float16 cache, of the drafts or of a quantised cache, of which the
// first `valid` exist.
struct StepRows {
    const __half* k;
    const __half* v;
    const uint8_t* rec;
    int valid;
    int base;    // cache row of key 0
    int drafts;  // < 0, or the number of the draft that key 0 is
};

template <int NQ, int KB, int VB, bool WINDOW>
__global__ __launch_bounds__(kCaThreads, 2) void chunk_attend_kernel(ChunkArgs a, int mtiles, int64_t groups) {
    constexpr bool kQuant = KB < 16;
    constexpr int kRecord = kQuant ? quant_record_bytes(KB, VB) : 0;
    constexpr int kRows = 16 * NQ;
    __shared__ __attribute__((aligned(16))) unsigned char lds[ca_lds_bytes(NQ)];

    // Consecutive blocks go to the 8 XCDs in turn: the row tiles of one share of the keys are 8
    // apart, so that one XCD's L2 serves them all.
    int64_t id = blockIdx.x;
    const int64_t shares = groups * a.splits;
    const int64_t full = shares / 8 * 8 * mtiles;
    int mt;
    int64_t share;
    if (id < full) {
        share = id / (8 * mtiles) * 8 + id % 8;
        mt = (int)(id / 8 % mtiles);
    } else {
        id -= full;
        share = full / mtiles + id / mtiles;
        mt = (int)(id % mtiles);
    }
    const int64_t grp = share / a.splits;
    const int split = (int)(share % a.splits);
    const int seq = (int)(grp / a.hkv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, lg = lane >> 4;
    const int M = a.g * a.t, row0 = mt * kRows;
    const KeySpan span = key_span(a, seq, 0, a.t);

    // Steps of 32 keys: the sinks', the cached stretch's; this share's part of them, and the
    // drafts behind the last share's.
    const int sink_steps = (span.sink_end + kCaKeys - 1) / kCaKeys;
    const int steps = sink_steps + (span.hi - span.lo + kCaKeys - 1) / kCaKeys;
    const int per = (steps + a.splits - 1) / a.splits;
    const int first = min(split * per, steps), last = min(first + per, steps);
    const int draft_steps = (!WINDOW && split == a.splits - 1) ? (a.t + kCaKeys - 1) / kCaKeys : 0;
    const int end = last + draft_steps;

    const float c2 = score_factor(a.scale);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    h8v qf[NQ][4];
    int tok[NQ];  // token of this lane's row
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int r = min(row0 + 16 * x + col, M - 1);
        tok[x] = r % a.t;
        const __half* qr = static_cast<const __half*>(a.q) + (grp * M + r) * kD;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            qf[x][c] = query_part(*reinterpret_cast<const u4v*>(qr + step_dim<kQuant>(c, lg)), flip);
    }

    // A row's running maximum m as nm = 8 - m (P = 2^(c2 s + nm)), its sum over this lane's
    // keys, its outputs: lane holds dims 16 d + 4 lg + i of row col.
    float nm[NQ], sum[NQ];
    f4v o[NQ][8];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        nm[x] = __builtin_huge_valf();
        sum[x] = 0.f;
#pragma unroll
        for (int d = 0; d < 8; ++d) o[x][d] = f4v{0.f, 0.f, 0.f, 0.f};
    }

    unsigned char* vt = lds + wave * (kCaKeys * kD * 2);
    // Where this lane's transposing reads begin: key 4 lg + col / 4 of a half, dims 16 d + 4 (col % 4).
    const int tkey = 4 * lg + (col >> 2);
    const unsigned char* tr = vt + tkey * 256 + ((col & 3) >> 1) * 16 + (col & 1) * 8;
    // 16 bytes of key `key`'s V (chunk `chunk` of 16) into the wave's LDS.
    auto put_v = [&](int key, int chunk, h8v v) {
        *reinterpret_cast<h8v*>(vt + key * 256 + ((chunk ^ (2 * (key & 7))) << 4)) = v;
    };

    auto rows_of = [&](int st) {
        StepRows r{};
        r.drafts = -1;
        if (!WINDOW && st >= last) {
            r.drafts = (st - last) * kCaKeys;
            const int64_t at = grp * a.t + r.drafts;
            r.k = static_cast<const __half*>(a.Kt) + at * kD;
            r.v = static_cast<const __half*>(a.Vt) + at * kD;
            r.valid = a.t - r.drafts;
            return r;
        }
        const bool sink = WINDOW && st < sink_steps;
        r.base = sink ? st * kCaKeys : span.lo + (st - sink_steps) * kCaKeys;
        r.valid = (sink ? span.sink_end : span.hi) - r.base;
        const int64_t at = grp * a.capacity + r.base;
        if constexpr (kQuant) {
            r.rec = a.rec + at * kRecord;
        } else {
            r.k = static_cast<const __half*>(a.K) + at * kD;
            r.v = static_cast<const __half*>(a.V) + at * kD;
        }
        return r;
    };
    // Keys past the last repeat it: what lies behind is not read.
    auto load_k = [&](const StepRows& r, KeyRegs<KB>& kr) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = min(16 * h + col, r.valid - 1);
            if constexpr (kQuant) {
                const uint8_t* p = r.rec + key * kRecord;
#pragma unroll
                for (int c = 0; c < KB / 4; ++c) kr.k[h][c] = reinterpret_cast<const u4v*>(p + lg * (4 * KB))[c];
                kr.scale[h] = *reinterpret_cast<const uint32_t*>(p + quant_code_bytes(KB) + quant_code_bytes(VB));
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    kr.k[h][c] = *reinterpret_cast<const u4v*>(r.k + key * kD + step_dim<false>(c, lg));
            }
        }
    };
    auto load_v = [&](const StepRows& r, ValueRegs<VB>& vr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int key = min(4 * i + lg, r.valid - 1);
            if constexpr (kQuant) {
                const uint8_t* p = r.rec + key * kRecord + quant_code_bytes(KB);
                vr.v[i] = quant_load8<VB>(p + col * VB);
                vr.scale[i] = *reinterpret_cast<const uint32_t*>(p + quant_code_bytes(VB) + 4);
            } else {
                vr.v[i] = reinterpret_cast<const u4v*>(r.v + key * kD)[col];
            }
        }
    };
    auto key_part = [&](const KeyRegs<KB>& kr, int h, int c) {
        if constexpr (KB == 16) {
            return as_h8(kr.k[h][c]);
        } else {
            const float sc = quant_scale_value((kr.scale[h] >> (8 * lg)) & 255u);
            if constexpr (KB == 8)
                return quant_decode8<8>(kr.k[h][c / 2][2 * (c % 2)], kr.k[h][c / 2][2 * (c % 2) + 1], sc);
            else
                return quant_decode8<4>(kr.k[h][0][c], 0u, sc);
        }
    };

    f4v s[NQ][2];
    auto scores = [&](auto&& kpart) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const h8v kf = kpart(h, c);
#pragma unroll
                for (int x = 0; x < NQ; ++x)
                    s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        kf, qf[x][c], c == 0 ? f4v{0.f, 0.f, 0.f, 0.f} : s[x][h], 0, 0, 0);
            }
    };
    // From the step's scores s and its V in LDS; bits of w[x]: the keys that row tile x sees.
    auto accumulate = [&](const uint32_t (&w)[NQ]) {
        bool all_seen = true, raise = false;
#pragma unroll
        for (int x = 0; x < NQ; ++x) all_seen &= w[x] == ~0u;
        if (!__all(all_seen)) {
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const uint32_t b = w[x] >> (4 * lg);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(b & (1u << (16 * h + i)))) s[x][h][i] = -__builtin_huge_valf();
            }
        }
        float top[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            top[x] = -__builtin_huge_valf();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) top[x] = fmaxf(top[x], s[x][h][i]);
            top[x] *= c2;
            // nm = inf: no key seen yet.
            raise |= top[x] > -__builtin_huge_valf() && !(top[x] + nm[x] <= kCaUp + kCaSlack);
        }
        if (__any(raise)) {
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const float to = kCaUp - rows_max(top[x]);  // inf where the row saw nothing in this step
                if (to < nm[x]) {
                    const float c = __builtin_amdgcn_exp2f(to - nm[x]);  // 0 before the first key
                    nm[x] = to;
                    sum[x] *= c;
#pragma unroll
                    for (int d = 0; d < 8; ++d) o[x][d] *= c;
                }
            }
        }
        h8v hi[NQ], lo[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            const float base = nm[x] < __builtin_huge_valf() ? nm[x] : 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][h][i], c2, base));
                    sum[x] += p;
                    hi[x][4 * h + i] = (_Float16)p;
                    lo[x][4 * h + i] = (_Float16)(p - (float)hi[x][4 * h + i]);
                }
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            typedef __attribute__((address_space(3))) s4v* lds_s4;
            const unsigned char* at = tr + ((d ^ (tkey & 7)) << 5);
            const s4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(at));
            const s4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(at + 16 * 256));
            const h8v vf = join_h4(v0, v1);
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, hi[x], o[x][d], 0, 0, 0);
                o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, lo[x], o[x][d], 0, 0, 0);
            }
        }
    };

    // Drafts that some token of the sequence sees; the others may hold anything, and count as 0.
    uint64_t used = ~0ull;
    const int64_t* masks = !WINDOW && a.mask ? a.mask + (int64_t)seq * a.t : nullptr;
    if (draft_steps > 0 && masks) {
        used = lane < a.t ? (uint64_t)masks[lane] : 0ull;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1)
            used |= (uint64_t)lane_xor((uint32_t)used, m, lane) | (uint64_t)lane_xor((uint32_t)(used >> 32), m, lane) << 32;
    }
    auto draft_bits = [&](int x, const StepRows& r) {
        const uint64_t m = masks ? (uint64_t)masks[tok[x]] : ~0ull >> (63 - tok[x]);
        return (uint32_t)(m >> r.drafts) & bits_to(r.valid - 1);
    };

    // Quantised kernels take the drafts, which are float16, in a loop of their own.
    const int main_end = kQuant ? last : end;
    KeyRegs<KB> kr;
    ValueRegs<VB> vr;
    int st = first + wave;
    StepRows cur{};
    if (st < main_end) {
        cur = rows_of(st);
        load_v(cur, vr);
        load_k(cur, kr);
    }
    for (; st < main_end; st += kCaWaves) {
        const bool more = st + kCaWaves < main_end;
        StepRows next = cur;
        if (more) next = rows_of(st + kCaWaves);
        wave_lds_order();  // the step before has read its V
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kQuant) {
                put_v(4 * i + lg, col,
                      quant_decode8<VB>(vr.v[i].x, vr.v[i].y,
                                        quant_scale_value((vr.scale[i] >> (8 * (col >> 2))) & 255u)));
            } else {
                u4v v = vr.v[i];
                if (!WINDOW && cur.drafts >= 0 && !((used >> (cur.drafts + 4 * i + lg)) & 1)) v = u4v{0u, 0u, 0u, 0u};
                put_v(4 * i + lg, col, as_h8(v));
            }
        }
        wave_lds_order();
        if (more) load_v(next, vr);
        scores([&](int h, int c) { return key_part(kr, h, c); });
        if (more) load_k(next, kr);
        uint32_t w[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            w[x] = bits_to(cur.valid - 1);
            if constexpr (WINDOW) w[x] &= window_bits(span.start + tok[x], cur.base, (int)a.sink, (int)a.window);
            else if (!kQuant && cur.drafts >= 0) w[x] = draft_bits(x, cur);
        }
        accumulate(w);
        cur = next;
    }
    if constexpr (kQuant) {
        for (; st < end; st += kCaWaves) {
            const StepRows r = rows_of(st);
            wave_lds_order();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = 4 * i + lg;
                u4v v = reinterpret_cast<const u4v*>(r.v + min(key, r.valid - 1) * kD)[col];
                if (!((used >> (r.drafts + key)) & 1)) v = u4v{0u, 0u, 0u, 0u};
                put_v(key, col, as_h8(v));
            }
            wave_lds_order();
            scores([&](int h, int c) {
                return as_h8(*reinterpret_cast<const u4v*>(r.k + min(16 * h + col, r.valid - 1) * kD +
                                                           step_dim<true>(c, lg)));
            });
            uint32_t w[NQ];
#pragma unroll
            for (int x = 0; x < NQ; ++x) w[x] = draft_bits(x, r);
            accumulate(w);
        }
    }

    // Join the waves' states: [wave][row][dims], then each row's nm and sum.
    __syncthreads();
    float* so = reinterpret_cast<float*>(lds);
    float* snm = so + kCaWaves * kRows * kCaRow;
    float* ssum = snm + kCaWaves * kRows;
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const float l = rows_sum(sum[x]);
        const int r = wave * kRows + 16 * x + col;
        if (lg == 0) {
            snm[r] = nm[x];
            ssum[r] = l;
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) *reinterpret_cast<f4v*>(so + r * kCaRow + 16 * d + 4 * lg) = o[x][d];
    }
    __syncthreads();
    // 32 lanes a row, 4 dims a lane.
    for (int r = threadIdx.x >> 5; r < kRows; r += kCaThreads / 32) {
        if (row0 + r >= M) break;
        const int d4 = threadIdx.x & 31;
        float top = __builtin_huge_valf();
#pragma unroll
        for (int w = 0; w < kCaWaves; ++w) top = fminf(top, snm[w * kRows + r]);
        float l = 0.f;
        f4v acc{0.f, 0.f, 0.f, 0.f};
        if (top < __builtin_huge_valf())
#pragma unroll
            for (int w = 0; w < kCaWaves; ++w) {
                const float c = __builtin_amdgcn_exp2f(top - snm[w * kRows + r]);
                l += c * ssum[w * kRows + r];
                acc += c * *reinterpret_cast<const f4v*>(so + (w * kRows + r) * kCaRow + 4 * d4);
            }
        const int64_t row = grp * M + row0 + r;
        if (a.splits > 1) {
            const int64_t at = row * a.splits + split;
            reinterpret_cast<f4v*>(a.part)[at * (kD / 4) + d4] = acc;
            if (d4 == 0) {
                float* ml = a.part + groups * M * a.splits * kD + 2 * at;
                ml[0] = top;
                ml[1] = l;
            }
        } else {
            store_row<WINDOW>(a, row, d4, l > 0.f ? 1.f / l : 0.f, acc, (row0 + r) % a.t < span.tokens);
        }
    }
}

// Joins the shares' states of a row: 8 groups of 32 lanes take every eighth share, 4 dims a lane.
constexpr int kCcGroups = 8;
template <bool WINDOW>
__global__ __launch_bounds__(32 * kCcGroups) void chunk_combine_kernel(ChunkArgs a, int64_t rows) {
    __shared__ f4v so[kCcGroups][32];
    __shared__ float snm[kCcGroups], sl[kCcGroups];
    const int64_t row = blockIdx.x;
    const int d4 = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const int M = a.g * a.t;
    const float* ml = a.part + rows * a.splits * kD + 2 * row * a.splits;
    const f4v* part = reinterpret_cast<const f4v*>(a.part) + row * a.splits * (kD / 4) + d4;
    float top = __builtin_huge_valf(), l = 0.f;
    f4v acc{0.f, 0.f, 0.f, 0.f};
    for (int s = sub; s < a.splits; s += kCcGroups) {
        const float nm = ml[2 * s], ls = ml[2 * s + 1];
        const f4v v = part[s * (kD / 4)];
        const float to = fminf(top, nm);
        if (to < __builtin_huge_valf()) {
            const float c0 = __builtin_amdgcn_exp2f(to - top), c1 = __builtin_amdgcn_exp2f(to - nm);
            l = l * c0 + ls * c1;
            acc = acc * c0 + v * c1;
            top = to;
        }
    }
    so[sub][d4] = acc;
    if (d4 == 0) {
        snm[sub] = top;
        sl[sub] = l;
    }
    __syncthreads();
    if (sub != 0) return;
    top = __builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < kCcGroups; ++i) top = fminf(top, snm[i]);
    l = 0.f;
    acc = f4v{0.f, 0.f, 0.f, 0.f};
    if (top < __builtin_huge_valf())
#pragma unroll
        for (int i = 0; i < kCcGroups; ++i) {
            const float c = __builtin_amdgcn_exp2f(top - snm[i]);
            l += c * sl[i];
            acc += c * so[i][d4];
        }
    bool real = true;
    if (WINDOW && a.counts) real = (int)(row % M) % a.t < a.counts[row / M / a.hkv];
    store_row<WINDOW>(a, row, d4, l > 0.f ? 1.f / l : 0.f, acc, real);
}

}  // namespace

// 16 or 32 rows a block: 64 would need every register of a SIMD for one wave.
static int chunk_row_tiles(int64_t rows) { return rows <= 16 ? 1 : 2; }

int32_t chunk_splits(int64_t groups, int64_t rows, int64_t keys) {
    const int64_t nq = chunk_row_tiles(rows), mtiles = (rows + 16 * nq - 1) / (16 * nq);
    const int64_t want = kCaBlocks;
    int64_t s = (want + groups * mtiles - 1) / (groups * mtiles);
    const int64_t most = keys / (2 * kCaWaves * kCaKeys);  // no shorter than 2 steps of every wave
    if (s > most) s = most;
    if (s > 256) s = 256;
    return (int32_t)(s < 1 ? 1 : s);
}

size_t chunk_part_bytes(int64_t groups, int64_t rows, int32_t splits) {
    return splits > 1 ? (size_t)(groups * rows) * (size_t)splits * (kD + 2) * 4 : 0;
}

hipError_t launch_chunk_attend(const ChunkArgs& a, hipStream_t s) {
    const int64_t groups = (int64_t)a.batch * a.hkv;
    const int M = a.g * a.t;
    const int nq = chunk_row_tiles(M);
    const int mtiles = (M + 16 * nq - 1) / (16 * nq);
    const dim3 grid((unsigned)(groups * a.splits * mtiles));
    ProfEvents pe = prof_begin(a.window > 0 ? "sink_window_attend" : a.rec ? "quant_tree_attend" : "tree_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, grid, dim3(kCaThreads), 0, s, pe.start, pe.stop, 0, a, mtiles, groups);
    };
    auto rows = [&](auto k1, auto k2) { nq == 1 ? go(k1) : go(k2); };
    if (a.window > 0)
        rows(chunk_attend_kernel<1, 16, 16, true>, chunk_attend_kernel<2, 16, 16, true>);
    else if (!a.rec)
        rows(chunk_attend_kernel<1, 16, 16, false>, chunk_attend_kernel<2, 16, 16, false>);
    else if (a.k_bits == 8 && a.v_bits == 8)
        rows(chunk_attend_kernel<1, 8, 8, false>, chunk_attend_kernel<2, 8, 8, false>);
    else if (a.k_bits == 8)
        rows(chunk_attend_kernel<1, 8, 4, false>, chunk_attend_kernel<2, 8, 4, false>);
    else if (a.v_bits == 8)
        rows(chunk_attend_kernel<1, 4, 8, false>, chunk_attend_kernel<2, 4, 8, false>);
    else
        rows(chunk_attend_kernel<1, 4, 4, false>, chunk_attend_kernel<2, 4, 4, false>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t all = groups * M;
    const dim3 cgrid((unsigned)all);
    pe = prof_begin("chunk_combine");
    if (a.window > 0)
        hipExtLaunchKernelGGL(chunk_combine_kernel<true>, cgrid, dim3(32 * kCcGroups), 0, s, pe.start, pe.stop, 0, a, all);
    else
        hipExtLaunchKernelGGL(chunk_combine_kernel<false>, cgrid, dim3(32 * kCcGroups), 0, s, pe.start, pe.stop, 0, a, all);
    return hipGetLastError();
}

}  // namespace pariskv
