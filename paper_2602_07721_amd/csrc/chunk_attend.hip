// Attention of a few new tokens per sequence over a long cache, on matrix instructions.
//
// The g heads of a KV head times the t new tokens are M = g t rows over the same keys; a wave
// holds 16 or 32 of them.  Per wave and 32 keys:
//   S^T = K Q^T    a lane holds 8 or 16 keys' scores of one row,
//   P              exp2 of the scores less the row's running maximum,
//   O^T += V^T P^T the scores' own registers are the second operand: matrix instructions sum
//                  over 32 keys in any order, as long as both operands agree on it.
// Float32 results from float16 instructions: products are exact and summed in float32; P is
// split into two float16 values, two instructions instead of one, which leave 2^-22 of it or
// 2^-25, half their smallest step.  P is at least 2^8 for the largest weight, so that is 2^-33 of
// the largest weight, for a key that weighs less than 2^-11 of it; n such keys shift an output by
// up to n 2^-33 of the largest |v|.  The reference score is raised only when a weight passes 2^7
// times its own, so P stays below 2^16.
//
// Here, up to 32 rows: bound by HBM, so each wave walks keys of its own, nothing is shared and
// nothing waits.  Float16 K goes from HBM to registers as the operand it is.  V^T needs a
// column's keys in one lane: V goes through 8 KB of LDS of the wave's own and a transposing
// read.  The next keys' loads are in flight meanwhile.  Records are loaded as they lie, 1 KB of
// them an instruction, and taken apart in LDS: read part by part, the parts of a cache line
// reach it at different times and fetch it twice (128K records x 64, 32 rows: 456 us so, 419
// whole).  The waves' states are joined through LDS at the end, the states of blocks that share
// a sequence's keys by a second kernel.

#include <hip/hip_fp16.h>

#include "chunk_attend_device.hpp"

namespace pariskv {

namespace {

constexpr int kCaWaves = 4;  // waves of a block
constexpr int kCaMaxShares = 256;  // of a sequence's keys
constexpr int kFewTokens = 1024;   // the few-token form of the sliding window takes no more

// LDS of one wave: its V and its records, later its state.
constexpr int kCaVBytes = kCaKeys * kD * 2;
constexpr int ca_wave_lds(int rows, int record) {
    const int v = kCaVBytes + kCaKeys * record, o = ca_state_bytes(rows);
    return v > o ? v : o;
}

// Registers of 32 keys of a wave, as loaded.  Float16 K: the operand that ChunkRows names; V: 8
// loads of 4 whole rows.  Records: the 32 of them as they lie, 1 KB a load.
template <int KB, int VB>
struct StepRegs {
    static constexpr int kChunks = kCaKeys * quant_record_bytes(KB, VB) / 16;
    u4v raw[(kChunks + 63) / 64];
};
template <>
struct StepRegs<16, 16> {
    static constexpr int kChunks = 0;
    u4v k[8], v[8];
};

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

// 16 rows of float16 keys: 3 blocks a CU.
template <int R, int KB, int VB, bool WINDOW>
__global__ __launch_bounds__(64 * kCaWaves, R == 16 && KB == 16 ? 3 : 2) void chunk_attend_kernel(ChunkArgs a, int row_tiles, int64_t groups) {
    constexpr bool kQuant = KB < 16;
    constexpr int kRecord = kQuant ? quant_record_bytes(KB, VB) : 0;
    constexpr int kChunks = StepRegs<KB, VB>::kChunks;
    constexpr int kLoads = (kChunks + 63) / 64;
    constexpr int kWaveLds = ca_wave_lds(R, kRecord);
    // Steps whose loads are in flight: two of records where the registers hold them (32 rows and
    // 8-bit codes do not leave room), one of float16 rows.
    constexpr int kAhead = kQuant && (R == 16 || kLoads <= 5) ? 2 : 1;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kCaWaves * kWaveLds];

    const ChunkPlace pl = chunk_place(a, row_tiles, groups);
    const int64_t grp = pl.grp;
    const int seq = pl.seq;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    using Rows = ChunkRows<R>;
    constexpr int kHalves = Rows::kHalves, kSteps = Rows::kSteps;
    const int M = a.g * a.t, row0 = pl.tile * R;
    const KeySpan span = key_span(a, seq, 0, a.t);

    // Steps of 32 keys: the sinks', the cached stretch's; this share's part of them, and the
    // drafts behind the last share's.
    const int sink_steps = (span.sink_end + kCaKeys - 1) / kCaKeys;
    const int steps = sink_steps + (span.hi - span.lo + kCaKeys - 1) / kCaKeys;
    const bool closing = pl.split == a.splits - 1;  // takes what is left, and the drafts
    const int first = min(pl.split * a.per, steps), last = closing ? steps : min(first + a.per, steps);
    const int draft_steps = (!WINDOW && closing) ? (a.t + kCaKeys - 1) / kCaKeys : 0;
    const int end = last + draft_steps;
    if (first >= end && a.splits > 1) return leave_idle(a, pl, groups, row0, R);

    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    const int row = min(row0 + Rows::row(lane), M - 1), tok = row % a.t;  // this lane's
    const __half* qr = static_cast<const __half*>(a.q) + (grp * M + row) * kD;
    h8v qf[kSteps];
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
        qf[c] = query_part(*reinterpret_cast<const u4v*>(qr + Rows::template dim<kQuant>(c, lane)), flip);
    Rows rows(score_factor(a.scale), lane);

    unsigned char* vt = lds + wave * kWaveLds;
    unsigned char* rt = vt + kCaVBytes;  // the step's records
    const int vrow = lane >> 4, vchunk = lane & 15;  // of a load or a store of 4 rows of V

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
        r.valid = min((sink ? span.sink_end : span.hi) - r.base, kCaKeys);
        const int64_t at = grp * a.capacity + r.base;
        if constexpr (kQuant) {
            r.rec = a.rec + at * kRecord;
        } else {
            r.k = static_cast<const __half*>(a.K) + at * kD;
            r.v = static_cast<const __half*>(a.V) + at * kD;
        }
        return r;
    };
    // What lies behind the last key is not read: rows repeat it, records are cleared in take().
    auto load = [&](const StepRows& r, StepRegs<KB, VB>& regs) {
        if constexpr (kQuant) {
            const u4v* p = reinterpret_cast<const u4v*>(r.rec);
            const int most = r.valid * (kRecord / 16) - 1;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) regs.raw[i] = p[min(64 * i + lane, most)];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                regs.v[i] = reinterpret_cast<const u4v*>(r.v + min(4 * i + vrow, r.valid - 1) * kD)[vchunk];
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int c = 0; c < kSteps; ++c)
                    regs.k[h * kSteps + c] = *reinterpret_cast<const u4v*>(
                        r.k + min(Rows::key(h, lane), r.valid - 1) * kD + Rows::template dim<false>(c, lane));
        }
    };
    bool odd = false;  // whether some V there had values that are not finite
    // Quantised kernels take the drafts, which are float16, in a loop of their own.
    const int main_end = kQuant ? last : end;
    StepRegs<KB, VB> regs[kAhead];
    // Step st, whose rows are in `reg`; loads those of step st + kAhead kCaWaves into it.
    auto take = [&](int st, StepRegs<KB, VB>& reg) {
        const StepRows cur = rows_of(st);
        const int ahead = st + kAhead * kCaWaves;
        uint32_t w = bits_to(cur.valid - 1);
        if constexpr (WINDOW) w &= window_bits(span.start + tok, cur.base, (int)a.sink, (int)a.window);
        else if (!kQuant && cur.drafts >= 0) w = draft_bits(a, seq, tok, cur.drafts, cur.valid);
        wave_lds_order();  // the step before has read its V
        if constexpr (kQuant) {
            // Records that are not there: codes of 0, not what the bytes of another part would mean.
            const int have = cur.valid * (kRecord / 16);
            if (have < kChunks)
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    if (64 * i + lane >= have) reg.raw[i] = u4v{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (64 * i + 64 <= kChunks || 64 * i + lane < kChunks)
                    reinterpret_cast<u4v*>(rt)[64 * i + lane] = reg.raw[i];
            if (ahead < main_end) load(rows_of(ahead), reg);
            wave_lds_order();
            // Everything is read before V is written: the reads need not wait for each other.
            u2v vc[8];
            uint32_t vs[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned char* p = rt + (4 * i + vrow) * kRecord + quant_code_bytes(KB);
                vc[i] = quant_load8<VB>(p + vchunk * VB);
                vs[i] = p[quant_code_bytes(VB) + 4 + (vchunk >> 2)];
            }
            // 128 / kHalves bits of codes a step of 8 dims, and a scale for every 4 of them.
            constexpr int kWords = kSteps * KB / 16;
            u4v kc[kHalves][kWords];
            float ks[kHalves][kSteps / 4];
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const unsigned char* p = rt + Rows::key(h, lane) * kRecord;
                const int d0 = Rows::template dim<true>(0, lane);
#pragma unroll
                for (int c = 0; c < kWords; ++c) kc[h][c] = reinterpret_cast<const u4v*>(p + d0 * KB / 8)[c];
#pragma unroll
                for (int c = 0; c < kSteps / 4; ++c)
                    ks[h][c] = quant_scale_value(p[quant_code_bytes(KB) + quant_code_bytes(VB) + d0 / 32 + c]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                put_v(vt, 4 * i + vrow, vchunk, quant_decode8<VB>(vc[i][0], vc[i][1], quant_scale_value(vs[i])));
            wave_lds_order();
            rows.scores(qf, [&](int h, int c) {
                if constexpr (KB == 8)
                    return quant_decode8<8>(kc[h][c / 2][2 * (c % 2)], kc[h][c / 2][2 * (c % 2) + 1], ks[h][c / 4]);
                else
                    return quant_decode8<4>(kc[h][c / 4][c % 4], 0u, ks[h][c / 4]);
            });
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) put_v(vt, 4 * i + vrow, vchunk, as_h8(reg.v[i]));
            if (WINDOW ? !__all(w == ~0u) : cur.drafts >= 0) {
                uint32_t m = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) note_odd(reg.v[i], m);
                if (__builtin_expect(__any(m & kOddBits), 0)) {
                    odd = true;
                    clean_v(vt, lane);
                }
            }
            wave_lds_order();
            rows.scores(qf, [&](int h, int c) { return as_h8(reg.k[h * kSteps + c]); });
            if (ahead < main_end) load(rows_of(ahead), reg);
        }
        rows.accumulate(w, vt, lane);
    };

    int st = first + wave;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (st + i * kCaWaves < main_end) load(rows_of(st + i * kCaWaves), regs[i]);
    for (; st < main_end; st += kCaWaves) {
        take(st, regs[0]);
        if constexpr (kAhead == 2) {
            st += kCaWaves;
            if (st >= main_end) break;
            take(st, regs[1]);
        }
    }
    if constexpr (kQuant) {
        for (int ds = st - last; ds < draft_steps; ds += kCaWaves) {
            const StepRows r = rows_of(last + ds);
            uint32_t m = 0u;
            wave_lds_order();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = 4 * i + vrow;
                const u4v v = reinterpret_cast<const u4v*>(r.v + min(key, r.valid - 1) * kD)[vchunk];
                note_odd(v, m);
                put_v(vt, key, vchunk, as_h8(v));
            }
            if (__builtin_expect(__any(m & kOddBits), 0)) {
                odd = true;
                clean_v(vt, lane);
            }
            wave_lds_order();
            rows.scores(qf, [&](int h, int c) {
                return as_h8(*reinterpret_cast<const u4v*>(r.k + min(Rows::key(h, lane), r.valid - 1) * kD +
                                                           Rows::template dim<true>(c, lane)));
            });
            rows.accumulate(draft_bits(a, seq, tok, r.drafts, r.valid), vt, lane);
        }
    }

    __syncthreads();
    rows.leave(vt, lane, odd);
    __syncthreads();
    join_waves<R, kCaWaves, WINDOW>(a, pl, groups, row0, span.tokens, lds, kWaveLds, threadIdx.x >> 5, 2 * kCaWaves);
}

// Joins the shares' states of a row: 8 groups of 32 lanes take every eighth share, 4 dims a lane.
constexpr int kCcGroups = 8;
template <bool WINDOW>
__global__ __launch_bounds__(32 * kCcGroups) void chunk_combine_kernel(ChunkArgs a, int64_t groups) {
    __shared__ f4v so[kCcGroups][32];
    __shared__ float sr[kCcGroups], sl[kCcGroups];
    const uint32_t row = blockIdx.x;
    const int d4 = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const float2* state = part_state(a, groups, row);
    const f4v* part = reinterpret_cast<const f4v*>(a.part) + (int64_t)row * a.splits * (kD / 4) + d4;
    const float c2 = score_factor(a.scale);
    bool odd = false;
    float top = -__builtin_huge_valf(), l = 0.f;
    f4v acc{0.f, 0.f, 0.f, 0.f};
    for (int s = sub; s < a.splits; s += kCcGroups) {
        const float2 st = state[s];
        const f4v v = part[s * (kD / 4)];
        if (st.x == -__builtin_huge_valf()) continue;  // saw no key; its outputs may not have been written
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
#pragma unroll
    for (int i = 0; i < kCcGroups; ++i) top = fmaxf(top, sr[i]);
    l = 0.f;
    acc = f4v{0.f, 0.f, 0.f, 0.f};
    odd = false;
#pragma unroll
    for (int i = 0; i < kCcGroups; ++i) odd |= __builtin_signbit(sl[i]);
    if (top > -__builtin_huge_valf())
#pragma unroll
        for (int i = 0; i < kCcGroups; ++i) {
            const float c = rescale(sr[i], top, c2);
            l += c * __builtin_fabsf(sl[i]);
            acc += c * so[i][d4];
        }
    bool real = true;
    if (WINDOW && a.counts) {
        const uint32_t M = (uint32_t)(a.g * a.t);
        real = (int)(row % M % (uint32_t)a.t) < a.counts[row / M / (uint32_t)a.hkv];
    }
    store_row<WINDOW>(a, row, d4, l > 0.f ? 1.f / l : 0.f, acc, odd, real);
}

}  // namespace

// Rows of a block: up to 32 by the kernel of this file (64 rows of one wave would need every
// register of a SIMD), more by tile_attend.hip, whose waves share the keys' tiles.
static int chunk_block_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

static int64_t chunk_steps(const ChunkArgs& a) {
    if (a.window == 0) return (a.n + kCaKeys - 1) / kCaKeys;
    const int64_t near = a.window + a.t - 1, all = a.n + a.t, sinks = a.sink < a.n ? a.sink : a.n;
    return (sinks + kCaKeys - 1) / kCaKeys + ((near < all ? near : all) + kCaKeys - 1) / kCaKeys;
}

// Shares of the keys that `blocks` blocks of `block` rows are cut into at most: about two rounds of
// the blocks that the chip holds at a time (2 a CU).
static int64_t chunk_rounds(int64_t block) { return block <= 32 ? 1024 : 512; }
static int64_t chunk_shares(int64_t block, int64_t blocks) {
    const int64_t splits = (chunk_rounds(block) + blocks - 1) / blocks;
    return splits > kCaMaxShares ? kCaMaxShares : splits;
}

void chunk_plan(ChunkArgs& a) {
    const int64_t groups = (int64_t)a.batch * a.hkv, rows = (int64_t)a.g * a.t;
    const int64_t block = chunk_block_rows(rows), steps = chunk_steps(a);
    int64_t splits = chunk_shares(block, groups * ((rows + block - 1) / block));
    // A share is a multiple of 4 steps, one for every wave.
    int64_t per = (steps + splits - 1) / splits;
    per = (per + kCaWaves - 1) / kCaWaves * kCaWaves;
    if (per < kCaWaves) per = kCaWaves;
    splits = (steps + per - 1) / per;
    a.per = (int32_t)per;
    a.splits = (int32_t)(splits < 1 ? 1 : splits);
}

// Both forms' times in ns, fitted to 165 calls of 1 to 512 tokens, 1 to 128 (sequence, KV head)s
// and windows of 512 to 16384 rows: 1 x 8 x 4 heads, 4096 rows, 16 tokens: 20 us here, 78 in the
// prompt form; 128 tokens 39 and 83; 16 x 8 x 4, 4096 rows, 32 tokens 88 and 125, 64 tokens 144 and
// 130, 128 tokens 235 and 147; 512 rows, 32 tokens 37 and 25.  Over 135 other calls the choice is
// 0.5% behind the faster form on average, more than 5% in 4, 31% at worst (2 x 7 heads, 1024 tokens,
// 4096 rows: 107 us here, 81 in the prompt form).
bool few_tokens(const ChunkArgs& a) {
    if (a.t > kFewTokens) return false;
    const double groups = (double)a.batch * a.hkv, rows = (double)a.g * a.t, all = (double)(a.n + a.t);
    auto tiles = [&](double tokens) {
        const double keys = (double)a.sink + (double)a.window + tokens;
        return (keys < all ? keys : all) / 64;
    };
    const double blocks = groups * a.g * ((a.t + 127) / 128);
    // Two launches and the parts' way through memory; 64 rows of K and V, or the work on them.
    const double few = 12000 + groups * rows + groups * tiles(a.t) * (rows > 92 ? 0.0586 * rows : 5.4);
    // A tile's latency, or the blocks' work once they fill the chip.
    const double prompt = 4000 + tiles(a.t < 128 ? a.t : 128) * (blocks > 325 ? 4.3 * blocks : 1400);
    return few < prompt;
}

static size_t part_bytes(int64_t rows, int64_t splits) { return splits > 1 ? (size_t)rows * splits * (kD + 2) * 4 : 0; }

size_t chunk_part_bytes(const ChunkArgs& a) { return part_bytes((int64_t)a.batch * a.hkv * a.g * a.t, a.splits); }

// Fewer keys, tokens or sequences can take more shares (rounding a share to whole steps leaves fewer
// of more keys), so this is the largest of them all.  For every number of blocks that the rows of a
// (sequence, KV head) make, the most tokens that make it; there, for every number of shares, the
// most sequences that are cut into it.
size_t chunk_part_bound(ChunkArgs a) {
    const int64_t most = a.window > 0 && a.t > kFewTokens ? kFewTokens : a.t, batch = a.batch;
    size_t bytes = 0;
    for (int64_t t = 1; t <= most; t = a.t + 1) {
        const int64_t block = chunk_block_rows(a.g * t), tiles = (a.g * t + block - 1) / block;
        const int64_t full = tiles * block / a.g;
        a.t = (int32_t)(full < most ? full : most);
        const int64_t shares = (chunk_steps(a) + kCaWaves - 1) / kCaWaves, blocks = a.hkv * tiles;
        for (int64_t b = 1; b <= batch; ++b) {
            int64_t splits = chunk_shares(block, b * blocks);
            if (shares < splits) splits = shares;
            if (splits <= 1) break;
            const int64_t same = (chunk_rounds(block) - 1) / (blocks * (splits - 1));
            b = same < batch ? same : batch;
            const size_t need = part_bytes(b * a.hkv * a.g * a.t, splits);
            if (need > bytes) bytes = need;
        }
    }
    return bytes;
}

hipError_t launch_chunk_attend(const ChunkArgs& a, hipStream_t s) {
    const int64_t groups = (int64_t)a.batch * a.hkv;
    const int M = a.g * a.t;
    const int block = chunk_block_rows(M);
    const int row_tiles = (M + block - 1) / block;
    const char* name = a.window > 0 ? "sink_window_attend" : a.rec ? "quant_tree_attend" : "tree_attend";
    hipError_t e;
    if (block > 32) {
        e = launch_tile_attend(a, block, row_tiles, groups, name, s);
    } else {
        const ProfEvents pe = prof_begin(name);
        auto go = [&](auto kernel) {
            hipExtLaunchKernelGGL(kernel, dim3((unsigned)(groups * a.splits * row_tiles)), dim3(64 * kCaWaves), 0, s,
                                  pe.start, pe.stop, 0, a, row_tiles, groups);
        };
        auto rows = [&](auto k16, auto k32) { block == 16 ? go(k16) : go(k32); };
        if (a.window > 0)
            rows(chunk_attend_kernel<16, 16, 16, true>, chunk_attend_kernel<32, 16, 16, true>);
        else if (!a.rec)
            rows(chunk_attend_kernel<16, 16, 16, false>, chunk_attend_kernel<32, 16, 16, false>);
        else if (a.k_bits == 8 && a.v_bits == 8)
            rows(chunk_attend_kernel<16, 8, 8, false>, chunk_attend_kernel<32, 8, 8, false>);
        else if (a.k_bits == 8)
            rows(chunk_attend_kernel<16, 8, 4, false>, chunk_attend_kernel<32, 8, 4, false>);
        else if (a.v_bits == 8)
            rows(chunk_attend_kernel<16, 4, 8, false>, chunk_attend_kernel<32, 4, 8, false>);
        else
            rows(chunk_attend_kernel<16, 4, 4, false>, chunk_attend_kernel<32, 4, 4, false>);
        e = hipGetLastError();
    }
    if (e != hipSuccess || a.splits == 1) return e;
    const ProfEvents pe = prof_begin("chunk_combine");
    const int64_t all = groups * M;
    auto combine = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)all), dim3(32 * kCcGroups), 0, s, pe.start, pe.stop, 0, a, groups);
    };
    a.window > 0 ? combine(chunk_combine_kernel<true>) : combine(chunk_combine_kernel<false>);
    return hipGetLastError();
}

}  // namespace pariskv
