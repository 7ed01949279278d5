// Attention of a few new tokens per sequence where they make more than 32 rows over the same
// keys (chunk_attend.hip has the method and the kernel for fewer).
//
// 4 waves: SETS sets of 32 rows, and 4 / SETS waves a set that take 32 keys each of a tile of
// keys.  The tile is read from HBM once and lies in LDS as float16 for all sets: waves that
// fetched the same rows at the same time for themselves had them fetched from HBM twice, for
// misses on one cache line are not joined while it is on its way (16 drafts x 4 heads, 8 x 8 x
// 128K float16 rows: 1317 us so, 920 with the sets in blocks of their own, 757 here, 93% of the
// rate of a plain read).  Records are taken apart once for all rows.  Two tiles are in flight in
// registers while one is computed on, and two blocks share a CU: one computes while the other
// waits at its barrier.
// 128 rows: 31 drafts x 4 heads over the same rows take 1000 to 1200 us from launch to launch and card
// to card, always 1.6 million cycles, of which the matrix units are busy 48% and LDS 32% (a plain
// float16 product: 70% and 35%); the rest is the vector instructions between the two products and
// waiting.  The clock follows the power drawn, 1.4 to 1.9 GHz; with all values 0 it is 2.1 to 2.3,
// and the time 745 to 810 us.

#include <hip/hip_fp16.h>

#include "chunk_attend_device.hpp"

namespace pariskv {

namespace {

constexpr int kTaWaves = 4;
constexpr int kTaThreads = 64 * kTaWaves;

// What a thread holds of a tile on its way: 8 dims of K and of V of N keys.
template <int N, int KB, int VB>
struct TileRegs {
    u2v k[N], v[N];
    uint32_t ks[N], vs[N];
};
template <int N>
struct TileRegs<N, 16, 16> {
    u4v k[N], v[N];
};

template <int SETS, int KB, int VB, bool WINDOW>
__global__ __launch_bounds__(kTaThreads, 2) void tile_attend_kernel(ChunkArgs a, int row_tiles, int64_t groups) {
    constexpr int R = 32;  // rows of a wave
    using Rows = ChunkRows<R>;
    constexpr bool kQuant = KB < 16;
    constexpr int kRecord = kQuant ? quant_record_bytes(KB, VB) : 0;
    constexpr int kParts = kTaWaves / SETS;      // waves that share a set's keys
    constexpr int kSub = SETS == 4 ? 2 : 1;      // 32-key steps of a wave in a tile
    constexpr int kTile = kCaKeys * kParts * kSub;  // keys of a tile
    constexpr int kRowLoads = kTile * 16 / kTaThreads;  // 16-byte pieces of K (of V) a thread holds
    constexpr int kTileBytes = kTile * kD * 2;
    constexpr int kUse = 4 * kTileBytes, kState = ca_state_bytes(R);  // two buffers of K and V
    constexpr int kLds = kUse > kTaWaves * kState ? kUse : kTaWaves * kState;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kLds];

    const ChunkPlace pl = chunk_place(a, row_tiles, groups);
    const int64_t grp = pl.grp;
    const int seq = pl.seq;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = wave % kParts, set = wave / kParts;
    const int M = a.g * a.t, row0 = (pl.tile * SETS + set) * R;
    const KeySpan span = key_span(a, seq, 0, a.t);

    // Tiles: the sinks', the cached stretch's; this share's part of them, and the drafts behind
    // the last share's.
    const int sink_tiles = (span.sink_end + kTile - 1) / kTile;
    const int tiles = sink_tiles + (span.hi - span.lo + kTile - 1) / kTile;
    const int per = a.per * kCaKeys / kTile;
    const bool closing = pl.split == a.splits - 1;  // takes what is left, and the drafts
    const int first = min(pl.split * per, tiles), last = closing ? tiles : min(first + per, tiles);
    const int end = last + ((!WINDOW && closing) ? (a.t + kTile - 1) / kTile : 0);
    if (first >= end && a.splits > 1) return leave_idle(a, pl, groups, pl.tile * SETS * R, SETS * R);

    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    const int row = min(row0 + Rows::row(lane), M - 1), tok = row % a.t;  // this lane's
    const u4v* qr = reinterpret_cast<const u4v*>(static_cast<const __half*>(a.q) + (grp * M + row) * kD);
    h8v qf[Rows::kSteps];
#pragma unroll
    for (int c = 0; c < Rows::kSteps; ++c) qf[c] = query_part(qr[Rows::dim<false>(c, lane) / 8], flip);
    Rows rows(score_factor(a.scale), lane);

    // Of a tile: cache row (or draft) of its first key, and how many of its keys there are.
    auto tile_base = [&](int t) {
        if (!WINDOW && t >= last) return (t - last) * kTile;
        return WINDOW && t < sink_tiles ? t * kTile : span.lo + (t - sink_tiles) * kTile;
    };
    auto tile_keys = [&](int t) {
        const int stop = !WINDOW && t >= last ? a.t : WINDOW && t < sink_tiles ? span.sink_end : span.hi;
        return stop - tile_base(t);
    };
    unsigned char* kt = lds;
    unsigned char* vt = lds + 2 * kTileBytes;
    const int lrow = tid >> 4, lchunk = tid & 15;
    constexpr int kStepRows = kTaThreads / 16;  // rows that the block's 16-byte pieces cover at once
    auto put = [&](int buf, int key, h8v k, h8v v) {
        *reinterpret_cast<h8v*>(kt + buf * kTileBytes + key * 256 + ((lchunk ^ (key & 15)) << 4)) = k;
        put_v(vt + buf * kTileBytes, key, lchunk, v);
    };

    // What lies behind the last key is not read: it is repeated.
    auto load = [&](int t, TileRegs<kRowLoads, KB, VB>& regs) {
        const int most = tile_keys(t) - 1;
        const bool drafts = !WINDOW && t >= last;
        if constexpr (kQuant) {
            if (drafts) return;
            const uint8_t* p = a.rec + (grp * a.capacity + tile_base(t)) * kRecord;
#pragma unroll
            for (int i = 0; i < kRowLoads; ++i) {
                const int at = min(kStepRows * i + lrow, most) * kRecord;
                regs.k[i] = quant_load8<KB>(p + (at + lchunk * KB));
                regs.v[i] = quant_load8<VB>(p + (at + quant_code_bytes(KB) + lchunk * VB));
                regs.ks[i] = p[at + quant_code_bytes(KB) + quant_code_bytes(VB) + (lchunk >> 2)];
                regs.vs[i] = p[at + quant_code_bytes(KB) + quant_code_bytes(VB) + 4 + (lchunk >> 2)];
            }
        } else {
            const int64_t at = (drafts ? grp * a.t : grp * a.capacity) + tile_base(t);
            const u4v* K = static_cast<const u4v*>(drafts ? a.Kt : a.K) + at * 16;
            const u4v* V = static_cast<const u4v*>(drafts ? a.Vt : a.V) + at * 16;
#pragma unroll
            for (int i = 0; i < kRowLoads; ++i) {
                const int from = min(kStepRows * i + lrow, most) * 16 + lchunk;
                regs.k[i] = K[from];
                regs.v[i] = V[from];
            }
        }
    };
    uint32_t odd = 0u;  // kOddBits: some V there had values that are not finite
    // Whether some token does not see some key of tile t.
    auto partly = [&](int t) {
        const int base = tile_base(t), end = base + kTile - 1;
        if (!WINDOW) return t >= last;
        return tile_keys(t) < kTile || end > span.start ||
               (end >= (int)a.sink && base <= span.start + span.tokens - 1 - (int)a.window);
    };
    // Puts tile t, loaded into regs, into buffer buf as float16.
    auto place = [&](int t, int buf, const TileRegs<kRowLoads, KB, VB>& regs) {
        const bool drafts = !WINDOW && t >= last;
        if (kQuant && !drafts) {
            if constexpr (kQuant)
#pragma unroll
                for (int i = 0; i < kRowLoads; ++i)
                    put(buf, kStepRows * i + lrow, quant_decode8<KB>(regs.k[i][0], regs.k[i][1], quant_scale_value(regs.ks[i])),
                        quant_decode8<VB>(regs.v[i][0], regs.v[i][1], quant_scale_value(regs.vs[i])));
            return;
        }
        const int first_draft = tile_base(t), most = tile_keys(t) - 1;
        const bool some = partly(t);
#pragma unroll
        for (int i = 0; i < kRowLoads; ++i) {
            const int key = kStepRows * i + lrow;
            u4v k, v;
            if constexpr (kQuant) {  // drafts: straight from memory, once a call
                const int64_t from = (grp * a.t + first_draft + min(key, most)) * 16 + lchunk;
                k = static_cast<const u4v*>(a.Kt)[from];
                v = static_cast<const u4v*>(a.Vt)[from];
            } else {
                k = regs.k[i];
                v = regs.v[i];
            }
            if (some) {
                note_odd(v, odd);
                v = finite_part(v);
            }
            put(buf, key, as_h8(k), as_h8(v));
        }
    };

    auto compute = [&](int t, int buf) {
        if (row0 >= M) return;
#pragma unroll 1
        for (int sub = 0; sub < kSub; ++sub) {
            const int at = (part * kSub + sub) * kCaKeys;
            const int base = tile_base(t) + at, valid = tile_keys(t) - at;
            if (valid <= 0) return;
            const int from = buf * kTileBytes + at * 256, key = Rows::key(0, lane);
            rows.scores(qf, [&](int, int c) {
                return *reinterpret_cast<const h8v*>(kt + from + key * 256 +
                                                     (((Rows::dim<false>(c, lane) / 8) ^ (key & 15)) << 4));
            });
            uint32_t w = bits_to(valid - 1);
            if constexpr (WINDOW) w &= window_bits(span.start + tok, base, (int)a.sink, (int)a.window);
            else if (t >= last) w = draft_bits(a, seq, tok, base, valid);
            __builtin_amdgcn_s_setprio(1);  // ahead of another wave's S^T: 2 to 5%
            rows.accumulate(w, vt + from, lane);
            __builtin_amdgcn_s_setprio(0);
        }
    };

    TileRegs<kRowLoads, KB, VB> regs[2];
    if (first < end) load(first, regs[0]);
    if (first + 1 < end) load(first + 1, regs[1]);
    if (first < end) place(first, 0, regs[0]);
    if (first + 2 < end) load(first + 2, regs[0]);
    // Tile t lies in buffer b; r holds tile t + 1 and takes tile t + 3.
    auto turn = [&](int t, int b, TileRegs<kRowLoads, KB, VB>& r) {
        __syncthreads();
        compute(t, b);
        if (t + 1 < end) place(t + 1, b ^ 1, r);
        if (t + 3 < end) load(t + 3, r);
    };
    for (int t = first; t < end; t += 2) {
        turn(t, 0, regs[1]);
        if (t + 1 < end) turn(t + 1, 1, regs[0]);
    }

    const bool any_odd = __syncthreads_or((odd & kOddBits) != 0u);
    rows.leave(lds + wave * kState, lane, any_odd);
    __syncthreads();
    join_waves<R, kParts, WINDOW>(a, pl, groups, row0, span.tokens, lds + set * kParts * kState, kState,
                                   (tid >> 5) % (2 * kParts), 2 * kParts);
}

}  // namespace

hipError_t launch_tile_attend(const ChunkArgs& a, int block, int row_tiles, int64_t groups, const char* name,
                              hipStream_t s) {
    const ProfEvents pe = prof_begin(name);
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)(groups * a.splits * row_tiles)), dim3(kTaThreads), 0, s, pe.start,
                              pe.stop, 0, a, row_tiles, groups);
    };
    auto rows = [&](auto k64, auto k128) { block == 64 ? go(k64) : go(k128); };
    if (a.window > 0)
        rows(tile_attend_kernel<2, 16, 16, true>, tile_attend_kernel<4, 16, 16, true>);
    else if (!a.rec)
        rows(tile_attend_kernel<2, 16, 16, false>, tile_attend_kernel<4, 16, 16, false>);
    else if (a.k_bits == 8 && a.v_bits == 8)
        rows(tile_attend_kernel<2, 8, 8, false>, tile_attend_kernel<4, 8, 8, false>);
    else if (a.k_bits == 8)
        rows(tile_attend_kernel<2, 8, 4, false>, tile_attend_kernel<4, 8, 4, false>);
    else if (a.v_bits == 8)
        rows(tile_attend_kernel<2, 4, 8, false>, tile_attend_kernel<4, 4, 8, false>);
    else
        rows(tile_attend_kernel<2, 4, 4, false>, tile_attend_kernel<4, 4, 4, false>);
    return hipGetLastError();
}

}  // namespace pariskv
