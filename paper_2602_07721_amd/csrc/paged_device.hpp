// Device code that both forms of the attention over pages share.
#pragma once

#include <type_traits>

#include "chunk_attend_device.hpp"
#include "pages.hpp"

namespace pariskv {

// One sequence's new tokens [begin, begin + count) of q and its cached rows, as the call's arrays say
// and its sizes allow.
struct PagedSeq {
    int begin, count, len;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int b) {
    PagedSeq s;
    s.begin = min(max(a.offsets[b], 0), a.t);
    const int end = min(max(a.offsets[b + 1], s.begin), a.t);
    s.count = min(end - s.begin, a.most);
    if (a.counts) s.count = min(s.count, max(a.counts[b], 0));
    const int64_t room = min(a.width * (int64_t)a.page.d, kMaxKvRows);
    s.len = (int)min((int64_t)max(a.lens[b], 0), room);
    return s;
}

// Where a key's row lies in K and V: its page's entry, and whether there is such a page.
__device__ __forceinline__ int page_entry(const PagedArgs& a, int b, int row) {
    return a.table[b * a.width + a.page((uint32_t)row)];
}
__device__ __forceinline__ int page_row(const PagedArgs& a, int entry, int head, int row) {
    const int size = (int)a.page.d;
    return (entry * a.hkv + head) * size + (row - (int)a.page((uint32_t)row) * size);
}

// What is done to scores before their softmax.  Caps above kWaveCap have forms of their own.
enum { kPlainScores = 0, kCappedScores = 1, kBiasedScores = 2, kLargeCap = 4 };
constexpr float kWaveCap = 64.f;
inline int score_shape(const PagedArgs& a) {
    return (a.cap > 0.f ? kCappedScores : 0) | (a.slopes ? kBiasedScores : 0) | (a.cap > kWaveCap ? kLargeCap : 0);
}
// f(std::integral_constant of the shape)
template <class F>
void by_shape(int shape, F&& f) {
    switch (shape) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 5: return f(std::integral_constant<int, 5>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, 0>());
    }
}

// With a shape, scores are in powers of two: s' = cap log2(e) tanh(scale s / cap), or the plain
// product, plus slope log2(e) times the distance.
template <int SHAPE>
struct ScoreShape {
    float unit, cap, slope;  // s times unit is u (capped) or the score in powers of two
    __device__ __forceinline__ ScoreShape(const PagedArgs& a, int head) {
        constexpr float kLog2e = 1.4426950408889634f;
        const float scale = fabsf(a.scale);
        // Finite, as score_factor's.
        unit = fminf(SHAPE & kCappedScores ? scale / a.cap : scale * kLog2e, kMostFactor);
        cap = SHAPE & kCappedScores ? a.cap * kLog2e : 0.f;
        slope = 0.f;
        if constexpr ((SHAPE & kBiasedScores) != 0) {
            const float x = a.slopes[head];
            slope = __builtin_fabsf(x) <= kMostFactor ? fminf(fmaxf(x * kLog2e, -kMostFactor), kMostFactor) : x;
        }
    }
    // Of a lane's N scores, which the functions give for their numbers: the score, and how far its key is
    // behind the token (negative).
    //
    // Where all of a wave's |u| are below 0.2, a series, within 2^-22 of itself, in five instructions of
    // the vector unit; else tanh(u) = 1 - 2 / (2^(2 log2(e) u) + 1), within 2^-21 of 1, with two that take
    // four times as long.  8192 tokens, 32 heads, cap 30: 716 to 760 us so, 867 with the second for every score.
    // So a wave's other scores, those of keys that a row does not see among them, decide on 2^-21 of the cap:
    // up to a cap of 64 at most 2^-15 of a weight.  Above it each score takes its own of the two (917 us where 716 are taken so).
    template <int N, class Score, class Distance>
    __device__ __forceinline__ void operator()(Score&& score, Distance&& distance) const {
        if constexpr ((SHAPE & kCappedScores) != 0) {
            auto near = [&](float u) {
                const float u2 = u * u;
                float x = __builtin_fmaf(u2, cap * -0.053968254f, cap * 0.13333334f);
                x = __builtin_fmaf(u2, x, cap * -0.33333334f);
                return u * __builtin_fmaf(u2, x, cap);
            };
            auto far = [&](float u) {
                const float e = __builtin_amdgcn_exp2f(u * 2.8853900817779268f);
                return __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(e + 1.f), cap);
            };
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                score(i) *= unit;
                top = fmaxf(top, __builtin_fabsf(score(i)));
            }
            if (__all(top < 0.2f)) {
#pragma unroll
                for (int i = 0; i < N; ++i) score(i) = near(score(i));
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float u = score(i);
                    score(i) = (SHAPE & kLargeCap) != 0 && __builtin_fabsf(u) < 0.2f ? near(u) : far(u);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) score(i) *= unit;
        }
        if constexpr ((SHAPE & kBiasedScores) != 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) score(i) = __builtin_fmaf(slope, distance(i), score(i));
        }
    }
};

// Sum over the lanes before this one and over all, of values of 0 to 2^57: their bits in three parts
// whose sums fit 32, which are moved between lanes in registers.
__device__ __forceinline__ int64_t wave_sum_before(int64_t v, int64_t* all) {
    const uint32_t low = wave_incl_sum((uint32_t)v & 0xffffu);
    const uint32_t mid = wave_incl_sum((uint32_t)(v >> 16) & 0xffffu);
    const uint32_t high = wave_incl_sum((uint32_t)(v >> 32));
    const int64_t sum = ((int64_t)high << 32) + ((int64_t)mid << 16) + low;
    *all = ((int64_t)__builtin_amdgcn_readlane((int)high, 63) << 32) +
           ((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)mid, 63) << 16) +
           (uint32_t)__builtin_amdgcn_readlane((int)low, 63);
    return sum - v;
}

constexpr int kPgThreads = 256, kPgWaves = kPgThreads / 64;
constexpr int kPgBlocks = 512;  // that the chip holds, 2 a CU

__device__ __forceinline__ int64_t read_lane(int64_t x, int lane) {
    return ((int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}
__device__ __forceinline__ PagedSeq read_lane(const PagedSeq& s, int lane) {
    return PagedSeq{__builtin_amdgcn_readlane(s.begin, lane), __builtin_amdgcn_readlane(s.count, lane),
                    __builtin_amdgcn_readlane(s.len, lane)};
}

// The first sequence from b on that has work, and what it is; a.batch if there is none.  64 are looked up at a
// time, since a server's batch may be mostly places without a sequence (16 of 4000 rows in 2048 places: 68 us,
// 88 one by one).
template <class Has>
__device__ __forceinline__ int next_seq(const PagedArgs& a, int b, PagedSeq& seq, Has&& has) {
    for (; b < a.batch; b += 64) {
        const int at = b + (int)(threadIdx.x & 63);
        const PagedSeq s = paged_seq(a, min(at, a.batch - 1));
        const uint64_t who = __ballot(at < a.batch && has(s));
        if (who != 0) {
            const int lane = (int)__builtin_ctzll(who);
            seq = read_lane(s, lane);
            return b + lane;
        }
    }
    return a.batch;
}

// Work is planned by every wave for itself, without barriers: a lane has some neighbouring sequences.
struct LaneSeqs {
    int each, b0, b1;
    __device__ __forceinline__ explicit LaneSeqs(const PagedArgs& a) {
        each = (a.batch + 63) / 64;
        b0 = min((int)(threadIdx.x & 63) * each, a.batch);
        b1 = min(b0 + each, a.batch);
    }
    // f(b, sequence b) for each of them; the loads of 8 are on their way at a time.
    template <class F>
    __device__ __forceinline__ void each_of(const PagedArgs& a, F&& f) const {
        if (each == 1) {
            if (b0 < b1) f(b0, paged_seq(a, b0));
            return;
        }
        for (int b = b0; b < b1; b += 8) {
            PagedSeq s[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] = paged_seq(a, min(b + u, b1 - 1));
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (b + u < b1) f(b + u, s[u]);
        }
    }
};

// Which of a line's stretches, a multiple of 8, a block takes: consecutive blocks go to the 8 XCDs in turn,
// and each XCD takes one length of the line, whose neighbours read the same keys.
__device__ __forceinline__ int line_block(uint32_t block, int blocks) { return (int)(block % 8 * (blocks / 8) + block / 8); }

// The quotient of numbers that mostly fit 32 bits.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t d) {
    return ((x | d) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)d) : x / d;
}

// ---- at most 16 or 32 rows: a block's waves take 32 keys each in turn

constexpr int kPfKeys = kPgWaves * kCaKeys;  // keys of a part, one step of every wave

// Parts of a sequence's keys for one KV head; one also where there are tokens but no keys.
__device__ __forceinline__ int few_parts(const PagedSeq& s) {
    return s.count > 0 ? max(1, (s.len + kPfKeys - 1) / kPfKeys) : 0;
}

// The line of all parts, sequence by sequence and head by head, cut into stretches, one a block: the
// first `more` have one part more than the others.  No block of the first `blocks` is without work.
struct FewLine {
    int64_t all, blocks, each, more;
    __device__ __forceinline__ FewLine(const PagedArgs& a, int64_t parts) {
        all = parts * a.hkv;
        blocks = min(all, (int64_t)kPgBlocks);
        each = blocks > 0 ? quotient(all, blocks) : 0;
        more = all - each * blocks;
    }
    __device__ __forceinline__ int64_t begin(int64_t block) const { return block * each + min(block, more); }
    __device__ __forceinline__ int64_t block_of(int64_t x) const {
        const int64_t y = x - more * (each + 1);
        return y < 0 ? quotient(x, each + 1) : more + quotient(y, each);
    }
};

// Parts (64 KB of K and V) from which on all that is read cannot stay in the caches until it is read
// again: it is then read past them.  A step of 4.3 GB takes 637 us so and 715 through the caches, one of
// 95 MB, read before, 34 and 30.5.  Not so the keys of 32 rows, of which a load takes 32 bytes of 32 lines:
// 8 tokens of each of 8 sequences of 131072 rows take 652 us with keys through the caches, 805 past them.
constexpr int64_t kStreamParts = (192 << 20) / (kPfKeys * 4 * kD);

// What a block leaves for the joining kernel: the head that its stretch began and did not end (b < 0:
// none), and the block that ends it.
struct FewRecord {
    int b, head, last;
};
// The workspace of sequences walked so: records; then outputs and states of the heads that blocks
// share, two slots of `rows` rows a block: a head begun in another block in slot 2 i, one that is not
// ended in slot 2 i + 1.
constexpr size_t kFewRecordBytes = (kPgBlocks * sizeof(FewRecord) + 255) / 256 * 256;
struct FewSpace {
    FewRecord* record;  // [kPgBlocks]
    float* part;        // [2 kPgBlocks][rows][D]
    float2* state;      // [2 kPgBlocks][rows]
    char* end;
    __device__ __forceinline__ FewSpace(const PagedArgs& a, int rows) {
        char* p = static_cast<char*>(a.workspace);
        record = reinterpret_cast<FewRecord*>(p);
        part = reinterpret_cast<float*>(p + kFewRecordBytes);
        state = reinterpret_cast<float2*>(part + (int64_t)2 * kPgBlocks * rows * kD);
        end = reinterpret_cast<char*>(state + (int64_t)2 * kPgBlocks * rows);
    }
    static size_t bytes(int rows) { return kFewRecordBytes + (size_t)2 * kPgBlocks * rows * (kD + 2) * 4; }
};

constexpr int few_wave_lds(int rows) {
    return kCaKeys * kD * 2 > ca_state_bytes(rows) ? kCaKeys * kD * 2 : ca_state_bytes(rows);
}

// What the sum and the outputs of a state at r are multiplied by when they are joined at `to` >= r.  One that saw
// no key that counts has a sum of 0, and outputs of 0 or values that are not finite: they stay what they are.
__device__ __forceinline__ float state_factor(float r, float to, float c2) {
    return r == -__builtin_huge_valf() ? 1.f : rescale(r, to, c2);
}

// What a block takes of a head at a time: parts [part0, part1) of the keys of its M = count g rows.
struct FewSegment {
    int b, head, part0, part1, parts;
    PagedSeq seq;
    __device__ __forceinline__ int first() const { return part0 * kPgWaves; }  // steps of 32 keys
    __device__ __forceinline__ int last() const {
        return min(part1 * kPgWaves, (seq.len + kCaKeys - 1) / kCaKeys);
    }
};

// Walks segments from g, at place x of the line, up to `end`.  lds(w): few_wave_lds(R) bytes of wave w,
// 16-byte aligned.  A head's outputs where its parts are all here, else states: row r's outputs, its
// reference and sum.  A wave's next step, of this segment or of the next, is on its way while one is
// computed on and while segments end.
//
// Values of V that are not finite are taken out of a step that not every row sees whole.  The rows that
// see them get them from memory when the segment ends: of the steps from the first to the last that held
// some (131067 rows of one head, 4 rows: 29.4 us; with an infinity in the last 30.6, in the last 27 39.5).
template <int R, int SHAPE, bool STREAM, class Parts, class Lds>
__device__ __forceinline__ FewRecord few_walk(const PagedArgs& a, const FewSpace& ws, const FewLine& line, int id,
                                              FewSegment g, int64_t x, int64_t end, Parts&& parts_of, Lds&& lds) {
    using Rows = ChunkRows<R>;
    constexpr int kHalves = Rows::kHalves, kSteps = Rows::kSteps;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned char* vt = lds(wave);
    const int vrow = lane >> 4, vchunk = lane & 15;  // of a load or a store of 4 rows of V
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;

    // A step's pages, one key a lane (and lane + 32): entries of the table, then rows of K and V and
    // which of them there are.  Keys behind the last repeat it, those without a page the first that
    // has one (there or not, row 0 of the pages is memory).
    auto key_row = [&](int st, int len) { return min(st * kCaKeys + (lane & 31), len - 1); };
    auto entry_of = [&](int b, int st, int len) { return page_entry(a, b, key_row(st, len)); };
    auto read = [](const u4v* p) { return STREAM ? __builtin_nontemporal_load(p) : *p; };
    u4v kreg[8], vreg[8];
    uint32_t there = 0;  // the step's keys that have pages
    int entry = 0;       // of this lane's key of the step behind
    auto fetch = [&](int b, int head, int len, int st, int last, int e) __attribute__((always_inline)) {
        const bool good = (uint32_t)e < (uint32_t)a.n_pages;
        there = (uint32_t)__ballot(good);
        int at = good ? page_row(a, e, head, key_row(st, len)) : 0;
        if (__builtin_expect(there != ~0u, 0)) {
            const int other = there ? __builtin_amdgcn_readlane(at, __builtin_ctz(there)) : 0;
            at = good ? at : other;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = __builtin_amdgcn_ds_bpermute((4 * i + vrow) << 2, at);
            vreg[i] = read(reinterpret_cast<const u4v*>(static_cast<const _Float16*>(a.V) + (int64_t)r * kD) + vchunk);
        }
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const int r = __builtin_amdgcn_ds_bpermute(Rows::key(h, lane) << 2, at);
            const _Float16* k = static_cast<const _Float16*>(a.K) + (int64_t)r * kD;
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                const u4v* part = reinterpret_cast<const u4v*>(k + Rows::template dim<false>(c, lane));
                kreg[h * kSteps + c] = R == 32 ? *part : read(part);
            }
        }
        if (st + kPgWaves < last) entry = entry_of(b, st + kPgWaves, len);
    };
    h8v qf[kSteps];
    auto load_q = [&](const FewSegment& s) {
        const int row = min(Rows::row(lane), s.seq.count * a.g - 1);
        const _Float16* qr = static_cast<const _Float16*>(a.q) + (int64_t)(s.seq.begin + row / a.g) * a.q_stride +
                             (s.head * a.g + row % a.g) * kD;
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
            qf[c] = query_part(*reinterpret_cast<const u4v*>(qr + Rows::template dim<false>(c, lane)), flip);
    };

    FewRecord record{-1, 0, 0};
    if (g.first() + wave < g.last())
        fetch(g.b, g.head, g.seq.len, g.first() + wave, g.last(), entry_of(g.b, g.first() + wave, g.seq.len));
    load_q(g);
    for (;;) {
        // The segment behind this one, and this wave's first step of it.
        const int64_t next_x = x + g.part1 - g.part0;
        bool more = next_x < end;
        FewSegment n = g;
        int next_st = 0, next_last = 0, next_entry = 0;
        if (more) {
            if (++n.head == a.hkv) {
                n.head = 0;
                n.b = next_seq(a, n.b + 1, n.seq, [&](const PagedSeq& s) { return parts_of(s) > 0; });
                n.parts = parts_of(n.seq);
                more = n.b < a.batch;  // with lengths that stay as they are
            }
            n.part0 = 0;
            n.part1 = (int)min((int64_t)n.parts, end - next_x);
        }
        if (more) {
            next_st = wave;
            next_last = n.last();
            if (next_st < next_last) next_entry = entry_of(n.b, next_st, n.seq.len);
        }

        const int M = g.seq.count * a.g, len = g.seq.len, last = g.last();
        const int row = min(Rows::row(lane), M - 1), p = len - g.seq.count + row / a.g;
        const ScoreShape<SHAPE> shape(a, g.head * a.g + row % a.g);
        Rows rows(SHAPE ? 1.f : score_factor(a.scale), lane);
        int odd_first = 0, odd_last = -1;  // the steps whose V had values that are not finite taken out
        int st = g.first() + wave;
        const bool idle = st >= last;  // no step of this segment
        for (; st < last; st += kPgWaves) {
            const uint32_t w = bits_to(min(p, len - 1) - st * kCaKeys) & there;
            wave_lds_order();  // the step before has read its V
#pragma unroll
            for (int i = 0; i < 8; ++i) put_v(vt, 4 * i + vrow, vchunk, as_h8(vreg[i]));
            if (__builtin_expect(!__all(w == ~0u), 0)) {
                uint32_t m = 0u;
                wave_lds_order();
#pragma unroll 1
                for (int i = 0; i < 8; ++i) note_odd(reinterpret_cast<const u4v*>(vt)[64 * i + lane], m);
                if (__any(m & kOddBits)) {
                    if (odd_last < 0) odd_first = st;
                    odd_last = st;
                    clean_v(vt, lane);
                }
            }
            wave_lds_order();
            rows.scores(qf, [&](int h, int c) { return as_h8(kreg[h * kSteps + c]); });
            const bool here = st + kPgWaves < last;
            if (here || next_st < next_last)
                fetch(here ? g.b : n.b, here ? g.head : n.head, here ? len : n.seq.len, here ? st + kPgWaves : next_st,
                      here ? last : next_last, here ? entry : next_entry);
            if constexpr (SHAPE != kPlainScores) {
                const float from = (float)(st * kCaKeys - p);
                if constexpr (R == 16)
                    shape.template operator()<8>([&](int i) -> float& { return reinterpret_cast<float*>(rows.s)[i]; },
                                                 [&](int i) { return from + (float)(16 * (i / 4) + 4 * rows.lg + i % 4); });
                else
                    shape.template operator()<16>([&](int i) -> float& { return reinterpret_cast<float*>(&rows.s)[i]; },
                                                  [&](int i) { return from + (float)(8 * (i / 4) + 4 * rows.half + i % 4); });
            }
            rows.accumulate(w, vt, lane);
        }
        if (idle && next_st < next_last) fetch(n.b, n.head, n.seq.len, next_st, next_last, next_entry);
        if (more) load_q(n);

#pragma unroll 1
        for (int odd = odd_first; odd <= odd_last; odd += kPgWaves) {
            const int key = key_row(odd, len), e = page_entry(a, g.b, key);
            const bool good = (uint32_t)e < (uint32_t)a.n_pages;
            const int at = good ? page_row(a, e, g.head, key) : 0;
            const uint32_t w = bits_to(min(p, len - 1) - odd * kCaKeys) & (uint32_t)__ballot(good);
            if (__all(w == ~0u)) continue;  // the products had them
            uint32_t keys = 0;  // with such values
#pragma unroll 4
            for (int i = 0; i < 8; ++i) {
                const int r = __builtin_amdgcn_ds_bpermute((4 * i + vrow) << 2, at);
                uint32_t m = 0u;
                note_odd(*(reinterpret_cast<const u4v*>(static_cast<const _Float16*>(a.V) + (int64_t)r * kD) + vchunk), m);
                const uint64_t who = __ballot(m & kOddBits);
#pragma unroll
                for (int j = 0; j < 4; ++j) keys |= (who >> (16 * j) & 0xffff) != 0 ? 1u << (4 * i + j) : 0u;
            }
#pragma unroll 1
            for (; keys != 0; keys &= keys - 1) {
                const int k = __builtin_ctz(keys);
                const h4v* v = static_cast<const h4v*>(a.V) + (int64_t)__builtin_amdgcn_readlane(at, k) * (kD / 4);
                if (w >> k & 1) rows.add_odd_values(v);
            }
        }
        wave_lds_order();
        rows.leave(vt, lane, false);
        __syncthreads();
        // Joins the waves' states, 32 lanes a row, 4 dims a lane.
        const bool whole = g.part0 == 0 && g.part1 == g.parts;
        const int64_t slot = 2 * id + (g.part0 == 0 ? 1 : 0);
        if (g.part0 == 0 && !whole) record = FewRecord{g.b, g.head, (int)line.block_of(x + g.parts - 1)};
        const float c2 = rows.c2;
        const int d4 = tid & 31;
        for (int r = tid >> 5; r < M; r += kPgThreads / 32) {
            float top = -__builtin_huge_valf(), l = 0.f;
            f4v acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kPgWaves; ++w) top = fmaxf(top, reinterpret_cast<const float*>(lds(w))[R * kCaRow + r]);
#pragma unroll
            for (int w = 0; w < kPgWaves; ++w) {
                const float* of = reinterpret_cast<const float*>(lds(w));
                const float c = state_factor(of[R * kCaRow + r], top, c2);
                l += c * of[R * (kCaRow + 1) + r];
                acc += c * *reinterpret_cast<const f4v*>(of + r * kCaRow + 4 * d4);
            }
            if (whole) {
                const int tok = r / a.g;
                acc *= l > 0.f ? 1.f / l : l;
                static_cast<h4v*>(a.out)[((int64_t)(g.seq.begin + tok) * a.hkv * a.g + g.head * a.g + r % a.g) * (kD / 4) + d4] =
                    h4v{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
            } else {
                reinterpret_cast<f4v*>(ws.part)[(slot * R + r) * (kD / 4) + d4] = acc;
                if (d4 == 0) ws.state[slot * R + r] = float2{top, l};
            }
        }
        if (!more) return record;
        __syncthreads();  // the states are read
        g = n;
        x = next_x;
    }
}

// The stretch of block id over the sequences that `pick` takes.
template <int R, int SHAPE, class Pick, class Lds>
__device__ __forceinline__ void few_stretch(const PagedArgs& a, int id, Pick&& pick, Lds&& lds) {
    const FewSpace ws(a, R);
    auto parts_of = [&](const PagedSeq& s) { return pick(s) ? few_parts(s) : 0; };
    const LaneSeqs mine(a);
    PagedSeq seq{};
    int64_t sum = 0, all;
    mine.each_of(a, [&](int b, const PagedSeq& s) {
        seq = s;
        sum += parts_of(s);
    });
    const int64_t before = wave_sum_before(sum, &all);
    const FewLine line(a, all);
    FewRecord record{-1, 0, 0};
    if (id < line.blocks) {
        const int64_t x = line.begin(id), end = line.begin(id + 1);
        const bool own = before * a.hkv <= x && x < (before + sum) * a.hkv;
        const uint64_t who = __ballot(own);
        if (who != 0) {  // else lengths have changed
            const int owner = (int)__builtin_ctzll(who);
            int64_t at = before, found_at = before;
            int found = mine.b0;
            if (mine.each > 1 && own)
                mine.each_of(a, [&](int b, const PagedSeq& s) {
                    const int n = parts_of(s);
                    if (at * a.hkv <= x && n > 0) {  // the last of these
                        found = b;
                        found_at = at;
                        seq = s;
                    }
                    at += n;
                });
            FewSegment g;
            g.seq = read_lane(seq, owner);
            g.b = __builtin_amdgcn_readlane(found, owner);
            g.parts = parts_of(g.seq);
            if (g.parts > 0) {  // as above
                const int64_t skip = x - read_lane(found_at, owner) * a.hkv;
                g.head = min(__builtin_amdgcn_readfirstlane((int)quotient(skip, g.parts)), a.hkv - 1);
                g.part0 = __builtin_amdgcn_readfirstlane((int)(skip - (int64_t)g.head * g.parts));
                g.part1 = (int)min((int64_t)g.parts, g.part0 + (end - x));
                auto walk = [&](auto stream) __attribute__((always_inline)) {
                    return few_walk<R, SHAPE, decltype(stream)::value>(a, ws, line, id, g, x, end, parts_of, lds);
                };
                record = line.all > kStreamParts ? walk(std::true_type()) : walk(std::false_type());
            }
        }
    }
    if (threadIdx.x == 0) ws.record[id] = record;
}

// Joins the states of row r of the head that block id began and did not end: 8 groups of 32 lanes take
// every eighth block, 4 dims a lane, the states of kPjAhead blocks on their way at a time.
constexpr int kPjGroups = 8, kPjAhead = 8;
__device__ __forceinline__ void few_join(const PagedArgs& a, int rows, float c2, int id, int r) {
    __shared__ f4v so[kPjGroups][32];
    __shared__ float sr[kPjGroups], sl[kPjGroups];
    const FewSpace ws(a, rows);
    const FewRecord rec = ws.record[id];
    if (rec.b < 0) return;
    const int b = rec.b, head = rec.head;
    const PagedSeq seq = paged_seq(a, b);
    if (r >= seq.count * a.g) return;
    const int d4 = threadIdx.x & 31, sub = threadIdx.x >> 5;
    float top = -__builtin_huge_valf(), l = 0.f;
    f4v acc{0.f, 0.f, 0.f, 0.f};
    for (int i0 = id + sub; i0 <= rec.last; i0 += kPjGroups * kPjAhead) {
        float2 st[kPjAhead];
        f4v v[kPjAhead];
#pragma unroll
        for (int u = 0; u < kPjAhead; ++u) {
            const int i = i0 + u * kPjGroups;
            if (i > rec.last) continue;
            const int64_t at = (int64_t)(2 * i + (i == id ? 1 : 0)) * rows + r;
            st[u] = ws.state[at];
            v[u] = reinterpret_cast<const f4v*>(ws.part)[at * (kD / 4) + d4];
        }
#pragma unroll
        for (int u = 0; u < kPjAhead; ++u) {
            if (i0 + u * kPjGroups > rec.last) continue;
            const float to = fmaxf(top, st[u].x);
            const float c0 = state_factor(top, to, c2), c1 = state_factor(st[u].x, to, c2);
            l = l * c0 + st[u].y * c1;
            acc = acc * c0 + v[u] * c1;
            top = to;
        }
    }
    so[sub][d4] = acc;
    if (d4 == 0) {
        sr[sub] = top;
        sl[sub] = l;
    }
    __syncthreads();
    if (sub != 0) return;
    top = -__builtin_huge_valf();
    l = 0.f;
    acc = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kPjGroups; ++i) top = fmaxf(top, sr[i]);
#pragma unroll
    for (int i = 0; i < kPjGroups; ++i) {
        const float c = state_factor(sr[i], top, c2);
        l += c * sl[i];
        acc += c * so[i][d4];
    }
    acc *= l > 0.f ? 1.f / l : l;
    const int tok = r / a.g;
    static_cast<h4v*>(a.out)[((int64_t)(seq.begin + tok) * a.hkv * a.g + head * a.g + r % a.g) * (kD / 4) + d4] =
        h4v{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
}

hipError_t launch_paged_prompt(const PagedArgs& a, hipStream_t s);
size_t paged_prompt_bytes(const PagedArgs& a);

}  // namespace pariskv
