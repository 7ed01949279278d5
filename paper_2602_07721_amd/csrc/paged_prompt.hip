// Attention of new tokens over pages where some sequence and KV head may have more than 32 rows:
// prompts, chunks of them, and the single tokens of other sequences in the same call.
//
// A block takes 128 rows of one KV head of a sequence -- row r is token r / g, head r % g, so that
// one tile of keys serves all of its heads -- 32 a wave, and walks their keys, or a share of them, in
// tiles of 64 through LDS, two buffers deep.  Per wave and tile:
//   S^T = K Q^T    matrix instructions of 32 x 32: a lane holds 32 keys' scores of one row, so a
//                  row's maximum needs one exchange and its sum none until the end,
//   O^T += V^T P^T the scores' own registers are the second operand (the sum over keys may run in any
//                  order that both operands agree on); V^T by transposing LDS reads.
// P is rounded to one float16 value, by up to 2^-11 of it, for outputs that are float16 themselves;
// the sum adds the rounded values, so the weights add up to one.  8192 tokens, 32 heads: 567 us, 713 with
// P in two parts; errors against 64 bits 2.09e-4 and 2.02e-4 of the outputs, of which their own rounding is 2.02e-4.
//
// Tiles that every row sees whole take no masks.  The next tile goes straight into LDS while one is
// computed on; a lane has looked up one of its keys' pages while the tile before was computed on, and
// gets those of the rows that it loads by permutes.
//
// Sequences of at most 16 rows, single tokens mostly, are walked as paged_attend.hip does it instead, by
// blocks of their own, the first: bound by HBM, they all run at once, and the tiles' blocks follow in the
// place of those that are done.  Side by side with them from the start, tiles wait for their keys behind
// the others' many loads: 5 us for 64 keys that take 1.3 otherwise.  30 sequences of 3 tokens, 12 rows, take
// 225 us so and 250 as tiles, single tokens 229 and 239.
//
// How the work is shared out, which every wave finds for itself from sums over the lengths, so a
// captured call stays right when lengths change: a block takes a tile, the longest of a sequence first,
// or, where that would leave many of them idle at the end, the tiles, one behind the other, are cut into as
// many stretches of equal work as the chip holds blocks (fewer if they were short), wherever the cuts fall,
// and a second kernel joins the softmax states of the tiles that were cut (at most two halves of tiles a
// block through memory).  4096 tokens over themselves, 32 heads, take 165 us by tiles and 184 cut; 512 over
// 32768 800 and 310.

#include <hip/hip_fp16.h>

#include "paged_device.hpp"

namespace pariskv {

namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;

// 16 bytes a lane from memory straight into LDS, lane i's behind lane i - 1's.  The builtin for 64-bit
// addresses makes the compiler wait for every LDS read at once as long as one is under way, where here
// reads are waited for one by one (565 us for 605: 8192 tokens, 32 heads).  What it writes is seen after
// loads_done() and a barrier; the compiler's own waits count it in as they are in order.
__device__ __forceinline__ void load_lds(const void* from, void* to) {
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)to);
    uint32_t m0;  // which the compiler takes for its own
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "v"(from), "s"(lds)
                 : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

constexpr int kPmRows = 128;    // rows of a tile
constexpr int kPmKeys = 64;     // keys of a tile
constexpr int kPmAhead = 4;     // operands read ahead
constexpr int kPmFewRows = 16;  // rows of a sequence that is walked as few

struct FewRows {
    int g;
    __device__ __forceinline__ bool operator()(const PagedSeq& s) const { return s.count * g <= kPmFewRows; }
};

// How one sequence of more rows is cut: into tiles of rows of a KV head, which cost base + kPmRows (i +
// 1), in units of a key times a query head, with what its first loads and its outputs take, as long as
// 4 tiles of keys.
struct PromptCut {
    int tiles;
    int64_t base;
    __device__ __forceinline__ PromptCut(const PagedArgs& a, const PagedSeq& s) {
        const int M = s.count * a.g;
        tiles = M <= kPmFewRows ? 0 : (M + kPmRows - 1) / kPmRows;
        base = (int64_t)max(s.len - s.count, 0) * a.g + 4 * kPmKeys * a.g;
    }
    // Cost of the tiles before tile i, of one KV head.
    __device__ __forceinline__ int64_t cost(int64_t i) const { return i * base + kPmRows / 2 * i * (i + 1); }
};
// Tiles of keys that the last row of a tile sees.
__device__ __forceinline__ int tile_keys(const PagedArgs& a, const PagedSeq& s, int tile) {
    const int last = s.len - s.count + (min((tile + 1) * kPmRows, s.count * a.g) - 1) / a.g;
    return (max(last + 1, 0) + kPmKeys - 1) / kPmKeys;
}

// A place in the line of all tiles: before tile `key` of a tile's keys; b = batch: its end.
struct PromptPlace {
    int b, head, tile, key;
};
__device__ __forceinline__ PromptPlace read_place(const PromptPlace& p, int lane) {
    return PromptPlace{__builtin_amdgcn_readlane(p.b, lane), __builtin_amdgcn_readlane(p.head, lane),
                       __builtin_amdgcn_readlane(p.tile, lane), __builtin_amdgcn_readlane(p.key, lane)};
}
__device__ __forceinline__ bool operator<(const PromptPlace& x, const PromptPlace& y) {
    if (x.b != y.b) return x.b < y.b;
    if (x.head != y.head) return x.head < y.head;
    if (x.tile != y.tile) return x.tile < y.tile;
    return x.key < y.key;
}
// The place `cost` behind the beginning of sequence b.
__device__ __forceinline__ PromptPlace prompt_place(const PagedArgs& a, int b, const PagedSeq& s, const PromptCut& c,
                                                    int64_t cost) {
    PromptPlace p;
    p.b = b;
    const int64_t per = c.cost(c.tiles);
    p.head = (int)quotient(cost, per);
    cost -= p.head * per;
    // The last tile i whose tiles before cost no more: 64 i^2 + (base + 64) i = cost solved, then put right.
    const double h = (double)(c.base + kPmRows / 2) / kPmRows;
    int64_t i = (int64_t)(sqrt(h * h + (double)cost / (kPmRows / 2)) - h);
    i = min(max(i, (int64_t)0), (int64_t)c.tiles - 1);
    while (i > 0 && c.cost(i) > cost) --i;
    while (i + 1 < c.tiles && c.cost(i + 1) <= cost) ++i;
    p.tile = (int)i;
    p.key = (int)quotient((cost - c.cost(i)) * tile_keys(a, s, p.tile), c.base + kPmRows * (i + 1));
    return p;
}

// What a block leaves for the joining kernel: the tile that its stretch began and did not end (b < 0:
// none), and whether it begins in the middle of a tile, and ends that.
enum { kMiddle = 1, kEnds = 2 };
struct PromptRecord {
    int b, head, tile;
    int first;
};
// The workspace, behind that of the few rows: records, then outputs and states, two slots of kPmRows
// rows a block: a tile begun in another block in slot 2 i, one that is not ended in slot 2 i + 1.
constexpr size_t kPmRecordBytes = (kPgBlocks * sizeof(PromptRecord) + 255) / 256 * 256;
struct PromptSpace {
    PromptRecord* record;  // [kPgBlocks]
    float* part;           // [2 kPgBlocks][wave][D / 8][lane][4]: as the waves hold their outputs
    float2* state;         // [2 kPgBlocks][kPmRows]
    __device__ __forceinline__ explicit PromptSpace(const PagedArgs& a) {
        char* p = FewSpace(a, kPmFewRows).end;
        record = reinterpret_cast<PromptRecord*>(p);
        part = reinterpret_cast<float*>(p + kPmRecordBytes);
        state = reinterpret_cast<float2*>(part + (int64_t)2 * kPgBlocks * kPmRows * kD);
    }
};

// The stretch of a block, from one place up to another, the sequence that it begins in, and which of the
// line it is.
struct PromptStretch {
    PromptPlace begin, end;
    PagedSeq seq;
    int id;
};
// Stretches that a tile is cut into at most, and tiles of keys of a stretch at least, on average: more stretches
// take longer to join than they save.  16 tokens of 8 heads take 56 us over 131072 rows and 26 over 8000, with 512
// stretches 80 and 55; 32 tokens of 8 x 4 heads over 3000 28 and 51.
constexpr int kPmShares = 128, kPmLeast = 4;
__device__ __forceinline__ PromptStretch prompt_stretch(const PagedArgs& a, uint32_t block) {
    const LaneSeqs mine(a);
    const PromptPlace none{a.batch, 0, 0, 0};
    PromptStretch out{none, none, PagedSeq{}, (int)block};
    int64_t work = 0, most = 0, least = 0, all;
    int tokens = 0, items = 0;  // tokens up to t + 1; with at most t, no more tiles than blocks were launched
    PagedSeq s{};
    mine.each_of(a, [&](int b, const PagedSeq& q) {
        s = q;
        const PromptCut c(a, s);
        tokens = min(tokens + s.count, a.t + 1);
        if (c.tiles == 0) return;
        work += c.cost(c.tiles) * a.hkv;
        items = (int)((uint32_t)items + (uint32_t)c.tiles * (uint32_t)a.hkv);
        most = max(most, c.base + (int64_t)kPmRows * c.tiles);
        least = max(least, c.base + kPmRows);
    });
    const int64_t before = wave_sum_before(work, &all);
    if (all == 0 || __builtin_amdgcn_readlane((int)wave_incl_sum((uint32_t)tokens), 63) > a.t)
        return out;  // the second: offsets that do not rise
    const int items_to = (int)wave_incl_sum((uint32_t)items), first_item = items_to - items;
    const int all_items = __builtin_amdgcn_readlane(items_to, 63);
    // The sequence of this lane's that has place x of a line: the last that begins there or before.
    int found = mine.b0;
    int64_t found_at = 0;
    auto find = [&](int64_t x, int64_t at, auto&& size) {
        found_at = at;
        if (mine.each == 1) return;
        mine.each_of(a, [&](int b, const PagedSeq& q) {
            const int64_t n = size(PromptCut(a, q)) * a.hkv;
            if (at <= x && n > 0) {
                found = b;
                found_at = at;
                s = q;
            }
            at += n;
        });
    };
    PromptPlace place = none;
    const int64_t step = quotient(all, kPgBlocks);
    // Equal stretches cost a sixteenth more than tiles, and what takes as long as 9 tiles of keys: partial
    // outputs and their join.  So a tile a block, if neither the longest tile, 3/4 of its cost as blocks
    // that are alone on a CU are faster, nor the last round of tiles takes that much longer: whether it is
    // not full, by half of the shortest tiles' cost, or a sequence begins there, its longest tiles first.
    // Of 98 calls that were timed both ways the taken one is 1.3% behind the faster on average, 13% at worst;
    // tiles take up to 6 times as long as cuts, cuts up to 28% longer than tiles.
    const int64_t more = step / 16 + 9 * kPmKeys * a.g;
    const int last = all_items - kPgBlocks, idle = -all_items & (kPgBlocks - 1);
    const bool late = first_item + (mine.each > 1 ? items : 1) > max(last, kPgBlocks);
    const bool cut = most - most / 4 > step + more ||
                     (items > 0 && items_to > last &&
                      (least / 2 * idle > more * kPgBlocks || (late && most - most / 4 > (all - before) / kPgBlocks + more)));
    if (!__any(cut)) {
        const int id = (int)block;
        const uint64_t who = __ballot(first_item <= id && id < items_to);
        if (who == 0) return out;
        if (first_item <= id && id < items_to) {
            find(id, first_item, [](const PromptCut& c) { return (int64_t)c.tiles; });
            // Consecutive blocks go to the 8 XCDs in turn, and so do the KV heads: those that read the
            // same keys share an L2.
            const int in = (int)(id - found_at);
            place = PromptPlace{found, in % a.hkv, PromptCut(a, s).tiles - 1 - in / a.hkv, 0};
        }
        const int owner = (int)__builtin_ctzll(who);
        out.begin = out.end = read_place(place, owner);
        ++out.end.tile;
        out.seq = read_lane(s, owner);
        return out;
    }
    const int64_t shares = quotient(all, kPmLeast * kPmKeys * a.g) & ~7ll;
    const int blocks = (int)min(min((int64_t)kPmShares * all_items, max(shares, (int64_t)8)), (int64_t)kPgBlocks);
    if (block >= blocks) return out;
    out.id = line_block(block, blocks);
    const int64_t each = quotient(all, blocks), rest = all - each * blocks;
    // Where the stretch begins and where it ends, by two lanes at once.
    const bool odd_lane = threadIdx.x & 1;
    int place_b = a.batch;
    int64_t place_in = 0;
    PagedSeq place_s{}, begin_s{};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int64_t id = out.id + e, x = id * each + min(id, rest);
        const uint64_t who = __ballot(before <= x && x < before + work);
        if (who == 0) continue;  // the end of the line
        const int owner = (int)__builtin_ctzll(who);
        if (before <= x && x < before + work) find(x, before, [](const PromptCut& c) { return c.cost(c.tiles); });
        const PagedSeq q = read_lane(s, owner);
        const int b = __builtin_amdgcn_readlane(found, owner);
        const int64_t in = x - read_lane(found_at, owner);
        if (e == 0) begin_s = q;
        if (odd_lane == (e == 1)) {
            place_b = b;
            place_in = in;
            place_s = q;
        }
    }
    if (place_b < a.batch) place = prompt_place(a, place_b, place_s, PromptCut(a, place_s), place_in);
    out.begin = read_place(place, 0);
    out.end = read_place(place, 1);
    out.seq = begin_s;
    return out;
}

template <int SHAPE>
__global__ __launch_bounds__(kPgThreads, 2) void paged_prompt_kernel(PagedArgs a) {
    // Arrays of their own, chosen at compile time: in one array the compiler cannot tell a read of
    // this tile from the loads under way to the next, and waits for them first.
    __shared__ u4v sk0[kPmKeys * 16], sk1[kPmKeys * 16], sv0[kPmKeys * 16], sv1[kPmKeys * 16];
    static_assert(few_wave_lds(kPmFewRows) <= (int)sizeof sk0, "a wave's share of few rows takes one of them");
    __shared__ int again;  // whether a wave has outputs that are not finite
    if (blockIdx.x < kPgBlocks) {
        few_stretch<kPmFewRows, SHAPE>(a, line_block(blockIdx.x, kPgBlocks), FewRows{a.g}, [&](int w) {
            return reinterpret_cast<unsigned char*>(w == 0 ? sk0 : w == 1 ? sk1 : w == 2 ? sv0 : sv1);
        });
        return;
    }
    const uint32_t block = blockIdx.x - kPgBlocks;
    PromptStretch stretch = prompt_stretch(a, block);
    PromptPlace place_now = stretch.begin;
    PagedSeq seq = stretch.seq;
    const PromptPlace end = stretch.end;
    PromptRecord record{-1, 0, 0, 0};
    const PromptSpace ws(a);
    while (place_now < end) {
    const int b = place_now.b, head = place_now.head;
    const int keys = tile_keys(a, seq, place_now.tile);
    const bool last_one = b == end.b && head == end.head && place_now.tile == end.tile;
    const int tile0 = place_now.key, tile1 = last_one ? end.key : keys;
    const bool whole = tile0 == 0 && tile1 == keys;
    const int64_t slot = 2 * stretch.id + (tile0 > 0 ? 0 : 1);
    if (!whole) {
        if (tile0 > 0) record.first = kMiddle | (tile1 == keys ? kEnds : 0);
        else record = PromptRecord{b, head, place_now.tile, record.first};
    }
    int tid = threadIdx.x;
    asm("" : "+v"(tid));  // what follows from it is made here, not kept in registers for the next tile
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int M = seq.count * a.g, len = seq.len, start = len - seq.count;
    const int row0 = place_now.tile * kPmRows, row1 = min(row0 + kPmRows, M);
    // Positions of the tile's first row, and of this wave's last.
    const int first_p = start + row0 / a.g;
    const int wave_row = row0 + 32 * wave;
    const bool idle = wave_row >= row1;  // a wave without rows
    const int wave_last = start + min(wave_row + 31, row1 - 1) / a.g;
    const int row = min(wave_row + col, row1 - 1), tok = row / a.g, qhead = head * a.g + row % a.g;
    const int p = start + tok;
    const int full = max(first_p + 1, 0) / kPmKeys;  // the tiles of keys before it are whole for every row

    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    const ScoreShape<SHAPE> shape(a, qhead);
    const float c2 = SHAPE ? 1.f : score_factor(a.scale);
    float r, nm, sum;
    float one = 1.f;  // kept from the compiler: x * one + sum stays one instruction that takes a float16 x
    asm("" : "+s"(one));
    f16v o[4];

    // One key of a tile a lane: its page's entry; its row, and whether it has one.  Keys behind the
    // last repeat it, those without a page the first that has one (row 0 of the pages is memory).
    auto entry_of = [&](int tile) { return page_entry(a, b, min(tile * kPmKeys + lane, len - 1)); };
    auto place = [&](int tile, int entry, uint64_t& there) {
        const bool good = (uint32_t)entry < (uint32_t)a.n_pages;
        there = __ballot(good);
        int at = good ? page_row(a, entry, head, min(tile * kPmKeys + lane, len - 1)) : 0;
        if (__builtin_expect(there != ~0ull, 0)) {
            const int other = there ? __builtin_amdgcn_readlane(at, (int)__builtin_ctzll(there)) : 0;
            at = good ? at : other;
        }
        return at;
    };
    // This wave's quarter of a tile straight into LDS, 4 rows an instruction, lane i's 16 bytes
    // behind lane i - 1's: the swizzle is in what a lane reads.
    const char* Kg = static_cast<const char*>(a.K);
    const char* Vg = static_cast<const char*>(a.V);
    auto load = [&](int at, u4v* nk, u4v* nv) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int first = 16 * i + 4 * wave, key = first + (lane >> 4), c = lane & 15;
            const int64_t from = (int64_t)__builtin_amdgcn_ds_bpermute(key << 2, at) * 256;
            load_lds(Kg + from + ((c ^ (key & 15)) << 4), nk + first * 16);
            load_lds(Vg + from + ((c ^ (4 * (key & 3))) << 4), nv + first * 16);
        }
    };
    // Values of V that are not finite (see finite_part) matter where not every row sees every key.
    // Looking for them in every such tile costs more than looking at the outputs; a block that has
    // outputs that are not finite takes its tiles once more, carefully: each wave takes those values
    // out of its quarter of a tile before the others see it.
    bool careful = false, odd = false;
    auto partly = [&](int tile, uint64_t there) { return __builtin_expect(tile >= full || there != ~0ull, 0); };
    auto clean = [&](int tile, uint64_t there, u4v* nv) {
        if (!careful || !partly(tile, there)) return;
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) note_odd(nv[(16 * i + 4 * wave) * 16 + lane], m);
        if (!__any(m & kOddBits)) return;
        odd = true;
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            u4v* at = nv + (16 * i + 4 * wave) * 16 + lane;
            *at = finite_part(*at);
        }
    };
    // Where this lane's transposing reads begin: key 4 half + (lane % 16) / 4, dims
    // 16 (lane / 16 % 2) + 4 (lane % 4).
    const int tkey = 4 * half + ((lane & 15) >> 2);
    const int tchunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

    int entry = 0;
    uint64_t there = 0, next = 0;  // keys of this tile and of the next that have pages
    auto load_first = [&]() {
        if (tile0 >= tile1) return;
        load(place(tile0, entry_of(tile0), there), sk0, sv0);
        if (tile0 + 1 < tile1) entry = entry_of(tile0 + 1);
    };
    load_first();
    if (tid == 0) again = 0;  // seen at the first barrier
    const u4v* qr = reinterpret_cast<const u4v*>(static_cast<const __half*>(a.q) +
                                                 (int64_t)(seq.begin + tok) * a.q_stride + qhead * kD);
    h8v qf[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) qf[c] = query_part(qr[2 * c + half], flip);

    // Tile `tile`, whose keys lie in ck and cv; loads the next into nk and nv.
    auto take = [&](int tile, const u4v* ck, const u4v* cv, u4v* nk, u4v* nv) __attribute__((always_inline)) {
        if (tile + 1 < tile1) {
            load(place(tile + 1, entry, next), nk, nv);
            if (tile + 2 < tile1) entry = entry_of(tile + 2);
        }
        const int base_row = tile * kPmKeys;
        if (!idle && base_row <= wave_last) {
            // Operands are read from LDS four instructions ahead of their use; left alone, the compiler
            // reads each when it is needed.
            f16v s[2];
            auto key_part = [&](int i) {  // of instruction i: dims 16 (i / 2) on, keys 32 (i % 2) on
                return as_h8(ck[(32 * (i & 1) + col) * 16 + ((2 * (i >> 1) + half) ^ (col & 15))]);
            };
            h8v kf[kPmAhead];
#pragma unroll
            for (int i = 0; i < kPmAhead; ++i) kf[i] = key_part(i);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const h8v k = kf[i % kPmAhead];
                __builtin_amdgcn_sched_barrier(0);
                s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qf[i >> 1], s[i & 1], 0, 0, 0);
                if (i + kPmAhead < 16) kf[i % kPmAhead] = key_part(i + kPmAhead);
            }
            if constexpr (SHAPE != kPlainScores) {
                const float from = (float)(base_row + 4 * half - p);
                shape.template operator()<32>([&](int i) -> float& { return reinterpret_cast<float*>(s)[i]; },
                                              [&](int i) { return from + (float)(8 * (i / 4) + i % 4); });
            }
            if (partly(tile, there)) {
                uint32_t w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) w[h] = bits_to(min(p, len - 1) - base_row - 32 * h) & (uint32_t)(there >> (32 * h));
                if (!__all((w[0] & w[1]) == ~0u))
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t m = w[h] >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(m & (1u << (8 * (i / 4) + i % 4)))) s[h][i] = -__builtin_huge_valf();
                    }
            }
            float top = -__builtin_huge_valf();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[h][i]);
            float base = nm < __builtin_huge_valf() ? nm : 0.f;
            if (__builtin_expect(__any(top > -__builtin_huge_valf() &&
                                       !(__builtin_fmaf(top, c2, nm) <= kUp + kSlack)), 0)) {
                const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                const float m = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
                if (m > r) {
                    const float c = raise(m, c2, r, nm);
                    sum *= c;
#pragma unroll
                    for (int d = 0; d < 4; ++d) o[d] *= c;
                    base = nm;
                }
                if (__builtin_expect(__any(nm != nm), 0)) {
                    const float off = nm != nm ? r : 0.f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[h] -= off;
                    base = nm != nm ? kUp : base;
                }
            }
            __builtin_amdgcn_s_setprio(1);  // ahead of another wave's S^T
            // Values of instruction i: keys 16 (i / 4) on, dims 32 (i % 4) on.
            auto value_part = [&](int i) {
                // One offset from the array: longer chains lose which array it is.
                const int at = tkey * 256 + (((4 * (i & 3) + tchunk) ^ (4 * (tkey & 3))) << 4) + (lane & 1) * 8 +
                               16 * (i >> 2) * 256;
                const char* vp = reinterpret_cast<const char*>(cv);
                const s4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(vp + at));
                const s4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(vp + (at + 8 * 256)));
                return join_h4(a0, a1);
            };
            h8v vf[kPmAhead];
#pragma unroll
            for (int i = 0; i < kPmAhead; ++i) vf[i] = value_part(i);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                h8v pf[2];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const h2v e = __builtin_convertvector(
                        (f2v{__builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i], c2, base)),
                             __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i + 1], c2, base))}), h2v);
                    sum = __builtin_fmaf((float)e[0], one, sum);
                    sum = __builtin_fmaf((float)e[1], one, sum);
                    pf[i / 8][i % 8] = e[0];
                    pf[i / 8][i % 8 + 1] = e[1];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = 8 * h + j, d = j & 3;
                    const h8v v = vf[i % kPmAhead];
                    __builtin_amdgcn_sched_barrier(1);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pf[j >> 2], o[d], 0, 0, 0);
                    if (i + kPmAhead < 16) vf[i % kPmAhead] = value_part(i + kPmAhead);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        loads_done();
        if (careful && tile + 1 < tile1) clean(tile + 1, next, nv);
        __syncthreads();  // and the next tile is there
        there = next;
    };
    for (;; careful = true) {
        r = -__builtin_huge_valf();
        nm = __builtin_huge_valf();
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        if (careful) load_first();
        loads_done();
        if (careful && tile0 < tile1) clean(tile0, there, sv0);
        __syncthreads();
        for (int tile = tile0; tile < tile1; tile += 2) {
            take(tile, sk0, sv0, sk1, sv1);
            if (tile + 1 < tile1) take(tile + 1, sk1, sv1, sk0, sv0);
        }
        if (careful) break;
        float m = 0.f;  // maximum() hands a NaN on
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < 4; ++d) m = __builtin_elementwise_maximum(m, __builtin_fabsf(o[d][i]));
        if (__any(!(m < __builtin_huge_valf()))) again = 1;
        __syncthreads();
        if (!again) break;
    }
    if (careful && __syncthreads_or(odd)) {
#pragma unroll 1
        for (int tile = tile0; tile < tile1; ++tile) {
            place(tile, entry_of(tile), there);
            if (!partly(tile, there)) continue;
#pragma unroll 1
            for (int key = 0; key < kPmKeys; ++key) {
                const int j = tile * kPmKeys + key;
                if (j > min(p, len - 1) || !(there >> key & 1)) continue;
                const h4v* v = reinterpret_cast<const h4v*>(
                                   Vg + (int64_t)page_row(a, page_entry(a, b, j), head, j) * 256) + half;
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    f4v part{0.f, 0.f, 0.f, 0.f};
                    add_odd(part, v[2 * c]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[c / 4][4 * (c % 4) + i] += part[i];
                }
            }
        }
    }

    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    const float l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    if (wave_row + col < row1) {
        if (whole) {
            const float inv = l > 0.f ? 1.f / l : l;
            h4v* out = static_cast<h4v*>(a.out) + ((int64_t)(seq.begin + tok) * a.hkv * a.g + qhead) * (kD / 4);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    out[8 * d + 2 * (i / 4) + half] =
                        h4v{(_Float16)(o[d][i] * inv), (_Float16)(o[d][i + 1] * inv), (_Float16)(o[d][i + 2] * inv),
                            (_Float16)(o[d][i + 3] * inv)};
        } else {
            const float fix = at_r(r, nm, c2);
            f4v* out = reinterpret_cast<f4v*>(ws.part) + (slot * kPgWaves + wave) * 1024 + lane;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    out[(4 * d + i / 4) * 64] = f4v{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * fix;
            if (half == 0) ws.state[slot * kPmRows + row - row0] = float2{left_r(r, l), l * fix};
        }
    }
    if (last_one) break;
    place_now.key = 0;
    const PromptCut cut(a, seq);
    if (++place_now.tile == cut.tiles) {
        place_now.tile = 0;
        if (++place_now.head == a.hkv) {
            place_now.head = 0;
            place_now.b = next_seq(a, place_now.b + 1, seq, [&](const PagedSeq& s) { return PromptCut(a, s).tiles > 0; });
        }
    }
    __syncthreads();  // LDS is read
    }
    if (block < kPgBlocks && threadIdx.x == 0) ws.record[stretch.id] = record;
}

// Adds a share's state of a row, reference and sum, and some dims of its output to those so far.  One that saw
// no key that counts left zeros, or values that are not finite.
template <int N>
__device__ __forceinline__ void add_state(float2 st, const f4v (&v)[N], float c2, float& top, float& l, f4v (&acc)[N]) {
    const bool none = st.x == -__builtin_huge_valf();
    const float to = fmaxf(top, st.x);
    const float c0 = none ? 1.f : rescale(top, to, c2), c1 = none ? 1.f : rescale(st.x, to, c2);
    l = l * c0 + (none ? 0.f : st.y * c1);
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = acc[j] * c0 + v[j] * c1;
    top = to;
}

// Joins the states of the tiles that blocks of the line began and did not end: joining block (id, d) the
// dims 32 d on of the tile that block id began, every lane what a lane of its number held.  Where at least
// kPmManyStates blocks had a tile's keys, the joining blocks of the first so many, which have no tile of their
// own, share it: each 8 dims of 32 rows, its waves every fourth state (16 tokens of 8 heads over 131072 rows,
// 512 states: 195 us by the first alone).
constexpr int kPmJoinBlocks = kD / 32, kPmManyStates = 16, kPmJoinAhead = 8;
static_assert(kPmManyStates * kPmJoinBlocks == kPmRows / 32 * (kD / 8), "one part each");
__device__ __forceinline__ void tile_join(const PagedArgs& a, int shaped, int id, int d) {
    __shared__ int slots[kPgBlocks];
    __shared__ f4v so[kPgWaves][64][1];
    __shared__ float2 ss[kPgWaves][32];
    const PromptSpace ws(a);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // The tile begun last by a block up to this one, kPmManyStates - 1 before it at most, and whether as many
    // blocks behind that one have nothing but its keys.
    const int near = id - (kPmManyStates - 1) + lane;
    const PromptRecord none{-1, 0, 0, 0}, about = near >= 0 && near < kPgBlocks ? ws.record[near] : none;
    const uint64_t begun = __ballot(about.b >= 0) & ((1ull << kPmManyStates) - 1);
    const uint64_t inside = __ballot(about.first == kMiddle);
    if (begun == 0) return;
    const int at_begin = 63 - __builtin_clzll(begun), begin = id - (kPmManyStates - 1) + at_begin;
    constexpr uint64_t kOthers = (1ull << (kPmManyStates - 1)) - 1;
    const bool many = (inside >> (at_begin + 1) & kOthers) == kOthers;
    if (begin < id && !many) return;
    const PromptRecord rec = ws.record[begin];
    // The block that ends the tile is the first behind with that mark; each between, and it, may have a state.
    int states = 1;
    if (tid == 0) slots[0] = 2 * begin + 1;
    for (int i = begin + 1; i < kPgBlocks; i += 64) {  // every wave alike
        const int at = i + lane, first = at < kPgBlocks ? ws.record[at].first : 0;
        const uint64_t ends = __ballot(first & kEnds);
        const uint64_t mine = __ballot(first & kMiddle) & (ends ? (2ull << __builtin_ctzll(ends)) - 1 : ~0ull);
        if (mine >> lane & 1) slots[states + __builtin_popcountll(mine & ((1ull << lane) - 1))] = 2 * at;
        states += __builtin_popcountll(mine);
        if (ends) break;
    }
    __syncthreads();
    const PagedSeq seq = paged_seq(a, rec.b);
    const float c2 = shaped ? 1.f : score_factor(a.scale);
    const int M = seq.count * a.g;
    h4v* const outs = static_cast<h4v*>(a.out);
    // Where the 4 dims 8 c + 4 half on of row `row` lie.
    auto place = [&](int row, int c) {
        return ((int64_t)(seq.begin + row / a.g) * a.hkv * a.g + rec.head * a.g + row % a.g) * (kD / 4) + 2 * c + (lane >> 5);
    };
    auto rounded = [](f4v o) { return h4v{(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]}; };
    float top = -__builtin_huge_valf(), l = 0.f;
    if (many) {
        const int part = (id - begin) * kPmJoinBlocks + d, w = part / (kD / 8), c = part % (kD / 8);
        const int row = rec.tile * kPmRows + 32 * w + (lane & 31);
        f4v acc[1] = {f4v{0.f, 0.f, 0.f, 0.f}};
        for (int i0 = wave; i0 < states; i0 += kPgWaves * kPmJoinAhead) {
            float2 st[kPmJoinAhead];
            f4v v[kPmJoinAhead][1];
#pragma unroll
            for (int u = 0; u < kPmJoinAhead; ++u) {
                const int i = i0 + kPgWaves * u;
                const int64_t slot = slots[min(i, states - 1)];
                st[u] = ws.state[slot * kPmRows + 32 * w + (lane & 31)];
                v[u][0] = reinterpret_cast<const f4v*>(ws.part)[(slot * kPgWaves + w) * 1024 + c * 64 + lane];
            }
#pragma unroll
            for (int u = 0; u < kPmJoinAhead; ++u) {
                if (i0 + kPgWaves * u >= states) break;
                add_state(st[u], v[u], c2, top, l, acc);
            }
        }
        so[wave][lane][0] = acc[0];
        if (lane < 32) ss[wave][lane] = float2{top, l};
        __syncthreads();
        if (wave != 0 || row >= M) return;
#pragma unroll
        for (int x = 1; x < kPgWaves; ++x) add_state(ss[x][lane & 31], so[x][lane], c2, top, l, acc);
        outs[place(row, c)] = rounded(acc[0] * (l > 0.f ? 1.f / l : l));
        return;
    }
    const int row = rec.tile * kPmRows + 32 * wave + (lane & 31);
    if (row >= M) return;
    f4v acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f4v{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < states; ++i) {
        const int64_t slot = slots[i];
        const float2 st = ws.state[slot * kPmRows + 32 * wave + (lane & 31)];
        const f4v* part = reinterpret_cast<const f4v*>(ws.part) + (slot * kPgWaves + wave) * 1024 + 4 * d * 64 + lane;
        f4v v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = part[j * 64];
        add_state(st, v, c2, top, l, acc);
    }
    const float inv = l > 0.f ? 1.f / l : l;
#pragma unroll
    for (int j = 0; j < 4; ++j) outs[place(row, 4 * d + j)] = rounded(acc[j] * inv);
}

// Both joins in one launch: four blocks for every tile that may be cut, then one for every row of the
// sequences of few.
__global__ __launch_bounds__(32 * kPjGroups) void paged_prompt_join_kernel(PagedArgs a, int shaped) {
    static_assert(32 * kPjGroups == kPgThreads, "blocks of both take as many threads");
    const int id = (int)blockIdx.x - kPgBlocks * kPmJoinBlocks;
    if (id < 0)
        tile_join(a, shaped, (int)blockIdx.x / kPmJoinBlocks, (int)blockIdx.x % kPmJoinBlocks);
    else
        few_join(a, kPmFewRows, shaped ? 1.f : score_factor(a.scale), id / kPmFewRows, id % kPmFewRows);
}

}  // namespace

size_t paged_prompt_bytes(const PagedArgs& a) {
    return FewSpace::bytes(kPmFewRows) + kPmRecordBytes + (size_t)2 * kPgBlocks * kPmRows * (kD + 2) * 4;
}

hipError_t launch_paged_prompt(const PagedArgs& a, hipStream_t s) {
    const int shape = score_shape(a);
    // At most so many tiles of rows.
    const int64_t some = a.batch < a.t ? a.batch : a.t;
    const int64_t tiles = ((int64_t)a.t * a.g / kPmRows + some) * a.hkv;
    ProfEvents pe = prof_begin("paged_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)(kPgBlocks + (tiles > kPgBlocks ? tiles : kPgBlocks))), dim3(kPgThreads), 0, s,
                              pe.start, pe.stop, 0, a);
    };
    by_shape(shape, [&](auto x) { go(paged_prompt_kernel<decltype(x)::value>); });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    pe = prof_begin("paged_join");
    hipExtLaunchKernelGGL(paged_prompt_join_kernel, dim3(kPgBlocks * (kPmJoinBlocks + kPmFewRows)), dim3(32 * kPjGroups), 0,
                          s, pe.start, pe.stop, 0, a, shape);
    return hipGetLastError();
}

}  // namespace pariskv
