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
// the sum adds the rounded values, so the weights add up to one.
//
// Tiles that every row sees whole take no masks.  The next tile goes straight into LDS while one is
// computed on; a lane has looked up one of its keys' pages while the tile before was computed on, and
// gets those of the rows that it loads by permutes.
//
// Where the rows are few or lengths differ, one block a tile of rows would leave the chip to the
// longest sequence: keys are cut into shares of about a kPmShares-th of all the call's work each,
// and a second kernel joins the shares' softmax states.  Each block finds its place from sums over
// the lengths, so a captured call stays right when lengths change.

#include <hip/hip_fp16.h>

#include "paged_device.hpp"

namespace pariskv {

namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* global_ptr;

constexpr int kPmThreads = 256;
constexpr int kPmRows = 128;  // rows of a block
constexpr int kPmKeys = 64;   // keys of a tile
constexpr int kPmShares = 1024;  // shares of about equal work that a call is cut into at least
constexpr int kPmJoinRows = 8;   // rows of a joining block

// How one sequence is cut: tiles of rows of a KV head, tiles of keys that the last of them sees, and
// shares of the keys.
struct PromptCut {
    int tiles, keys, shares;
};
__device__ __forceinline__ PromptCut prompt_cut(const PagedArgs& a, const PagedSeq& s) {
    PromptCut c;
    c.tiles = (s.count * a.g + kPmRows - 1) / kPmRows;
    c.keys = s.count > 0 ? max(1, (s.len + kPmKeys - 1) / kPmKeys) : 0;
    c.shares = 1;
    return c;
}

// The workspace, for the joining kernel: for each sequence its shares, where the tiles of rows that
// are cut begin (its and all before), and where their states do; then states and outputs.
struct CutLine {
    int64_t row;    // of its first state
    int32_t tile;   // of its first cut tile of rows
    int32_t shares;
};
struct PromptSpace {
    CutLine* cuts;  // [batch + 1]
    float2* state;  // [rows]
    float* part;    // [rows][D]
};
// Rows of states: a sequence's M rows of hkv heads in S <= keys / cap + 1 shares, S > 1 only where
// keys > cap, are at most 2 M hkv keys / cap, all together 2 * kPmRows * kPmShares; and a row of a KV
// head has at most kPmShares + 1 shares.
__host__ __device__ inline int64_t prompt_state_rows(const PagedArgs& a) {
    const int64_t most = (int64_t)2 * kPmRows * kPmShares, few = (int64_t)a.t * a.g * a.hkv * (kPmShares / a.hkv + 2);
    return few < most ? few : most;
}
__host__ __device__ inline size_t prompt_line_bytes(const PagedArgs& a) {
    return (((size_t)a.batch + 1) * sizeof(CutLine) + 255) / 256 * 256;
}
__device__ __forceinline__ PromptSpace prompt_space(const PagedArgs& a) {
    PromptSpace w;
    char* p = static_cast<char*>(a.workspace);
    w.cuts = reinterpret_cast<CutLine*>(p);
    w.part = reinterpret_cast<float*>(p + prompt_line_bytes(a));
    w.state = reinterpret_cast<float2*>(w.part + prompt_state_rows(a) * kD);
    return w;
}

// What a block works on.
struct PromptPlace {
    int b, head, tile, share, shares;
    int64_t row;  // of the sequence's first state
};

// Sums of x over the threads before this one, and over all.
__device__ __forceinline__ int64_t block_sum_before(int64_t x, int64_t* totals, int64_t* all) {
    const int wave = threadIdx.x >> 6;
    int64_t sum;
    int64_t before = wave_sum_before(x, &sum);
    if ((threadIdx.x & 63) == 0) totals[wave] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kPmThreads / 64; ++w) {
        before += w < wave ? totals[w] : 0;
        sum += totals[w];
    }
    *all = sum;
    return before;
}

// The block's place; false where there is none.
__device__ __forceinline__ bool prompt_place(const PagedArgs& a, PromptPlace& pl) {
    __shared__ int64_t totals[4][kPmThreads / 64];
    __shared__ PromptPlace found;
    const int tid = threadIdx.x;
    const int each = (a.batch + kPmThreads - 1) / kPmThreads;
    const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
    int64_t work = 0, all;
    for (int b = b0; b < b1; ++b) {
        const PromptCut c = prompt_cut(a, paged_seq(a, b));
        work += (int64_t)c.tiles * c.keys;
    }
    block_sum_before(work, totals[0], &all);
    const int64_t cap = max((all * a.hkv + kPmShares - 1) / kPmShares, (int64_t)4);
    auto cut = [&](int b, PagedSeq& s) {
        s = paged_seq(a, b);
        PromptCut c = prompt_cut(a, s);
        c.shares = c.keys > 0 ? (int)((c.keys + cap - 1) / cap) : 0;
        return c;
    };
    int64_t items = 0, rows = 0, tiles = 0, all_items, all_rows, all_tiles;
    PagedSeq s;
    for (int b = b0; b < b1; ++b) {
        const PromptCut c = cut(b, s);
        items += (int64_t)c.tiles * c.shares * a.hkv;
        if (c.shares > 1) {
            rows += (int64_t)s.count * a.g * c.shares * a.hkv;
            tiles += (int64_t)c.tiles * a.hkv;
        }
    }
    const int64_t first = block_sum_before(items, totals[1], &all_items);
    int64_t at = first, row = block_sum_before(rows, totals[2], &all_rows);
    int64_t tile = block_sum_before(tiles, totals[3], &all_tiles);
    if (blockIdx.x == 0) {
        const PromptSpace ws = prompt_space(a);
        int64_t r = row, t = tile;
        for (int b = b0; b < b1; ++b) {
            const PromptCut c = cut(b, s);
            ws.cuts[b] = CutLine{r, (int32_t)t, c.shares};
            if (c.shares > 1) {
                r += (int64_t)s.count * a.g * c.shares * a.hkv;
                t += (int64_t)c.tiles * a.hkv;
            }
        }
        if (tid == 0) ws.cuts[a.batch] = CutLine{all_rows, (int32_t)all_tiles, 0};
    }
    const int64_t id = blockIdx.x;
    if (id >= all_items) return false;
    if (first <= id && id < first + items) {
        for (int b = b0;; ++b) {
            const PromptCut c = cut(b, s);
            const int64_t n = (int64_t)c.tiles * c.shares * a.hkv;
            if (id < at + n) {
                // Consecutive blocks go to the 8 XCDs in turn, and so do the KV heads: those that
                // read the same keys share an L2.  The last tiles, which see the most keys, first.
                const int in = (int)(id - at);
                found.b = b;
                found.head = in % a.hkv;
                found.tile = c.tiles - 1 - in / a.hkv / c.shares;
                found.share = in / a.hkv % c.shares;
                found.shares = c.shares;
                found.row = row;
                break;
            }
            at += n;
            if (c.shares > 1) row += (int64_t)s.count * a.g * c.shares * a.hkv;
        }
    }
    __syncthreads();
    pl = found;
    return true;
}

template <int SHAPE>
__global__ __launch_bounds__(kPmThreads, 2) void paged_prompt_kernel(PagedArgs a) {
    // Arrays of their own, chosen at compile time: in one array the compiler cannot tell a read of
    // this tile from the loads under way to the next, and waits for them first.
    __shared__ u4v sk0[kPmKeys * 16], sk1[kPmKeys * 16], sv0[kPmKeys * 16], sv1[kPmKeys * 16];
    __shared__ int again;  // whether a wave has outputs that are not finite
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;

    PromptPlace pl;
    if (!prompt_place(a, pl)) return;  // the whole block
    const int b = __builtin_amdgcn_readfirstlane(pl.b), head = __builtin_amdgcn_readfirstlane(pl.head);
    const PagedSeq seq = paged_seq(a, b);
    const int M = seq.count * a.g, len = seq.len, start = len - seq.count;
    const int row0 = pl.tile * kPmRows, row1 = min(row0 + kPmRows, M);
    // Positions of the block's and of this wave's first and last rows.
    const int first_p = start + row0 / a.g, last_p = start + (row1 - 1) / a.g;
    const int wave_row = row0 + 32 * wave;
    const bool idle = wave_row >= row1;  // a wave without rows
    const int wave_last = start + min(wave_row + 31, row1 - 1) / a.g;
    const int row = min(wave_row + col, row1 - 1), tok = row / a.g, qhead = head * a.g + row % a.g;
    const int p = start + tok;
    // The tiles of keys that some row sees; this share's.
    const int all_tiles = (max(last_p + 1, 0) + kPmKeys - 1) / kPmKeys;
    const int tile0 = (int)((int64_t)all_tiles * pl.share / pl.shares);
    const int tile1 = (int)((int64_t)all_tiles * (pl.share + 1) / pl.shares);
    const int full = max(first_p + 1, 0) / kPmKeys;  // the tiles before it are whole for every row

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
            __builtin_amdgcn_global_load_lds((global_ptr)(Kg + from + ((c ^ (key & 15)) << 4)),
                                             (lds_ptr)(nk + first * 16), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_ptr)(Vg + from + ((c ^ (4 * (key & 3))) << 4)),
                                             (lds_ptr)(nv + first * 16), 16, 0, 0);
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

    if (tid == 0) again = 0;  // seen at the first barrier
    const u4v* qr = reinterpret_cast<const u4v*>(static_cast<const __half*>(a.q) +
                                                 (int64_t)(seq.begin + tok) * a.q_stride + qhead * kD);
    h8v qf[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) qf[c] = query_part(qr[2 * c + half], flip);

    int entry = 0;
    uint64_t there = 0, next = 0;  // keys of this tile and of the next that have pages
    // Tile `tile`, whose keys lie in ck and cv; loads the next into nk and nv.
    auto take = [&](int tile, const u4v* ck, const u4v* cv, u4v* nk, u4v* nv) __attribute__((always_inline)) {
        if (tile + 1 < tile1) {
            load(place(tile + 1, entry, next), nk, nv);
            if (tile + 2 < tile1) entry = entry_of(tile + 2);
        }
        const int base_row = tile * kPmKeys;
        if (!idle && base_row <= wave_last) {
            f16v s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    s[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                        as_h8(ck[(32 * h + col) * 16 + ((2 * c + half) ^ (col & 15))]), qf[c], s[h], 0, 0, 0);
            if constexpr (SHAPE != kPlainScores) {
                const float from = (float)(base_row + 4 * half - p);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[h][i] = shape(s[h][i], from + (float)(32 * h + 8 * (i / 4) + i % 4));
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
                for (int k = 0; k < 2; ++k) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        // One offset from the array: longer chains lose which array it is.
                        const int at = tkey * 256 + (((4 * d + tchunk) ^ (4 * (tkey & 3))) << 4) + (lane & 1) * 8 +
                                       16 * (2 * h + k) * 256;
                        const char* vp = reinterpret_cast<const char*>(cv);
                        const s4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(vp + at));
                        const s4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v)(vp + (at + 8 * 256)));
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(join_h4(a0, a1), pf[k], o[d], 0, 0, 0);
                    }
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
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
        if (tile0 < tile1) {
            load(place(tile0, entry_of(tile0), there), sk0, sv0);
            if (tile0 + 1 < tile1) entry = entry_of(tile0 + 1);
            clean(tile0, there, sv0);
        }
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
    if (wave_row + col >= row1) return;
    if (pl.shares == 1) {
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
        const PromptSpace ws = prompt_space(a);
        const int64_t at = pl.row + ((int64_t)head * pl.shares + pl.share) * M + row;
        if (at >= prompt_state_rows(a)) return;  // offsets that do not rise
        const float fix = at_r(r, nm, c2);
        f4v* out = reinterpret_cast<f4v*>(ws.part) + at * (kD / 4);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                out[8 * d + 2 * (i / 4) + half] = f4v{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * fix;
        if (half == 0) ws.state[at] = float2{left_r(r, l), l * fix};
    }
}

// Joins the shares' states, 32 lanes a row, 4 dims a lane: a block takes 8 rows of a cut tile.
__global__ __launch_bounds__(32 * kPmJoinRows) void paged_prompt_join_kernel(PagedArgs a, int shaped) {
    constexpr int kBlocks = kPmRows / kPmJoinRows;
    const PromptSpace ws = prompt_space(a);
    const int id = (int)(blockIdx.x / kBlocks);
    if (id >= ws.cuts[a.batch].tile) return;
    int lo = 0, hi = a.batch;  // the last sequence whose first cut tile is not behind it
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ws.cuts[mid].tile <= id) lo = mid;
        else hi = mid;
    }
    const CutLine cut = ws.cuts[lo];
    const PagedSeq seq = paged_seq(a, lo);
    const int M = seq.count * a.g, in = id - cut.tile, head = in % a.hkv;
    if (in < 0) return;
    const int row = in / a.hkv * kPmRows + (int)(blockIdx.x % kBlocks) * kPmJoinRows + (int)(threadIdx.x >> 5);
    if (row >= M) return;
    const int d4 = threadIdx.x & 31;
    const float c2 = shaped ? 1.f : score_factor(a.scale);
    const int64_t at = cut.row + (int64_t)head * cut.shares * M + row;
    if (at + (int64_t)(cut.shares - 1) * M >= prompt_state_rows(a)) return;  // as above
    float top = -__builtin_huge_valf(), l = 0.f;
    f4v acc{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < cut.shares; ++s) {
        const float2 st = ws.state[at + (int64_t)s * M];
        const f4v v = reinterpret_cast<const f4v*>(ws.part)[(at + (int64_t)s * M) * (kD / 4) + d4];
        if (st.x == -__builtin_huge_valf()) {  // saw no key that counts: zeros, or values that are not finite
            acc += v;
            continue;
        }
        const float to = fmaxf(top, st.x);
        const float c0 = rescale(top, to, c2), c1 = rescale(st.x, to, c2);
        l = l * c0 + st.y * c1;
        acc = acc * c0 + v * c1;
        top = to;
    }
    acc *= l > 0.f ? 1.f / l : l;
    static_cast<h4v*>(a.out)[((int64_t)(seq.begin + row / a.g) * a.hkv * a.g + head * a.g + row % a.g) * (kD / 4) + d4] =
        h4v{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
}

}  // namespace

size_t paged_prompt_bytes(const PagedArgs& a) {
    return prompt_line_bytes(a) + (size_t)prompt_state_rows(a) * (kD + 2) * 4;
}

hipError_t launch_paged_prompt(const PagedArgs& a, hipStream_t s) {
    const int shape = (a.cap > 0.f ? kCappedScores : 0) | (a.slopes ? kBiasedScores : 0);
    // At most so many tiles of rows, and shares beyond one a tile.
    const int64_t some = a.batch < a.t ? a.batch : a.t;
    const int64_t tiles = ((int64_t)a.t * a.g / kPmRows + some) * a.hkv;
    ProfEvents pe = prof_begin("paged_attend");
    auto go = [&](auto kernel) {
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)(tiles + kPmShares)), dim3(kPmThreads), 0, s, pe.start, pe.stop, 0, a);
    };
    if (shape == kPlainScores) go(paged_prompt_kernel<0>);
    else if (shape == kCappedScores) go(paged_prompt_kernel<1>);
    else if (shape == kBiasedScores) go(paged_prompt_kernel<2>);
    else go(paged_prompt_kernel<3>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t cut = tiles < kPmShares ? tiles : kPmShares;
    pe = prof_begin("paged_join");
    hipExtLaunchKernelGGL(paged_prompt_join_kernel, dim3((unsigned)(cut * (kPmRows / kPmJoinRows))),
                          dim3(32 * kPmJoinRows), 0, s, pe.start, pe.stop, 0, a, shape);
    return hipGetLastError();
}

}  // namespace pariskv
