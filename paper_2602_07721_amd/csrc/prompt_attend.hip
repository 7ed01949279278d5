// Attention of a prompt, or of a long chunk of one, over a sliding window and the first tokens
// that stay visible: token p sees the rows j <= p with j < sink or j > p - window.
//
// P is rounded to one float16 value, by up to 2^-11 of it (2^-33 of the largest weight, where it
// is below 2^-22 of that), for outputs that are float16 themselves; the sum adds the rounded
// values, so that the weights add up to one.  8192 tokens, window 4096, outputs up to 4, against
// 64 bits: largest error 2.0e-3, root mean square 1.64e-4, of which rounding the outputs makes
// 1.95e-3 and 1.58e-4; with sums of the values before their rounding 3.3e-3 and 1.80e-4 in the
// same time.  P in two parts, as the few-token form has it, ends at the outputs' rounding, and
// takes 685 us where this takes 541.
//
// A block holds 128 tokens of one query head, 32 a wave, and walks the rows that any of them
// sees -- the sinks before the windows, then the stretch from the first token's window to the
// last token -- in tiles of 64 through LDS, two buffers deep.  Per wave and tile:
//   S^T = K Q^T    matrix instructions of 32 x 32: a lane holds 32 keys' scores of one token, so
//                  a row's maximum needs one exchange and its sum none until the end,
//   O^T += V^T P^T the scores' own registers are the second operand (the sum over keys may run in
//                  any order that both operands agree on); V^T by transposing LDS reads.
// Tiles inside every token's window take no masks.  The next tile goes straight into LDS while
// one is computed on.  Bound by the matrix and vector units together (4 D flops a visible pair,
// and an exponential, a maximum, a sum and a rounding), with LDS close behind: a wave reads 32
// KB a tile, which takes the block as long as its matrix instructions.  64 tokens a wave would
// halve that but leave one wave a SIMD: 870 us where 32 took 660.  32 heads, 8192 tokens after
// 8192 others, window 4096: 541 to 574 us from card to card, 990 to 1050 TFLOP/s (a plain float16
// matrix product: 1147).

#include <hip/hip_fp16.h>

#include "chunk_attend_device.hpp"

namespace pariskv {

namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kPaThreads = 256;
constexpr int kPaTokens = 128;  // tokens of a block
constexpr int kPaKeys = 64;     // keys of a tile
constexpr int kPaBufferWord3 = 0x00020000;  // buffer descriptor: raw, range-checked

__global__ __launch_bounds__(kPaThreads, 2) void prompt_attend_kernel(ChunkArgs a, int qtiles) {
    // Arrays of their own, chosen at compile time: in one array the compiler cannot tell a read of
    // this tile from the loads under way to the next, and waits for them first (653 us for 615 under a trace).
    __shared__ u4v sk0[kPaKeys * 16], sk1[kPaKeys * 16], sv0[kPaKeys * 16], sv1[kPaKeys * 16];
    __shared__ int again;  // whether a wave has outputs that are not finite
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;

    // The tiles with the most keys first (the last tokens of a prompt see the most), and the
    // heads of one KV head on one XCD, whose L2 then holds their keys.
    const uint32_t groups = (uint32_t)(a.batch * a.hkv), per = (uint32_t)(qtiles * a.g);
    uint32_t id = blockIdx.x, grp, in;
    const uint32_t full = groups / 8 * 8 * per;
    if (id < full) {
        grp = id / (8 * per) * 8 + id % 8;
        in = id / 8 % per;
    } else {
        id -= full;
        grp = full / per + id / per;
        in = id % per;
    }
    const int qt = qtiles - 1 - (int)(in / (uint32_t)a.g);
    const int seq = (int)(grp / (uint32_t)a.hkv);
    const int i0 = qt * kPaTokens;
    const KeySpan span = key_span(a, seq, i0, i0 + kPaTokens);
    if (i0 >= span.tokens) return;  // before any barrier, the whole block
    const int i1 = min(i0 + kPaTokens, span.tokens);
    const int sink = (int)a.sink, window = (int)a.window;
    // Tiles of 64 keys: the sinks', then the stretch's.
    const int sink_tiles = (span.sink_end + kPaKeys - 1) / kPaKeys;
    const int tiles = sink_tiles + (span.hi - span.lo + kPaKeys - 1) / kPaKeys;

    const int64_t head = (int64_t)grp * a.g + in % (uint32_t)a.g;  // (seq, query head)
    const float c2 = score_factor(a.scale);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    const int tok = min(i0 + 32 * wave + col, i1 - 1);
    const int p = span.start + tok;
    const int wave_first = span.start + min(i0 + 32 * wave, i1 - 1);
    const int wave_last = span.start + min(i0 + 32 * wave + 31, i1 - 1);
    float r, nm, sum;
    float one = 1.f;  // kept from the compiler: x * one + sum stays one instruction that takes a float16 x
    asm("" : "+s"(one));
    f16v o[4];

    char* Kg = static_cast<char*>(const_cast<void*>(a.K)) + (int64_t)grp * a.capacity * 256;
    char* Vg = static_cast<char*>(const_cast<void*>(a.V)) + (int64_t)grp * a.capacity * 256;
    // First row of a tile, and how many of its keys there are.
    auto tile_base = [&](int tile) {
        return tile < sink_tiles ? tile * kPaKeys : span.lo + (tile - sink_tiles) * kPaKeys;
    };
    auto tile_keys = [&](int tile) { return (tile < sink_tiles ? span.sink_end : span.hi) - tile_base(tile); };
    // This wave's quarter of a tile straight into LDS, 4 rows an instruction, lane i's 16 bytes
    // behind lane i - 1's: the swizzle is in what a lane reads.  Keys past the last repeat it:
    // what lies behind is not read.
    auto load = [&](int tile, u4v* nk, u4v* nv) {
        const int64_t base = (int64_t)tile_base(tile) * 256;
        const int most = tile_keys(tile) - 1;
        const auto kr = __builtin_amdgcn_make_buffer_rsrc(Kg + base, 0, kPaKeys * 256, kPaBufferWord3);
        const auto vr = __builtin_amdgcn_make_buffer_rsrc(Vg + base, 0, kPaKeys * 256, kPaBufferWord3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int first = 16 * i + 4 * wave, r = first + (lane >> 4), c = lane & 15;
            const int kat = min(r, most) * 256 + ((c ^ (r & 15)) << 4);
            const int vat = min(r, most) * 256 + ((c ^ (4 * (r & 3))) << 4);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_ptr)(nk + first * 16), 16, kat, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_ptr)(nv + first * 16), 16, vat, 0, 0, 0);
        }
    };
    // Tiles [full0, full1) are those of the stretch whose keys every token of the block sees.
    const int first_p = span.start + i0, last_p = span.start + i1 - 1;
    const int full0 = sink_tiles + (max(0, last_p - window + 1 - span.lo) + kPaKeys - 1) / kPaKeys;
    const int full1 = sink_tiles + max(0, first_p + 1 - span.lo) / kPaKeys;
    auto partly = [&](int tile) {
        return __builtin_expect(tile >= full1 || (tile < full0 && tile >= span.sink_end / kPaKeys), 0);
    };
    // Values of V that are not finite (see finite_part).  Looking for them in every other tile costs
    // 6% with a window of 512; so the outputs are looked at instead (1 to 2%), and a block that has
    // such ones takes its tiles once more, carefully: each wave takes those values out of its
    // quarter of a tile before the others see it.
    bool careful = false, odd = false;
    auto clean = [&](int tile, u4v* nv) {
        if (!careful || !partly(tile)) return;
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

    load(0, sk0, sv0);
    if (tid == 0) again = 0;  // seen at the first barrier
    const u4v* qr = reinterpret_cast<const u4v*>(static_cast<const __half*>(a.q) + (head * a.t + tok) * kD);
    h8v qf[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) qf[c] = query_part(qr[2 * c + half], flip);
    // Tile `tile`, whose keys lie in ck and cv; loads the next into nk and nv.
    auto take = [&](int tile, const u4v* ck, const u4v* cv, u4v* nk, u4v* nv) __attribute__((always_inline)) {
        if (tile + 1 < tiles) load(tile + 1, nk, nv);
        const int base_row = tile_base(tile), valid = tile_keys(tile);
        // Whether some token of the wave sees a key of the tile (its first key is at or before the
        // last token, and its first token's window or the sinks reach into it).
        const bool any = base_row <= wave_last &&
                         (base_row < sink || base_row + kPaKeys - 1 > wave_first - window);
        if (any) {
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
            if (partly(tile)) {
                uint32_t w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    w[h] = bits_to(valid - 1 - 32 * h) & window_bits(p, base_row + 32 * h, sink, window);
                if (!__all((w[0] & w[1]) == ~0u))
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t b = w[h] >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(b & (1u << (8 * (i / 4) + i % 4)))) s[h][i] = -__builtin_huge_valf();
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
            __builtin_amdgcn_s_setprio(1);  // ahead of another wave's S^T: 1%
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
        if (tile + 1 < tiles) clean(tile + 1, nv);
        __syncthreads();  // and the next tile is there
    };
    for (;; careful = true) {
        r = -__builtin_huge_valf();
        nm = __builtin_huge_valf();
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        if (careful) {
            load(0, sk0, sv0);
            clean(0, sv0);
        }
        __syncthreads();
        for (int tile = 0; tile < tiles; tile += 2) {
            take(tile, sk0, sv0, sk1, sv1);
            if (tile + 1 < tiles) take(tile + 1, sk1, sv1, sk0, sv0);
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
        for (int tile = 0; tile < tiles; ++tile) {
            if (!partly(tile)) continue;
#pragma unroll 1
            for (int key = 0; key < min(tile_keys(tile), kPaKeys); ++key) {
                const int j = tile_base(tile) + key;
                if (j > p || (j >= sink && j <= p - window)) continue;
                const h4v* v = reinterpret_cast<const h4v*>(Vg + (int64_t)j * 256) + half;
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
    const float inv = l > 0.f ? 1.f / l : 0.f;
    if (i0 + 32 * wave + col < i1) {
        h4v* out = static_cast<h4v*>(a.out) + (head * a.t + tok) * (kD / 4);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                out[8 * d + 2 * (i / 4) + half] =
                    h4v{(_Float16)(o[d][i] * inv), (_Float16)(o[d][i + 1] * inv), (_Float16)(o[d][i + 2] * inv),
                        (_Float16)(o[d][i + 3] * inv)};
    }
}

}  // namespace

hipError_t launch_prompt_attend(const ChunkArgs& a, hipStream_t s) {
    const int qtiles = (a.t + kPaTokens - 1) / kPaTokens;
    const ProfEvents pe = prof_begin("sink_window_attend");
    hipExtLaunchKernelGGL(prompt_attend_kernel, dim3((unsigned)((int64_t)a.batch * a.hkv * a.g * qtiles)),
                          dim3(kPaThreads), 0, s, pe.start, pe.stop, 0, a, qtiles);
    return hipGetLastError();
}

}  // namespace pariskv
