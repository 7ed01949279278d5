// Attention of a few new tokens per sequence over its cache: drafted tokens with the tree they
// form (tree_attend), and the few-token form of the sliding window with sinks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.hpp"

namespace pariskv {

// One call.  The t new tokens of a sequence and the g query heads of a KV head are g t rows that
// read the same keys: row r is head r / t, token r % t.  The keys of a sequence, in order:
//   rows [0, sink_end) and [lo, hi) of its cache, then the drafts' own rows (Kt, Vt).
// Tree (window == 0): sink_end = lo = 0, hi = lens[seq] or n; every row sees all of them, and
// the drafts its mask names.  Sliding window: new token i stands at p = start + i, start =
// lens[seq] or n; it sees cache rows j <= p with j < sink or j > p - window; no drafts.
struct ChunkArgs {
    const void* q;        // float16 [batch][hkv g][t][D]
    const void* K;        // float16 [batch][hkv][capacity][D], or null with rec
    const void* V;
    const uint8_t* rec;   // quantised records [batch][hkv][capacity], or null
    int32_t k_bits, v_bits;
    int64_t capacity;
    const void* Kt;       // float16 [batch][hkv][t][D] (tree)
    const void* Vt;
    const int64_t* mask;  // [batch][t] or null: drafts j <= i
    const int32_t* lens;  // [batch] or null
    const int32_t* counts;  // new tokens of each sequence [batch] or null: t (sliding window)
    int64_t n;
    int64_t sink, window;
    int32_t batch, hkv, g, t;
    float scale;
    void* out;            // [batch][hkv g][t][D], float32 (tree) or float16 (sliding window)
    float* part;          // chunk_part_bytes
    int32_t splits;       // blocks that share a (sequence, KV head)'s keys, each `per` steps of 32
    int32_t per;          // of them; sequences with fewer keys leave the last ones idle
};

// Sets splits and per from the call's sizes alone (not from lens and counts).
void chunk_plan(ChunkArgs& a);
size_t chunk_part_bytes(const ChunkArgs& a);
// Bytes that this call and every smaller one need (batch, n, t, sink or window smaller).
size_t chunk_part_bound(ChunkArgs a);
hipError_t launch_chunk_attend(const ChunkArgs& a, hipStream_t s);
// Its first kernel for blocks of 64 or 128 rows (tile_attend.hip).
hipError_t launch_tile_attend(const ChunkArgs& a, int block, int row_tiles, int64_t groups, const char* name,
                              hipStream_t s);

// Whether a sliding-window call takes the few-token form: its blocks share a sequence's keys,
// those of the prompt form hold 128 tokens of one head and walk all of theirs.
bool few_tokens(const ChunkArgs& a);

// The prompt form of the sliding window (many new tokens): the same arguments, float16 out.
hipError_t launch_prompt_attend(const ChunkArgs& a, hipStream_t s);

}  // namespace pariskv
