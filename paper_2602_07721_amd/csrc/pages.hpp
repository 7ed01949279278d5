// A cache of pages: K, V float16 [pages][hkv][page_size][D].  Row r of a sequence lies in page
// table[r / page_size] of its table, at r % page_size; a slot is page * page_size + that.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.hpp"

namespace pariskv {

// x / d for x < 2^31 by a product.  With d <= 2^l, mul = ceil(2^(31 + l) / d) = (2^(31 + l) + e) / d
// for an e < d, and x mul / 2^(31 + l) = x / d + x e / (d 2^(31 + l)), which adds less than 1 / d.
struct Divide {
    uint32_t d, mul, shift;
    __host__ __device__ uint32_t operator()(uint32_t x) const {
        return d == 1 ? x : (uint32_t)(((uint64_t)x * mul) >> 32) >> shift;
    }
};
inline Divide divide_by(int32_t d) {
    int l = 0;
    while ((int64_t(1) << l) < d) ++l;
    return Divide{(uint32_t)d, (uint32_t)(((uint64_t(1) << (31 + l)) + d - 1) / d), (uint32_t)(l > 0 ? l - 1 : 0)};
}

// Pages of the new rows of a step (plan_pages.hip).
struct PlanArgs {
    int32_t* table;  // [batch][width]
    int64_t width;
    Divide page;
    int32_t* free;  // the stack of free pages, of which *n_free hold something
    int64_t n_pages;
    const int32_t* n_free;
    const int32_t* lens;    // [batch]
    const int32_t* counts;  // [batch]
    int32_t batch, t;
    int32_t* new_lens;  // [batch], may be lens
    int32_t* new_free;  // [1], may be n_free
    int32_t* offsets;   // [batch + 1]
    int32_t* granted;   // [batch], may be counts
    int32_t* slots;     // [t]
    int32_t* positions; // [t]
};
hipError_t launch_plan_pages(const PlanArgs& a, hipStream_t s);

// New rows normalised, rotated and written (rotate_rows.hip).
struct RotateArgs {
    const void* q;  // float16 [t][hkv g][D], tokens *_stride values apart
    const void* k;  // [t][hkv][D]
    const void* v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t* positions;  // [t]
    const int32_t* slots;      // [t]
    const float* freqs;        // [rot / 2]
    const float* q_weight;     // [D] or null
    const float* k_weight;
    float eps;
    int32_t rot;
    bool pairs;
    void* q_out;  // [t][hkv g][D]
    void* K;
    void* V;
    int64_t n_slots;
    Divide page;
    int32_t t, hkv, g;
};
hipError_t launch_rotate_rows(const RotateArgs& a, hipStream_t s);

// Attention of packed new tokens over pages (paged_attend.hip, paged_prompt.hip).  The count new
// tokens of a sequence and the g query heads of a KV head are count g rows over the same keys: row r
// is token r / g, head r % g.  Token i stands at len - count + i and sees the keys up to there.
struct PagedArgs {
    const void* q;  // float16 [t][hkv g][D], tokens q_stride values apart
    int64_t q_stride;
    const void* K;
    const void* V;
    int32_t n_pages;
    Divide page;
    const int32_t* table;  // [batch][width]
    int64_t width;
    const int32_t* lens;     // [batch]
    const int32_t* offsets;  // [batch + 1]: where a sequence's tokens begin
    const int32_t* counts;   // [batch] or null: as far as the next one's
    int32_t t, most, batch, hkv, g;  // most: tokens of a sequence at most
    float scale, cap;        // cap 0: none
    const float* slopes;     // [hkv g] or null
    void* out;               // float16 [t][hkv g][D]
    void* workspace;         // paged_bytes
    int32_t blocks;          // of the few-token form
};

// Sets `blocks`; bytes of the workspace of the call and of every smaller one.
size_t paged_plan(PagedArgs& a);
hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s);

}  // namespace pariskv
