// Pages of a step's new tokens, planned where the lengths are: block tables, slots and offsets of a
// batch whose sequences grow, begin and end, without a word to the host.
//
// All of it is sums over the sequences before: sequence b's tokens begin at the sum of the counts
// before it, the i-th page that the step needs is the i-th from the top of the stack of free ones,
// and the pages that sequences give back go onto the stack first, the last one lowest, so that
// taking as many again takes the same ones in the same order.  A block takes as many
// sequences at a time as it has threads: a scan in each wave's registers and one over the waves' totals in LDS.
// Sums saturate at 2^32 - 1, which is past every limit that they are compared with.
//
// Bound by latency: lengths in, three scans, the popped pages, the slots, each waiting for the one
// before.  A decode step's tokens are placed by their sequences' threads; up to kPlanOwn of prompts by
// the same block, more by a second kernel of many blocks (a block writes 1024 slots in about 1 us, a
// launch costs 3).

#include "pages.hpp"

namespace pariskv {

namespace {

constexpr int kPlanMost = 1024;  // threads of the planning block, fewer for fewer sequences
constexpr int kPlanFew = 256;
constexpr int kPlanOwn = 4096;  // token slots that the planning block fills itself
constexpr int kFillThreads = 256;

__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// wave_incl_sum with sums that saturate.
__device__ __forceinline__ uint32_t wave_incl_sat(uint32_t v) {
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false));
    return v;
}

// Sum of v over the threads up to this one, and over all.  Ends with a barrier behind it that the
// next call's writes to `totals` have to wait for: calls in turn take two arrays in turn.
template <int THREADS>
__device__ __forceinline__ uint32_t block_incl_sat(uint32_t v, uint32_t* totals, uint32_t* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t in = wave_incl_sat(v);
    if (lane == 63) totals[wave] = in;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t x = totals[w];
        before = add_sat(before, w < wave ? x : 0u);
        sum = add_sat(sum, x);
    }
    *all = sum;
    return add_sat(before, in);
}

// What one sequence asks for.
struct Ask {
    uint32_t len, after;   // rows it has, rows it would have
    uint32_t held, wants;  // pages of both
    uint32_t fresh;        // new tokens
    bool shrinks, room;    // gives rows back; its table has room for the new ones
};
__device__ __forceinline__ Ask ask_of(const PlanArgs& a, int b) {
    Ask k{};
    if (b >= a.batch) return k;
    const int64_t most = min(a.width * (int64_t)a.page.d, kMaxKvRows);
    const int64_t len = min((int64_t)max(a.lens[b], 0), most);
    const int c = a.counts[b];
    const int64_t after = max(len + c, (int64_t)0);
    k.len = (uint32_t)len;
    k.fresh = (uint32_t)max(c, 0);
    k.shrinks = c < 0;
    k.room = after <= most;
    k.after = (uint32_t)min(after, most);
    k.held = a.page((uint32_t)len + a.page.d - 1);
    k.wants = a.page(k.after + a.page.d - 1);
    return k;
}

// The slot of row `in` of a page; -1 for a page below 0 and for a slot past 31 bits, which would wrap to another page's.
__device__ __forceinline__ int slot_of(const PlanArgs& a, int page, int in) {
    const int64_t slot = (int64_t)page * a.page.d + in;
    return page >= 0 && slot <= INT32_MAX ? (int)slot : -1;
}

// Slot and position of token i: its sequence is the last whose offset is not behind it.
template <class Offset>
__device__ __forceinline__ void fill_token(const PlanArgs& a, int i, Offset&& offset) {
    int slot = -1, pos = -1;
    if (i < offset(a.batch)) {
        // A decode step has token i at sequence i.
        int lo = min(i, a.batch - 1), hi = lo + 1;
        if (!(offset(lo) <= i && i < offset(hi))) {
            lo = 0;
            hi = a.batch;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (offset(mid) <= i) lo = mid;
                else hi = mid;
            }
        }
        const int n = a.granted[lo], at = i - offset(lo);
        if (at < n) {
            pos = a.new_lens[lo] - n + at;
            const uint32_t j = a.page((uint32_t)pos);
            slot = slot_of(a, a.table[lo * a.width + j], pos - (int)(j * a.page.d));
        }
    }
    a.slots[i] = slot;
    a.positions[i] = pos;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_pages_kernel(PlanArgs a) {
    __shared__ uint32_t t0[THREADS / 64], t1[THREADS / 64], taken;
    const int tid = threadIdx.x, lane = tid & 63;
    const uint32_t pages = (uint32_t)a.n_pages;
    const uint32_t free0 = (uint32_t)min((int64_t)max(a.n_free[0], 0), a.n_pages);

    // Given back: the i-th page, in the order of the sequences and of their rows, goes to place
    // free0 + all - 1 - i.
    uint32_t back = 0;
    if (a.batch > THREADS) {
        uint32_t mine = 0;
        for (int b = tid; b < a.batch; b += THREADS) {
            const Ask k = ask_of(a, b);
            mine = add_sat(mine, k.shrinks ? k.held - k.wants : 0u);
        }
        block_incl_sat<THREADS>(mine, t0, &back);
        __syncthreads();
    }
    uint32_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
        const Ask k = ask_of(a, b0 + tid);
        const uint32_t gives = k.shrinks ? k.held - k.wants : 0u;
        uint32_t all;
        const uint32_t first = add_sat(before, block_incl_sat<THREADS>(gives, t0, &all) - gives);
        if (a.batch <= THREADS) back = all;
        const int64_t end = (int64_t)free0 + back - 1;
        uint64_t who = __ballot(gives > 0);
        while (who) {  // a wave's lanes take the pages of one sequence after the other
            const int l = __builtin_ctzll(who);
            who &= who - 1;
            const uint32_t n = (uint32_t)__builtin_amdgcn_readlane((int)gives, l);
            const uint32_t f = (uint32_t)__builtin_amdgcn_readlane((int)first, l);
            const uint32_t keep = (uint32_t)__builtin_amdgcn_readlane((int)k.wants, l);
            const int32_t* from = a.table + (int64_t)(b0 + (tid - lane) + l) * a.width + keep;
            for (uint32_t j = lane; j < n; j += 64) {
                const int64_t at = end - f - j;
                if (at >= 0 && at < a.n_pages) a.free[at] = from[j];
            }
        }
        before = add_sat(before, all);
        __syncthreads();  // the totals are read, and the pages are there
    }
    const uint32_t top = min(add_sat(free0, back), pages);

    // The pages that are taken are the first of those that are wanted: once a sequence finds too few,
    // so does every one behind it that wants any.
    if (tid == 0) taken = 0u;  // seen at the next barrier
    uint32_t tokens = 0, wanted = 0;  // of the sequences before
    bool far = false;  // whether some sequence has more tokens than its thread places
    const bool place = a.t <= kPlanOwn;
    for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
        const int b = b0 + tid;
        const Ask k = ask_of(a, b);
        uint32_t all_tokens, all_pages;
        const uint32_t end = add_sat(tokens, block_incl_sat<THREADS>(k.fresh, t0, &all_tokens));
        const bool fits = k.room && end <= (uint32_t)a.t;
        const uint32_t needs = fits && k.fresh > 0 ? k.wants - k.held : 0u;
        const uint32_t upto = add_sat(wanted, block_incl_sat<THREADS>(needs, t1, &all_pages));
        const bool ok = fits && k.fresh > 0 && (needs == 0 || upto <= top);
        const uint32_t first = upto - needs;  // where it is ok, nothing saturated
        const uint32_t takes = ok ? needs : 0u;
        if (b < a.batch) {
            int32_t* row = a.table + (int64_t)b * a.width;
            int page = 0;
            if (takes == 1) row[k.held] = page = a.free[top - 1 - first];
            a.new_lens[b] = (int32_t)(ok || k.shrinks ? k.after : k.len);
            a.granted[b] = ok ? (int32_t)k.fresh : 0;
            a.offsets[b + 1] = (int32_t)min(end, (uint32_t)a.t);
            // A decode step's token: its page is at hand, or the last one held.
            if (place && k.fresh == 1 && end <= (uint32_t)a.t) {
                if (ok && takes == 0) page = row[k.held - 1];
                a.slots[end - 1] = ok ? slot_of(a, page, (int)(k.len - a.page(k.len) * a.page.d)) : -1;
                a.positions[end - 1] = ok ? (int)k.len : -1;
            }
            far |= k.fresh > 1;
            if (takes > 0) atomicMax(&taken, upto);
        }
        uint64_t who = __ballot(takes > 1);
        while (who) {
            const int l = __builtin_ctzll(who);
            who &= who - 1;
            const uint32_t n = (uint32_t)__builtin_amdgcn_readlane((int)takes, l);
            const uint32_t f = (uint32_t)__builtin_amdgcn_readlane((int)first, l);
            const uint32_t held = (uint32_t)__builtin_amdgcn_readlane((int)k.held, l);
            int32_t* to = a.table + (int64_t)(b0 + (tid - lane) + l) * a.width + held;
            for (uint32_t j = lane; j < n; j += 64) to[j] = a.free[top - 1 - f - j];
        }
        tokens = add_sat(tokens, all_tokens);
        wanted = add_sat(wanted, all_pages);
        if (b0 + THREADS < a.batch) __syncthreads();  // the totals are read
    }
    const bool rest = __syncthreads_or(far);  // and all of the plan is there
    if (tid == 0) {
        a.offsets[0] = 0;
        a.new_free[0] = (int32_t)(top - taken);
    }
    if (!place) return;
    const int real = (int)min(tokens, (uint32_t)a.t);
    for (int i = (rest ? 0 : real) + tid; i < a.t; i += THREADS) {
        if (i < real) {
            fill_token(a, i, [&](int b) { return b == 0 ? 0 : a.offsets[b]; });
        } else {
            a.slots[i] = -1;
            a.positions[i] = -1;
        }
    }
}

__global__ __launch_bounds__(kFillThreads) void fill_slots_kernel(PlanArgs a) {
    const int64_t i = (int64_t)blockIdx.x * kFillThreads + threadIdx.x;
    if (i < a.t) fill_token(a, (int)i, [&](int b) { return a.offsets[b]; });
}

}  // namespace

hipError_t launch_plan_pages(const PlanArgs& a, hipStream_t s) {
    ProfEvents pe = prof_begin("plan_pages");
    auto go = [&](auto kernel, int threads) {
        hipExtLaunchKernelGGL(kernel, dim3(1), dim3(threads), 0, s, pe.start, pe.stop, 0, a);
    };
    // Fewer waves meet at a barrier sooner: 64 sequences 6.1 us by 256 threads, 6.8 by 1024; 256 5.2 and 6.2.
    a.batch <= kPlanFew && a.t <= 4 * kPlanFew ? go(plan_pages_kernel<kPlanFew>, kPlanFew)
                                               : go(plan_pages_kernel<kPlanMost>, kPlanMost);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.t <= kPlanOwn) return e;
    pe = prof_begin("fill_slots");
    hipExtLaunchKernelGGL(fill_slots_kernel, dim3((unsigned)((a.t + kFillThreads - 1) / kFillThreads)), dim3(kFillThreads),
                          0, s, pe.start, pe.stop, 0, a);
    return hipGetLastError();
}

}  // namespace pariskv
