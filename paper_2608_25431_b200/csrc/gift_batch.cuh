// The requests of one serving step: shapes derived from their lengths, and the mapping of a
// running index (row, block) back to its request.  The arithmetic compiles for host and device
// so that it can be checked without a GPU.
#pragma once
#include <stdint.h>

#include "../../include/gift.h"
#include "gf128.cuh"

namespace gift {

constexpr int32_t BATCH_MAX_OWNER = 1 << 20;    // user ids of a ctx are below this

// Division by a number that is fixed for a call, for dividends below 2^31: with l = ceil(log2 d)
// and m = ceil(2^(31+l) / d), which is below 2^32, t / d = t m >> (31 + l), since the excess t (m d -
// 2^(31+l)) < 2^31 2^l.  (The compiler's own division of unknown numbers is some 20 instructions,
// and the kernels divide several times per token.)
struct FixedDiv {
    uint32_t d, mul, shift;
    GIFT_HD uint32_t quot(uint32_t t) const { return (uint32_t)((uint64_t)t * mul >> shift); }
    // how many d cover t
    GIFT_HD uint32_t cover(uint32_t t) const { return t ? quot(t - 1u) + 1u : 0u; }
};
inline FixedDiv fixed_div(uint32_t d)
{
    uint32_t l = 0;
    while (l < 31 && (1u << l) < d) l++;
    FixedDiv f;
    f.d = d;
    f.shift = 31 + l;
    f.mul = d ? (uint32_t)((((uint64_t)1 << f.shift) + d - 1) / d) : 0u;
    return f;
}

// What a request's lengths say.  A malformed request takes no part in any call: no rows, no blocks.
struct ReqShape {
    bool ok;
    uint32_t have, want;     // tokens cached before the step, tokens after it
    uint32_t bh, bw;         // blocks that hold them
    uint32_t rows;           // tokens the step adds
};

GIFT_HD ReqShape req_shape(int32_t owner, int32_t have, int32_t want, const FixedDiv& page, uint32_t max_blocks)
{
    ReqShape s;
    s.ok = owner >= 0 && owner < BATCH_MAX_OWNER && have >= 0 && want >= 0;
    s.have = s.ok ? (uint32_t)have : 0u;
    s.want = s.ok ? (uint32_t)want : 0u;
    s.bh = page.cover(s.have);
    s.bw = page.cover(s.want);
    if (s.bh > max_blocks || s.bw > max_blocks) {
        s.ok = false;
        s.have = s.want = s.bh = s.bw = 0u;
    }
    s.rows = s.want > s.have ? s.want - s.have : 0u;
    return s;
}

// Blocks the request gains, or gives back.
GIFT_HD uint32_t req_need(const ReqShape& s) { return s.bw > s.bh ? s.bw - s.bh : 0u; }
GIFT_HD uint32_t req_give(const ReqShape& s) { return s.bh > s.bw ? s.bh - s.bw : 0u; }

// Largest r with first[r] <= k, for the exclusive prefix first[0 .. n-1] of the requests' counts
// (first[0] = 0): the request that item k belongs to.  Requests without items share their
// successor's prefix and are never the last such r.  k is below the sum of the counts.
GIFT_HD uint32_t req_of(const uint32_t* first, uint32_t n, uint32_t k)
{
    uint32_t lo = 0, hi = n;             // first[lo] <= k < first[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}

// A label taken as claimed for the length of one call: bit 30 flipped.  User ids are below 2^20
// and the special labels are small negatives, so no label of a map looks claimed.
GIFT_HD int32_t label_flip(int32_t l) { return l ^ 0x40000000; }
GIFT_HD bool label_claimed(int32_t l) { return (((uint32_t)l >> 30) & 1u) != ((uint32_t)l >> 31); }

// A page may be handed out only when nobody owns it, and given back only by its owner (or when a
// failed import left it unowned): another user's page and a parameter page stay where they are.
GIFT_HD bool label_takable(int32_t l) { return l == GIFT_OWNER_NONE; }
GIFT_HD bool label_givable(int32_t l, int32_t owner)
{
    return l == owner || l == GIFT_OWNER_NONE || l == GIFT_OWNER_CONFLICT;
}

// What a page's label says to a reader or writer of `owner`: the status bits it earns.
// A parameter page may be read by everyone (a shared prompt prefix) and written by no one.
GIFT_HD uint32_t label_read_status(int32_t l, int32_t owner)
{
    if (l == owner || l == GIFT_OWNER_PARAM) return 0u;
    return l < 0 ? GIFT_ST_UNOWNED : GIFT_ST_OWNER_MISMATCH;
}
GIFT_HD uint32_t label_write_status(int32_t l, int32_t owner)
{
    if (l <= GIFT_OWNER_NONE) return GIFT_ST_UNOWNED;
    return l == owner && owner >= 0 ? 0u : GIFT_ST_OWNER_MISMATCH;
}

// One serving step's work, laid end to end and cut into equal slices, one per resident CTA: slice
// w is [w * slice, (w+1) * slice).  A slice is at least `least` units so that a small call uses
// fewer CTAs instead of thinner slices.
GIFT_HD uint64_t slice_units(uint64_t total, uint32_t n_cta, uint32_t least)
{
    const uint64_t s = (total + n_cta - 1u) / n_cta;
    return s < least ? least : s;
}

// Host checks shared by the calls that take a gift_batch.
inline int batch_args_ok(const gift_batch* b)
{
    if (!b) return GIFT_E_INVAL;
    if (b->n_req == 0) return GIFT_OK;
    if (!b->owner || !b->have || !b->want || !b->table) return GIFT_E_INVAL;
    if (b->max_blocks == 0 || b->page_tokens == 0) return GIFT_E_INVAL;
    if (b->n_req > GIFT_MAX_REQS || b->page_tokens > GIFT_MAX_PAGE_TOKENS) return GIFT_E_RANGE;
    if (b->max_blocks > 0x7FFFFFFFu) return GIFT_E_RANGE;
    // slots are numbered page * page_tokens + offset in 31 bits
    if ((uint64_t)b->n_pages * b->page_tokens > 0x7FFFFFFFu) return GIFT_E_RANGE;
    return GIFT_OK;
}

#if defined(__CUDACC__)

struct BatchArgs {
    uint32_t n_req, max_blocks, page_tokens, n_pages;
    FixedDiv page;                   // by page_tokens
    const int32_t* __restrict__ owner;
    const int32_t* __restrict__ have;
    const int32_t* __restrict__ want;
    int32_t* table;
};

inline BatchArgs batch_args(const gift_batch* b)
{
    BatchArgs a;
    a.n_req = b->n_req; a.max_blocks = b->max_blocks; a.page_tokens = b->page_tokens; a.n_pages = b->n_pages;
    a.page = fixed_div(b->page_tokens);
    a.owner = b->owner; a.have = b->have; a.want = b->want; a.table = b->table;
    return a;
}

__device__ __forceinline__ ReqShape load_shape(const BatchArgs& b, uint32_t r)
{
    return req_shape(b.owner[r], b.have[r], b.want[r], b.page, b.max_blocks);
}

// Inclusive sum of v over the threads of the block, in thread order; *total is the block's sum.
// warp_sums: shared array of THREADS / 32.  Ends with a barrier, so it can be called again.
template <int THREADS>
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* warp_sums, uint64_t* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t o = __shfl_up_sync(0xFFFFFFFFu, v, d);
        if (lane >= d) v += o;
    }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; w++) {
        const uint64_t s = warp_sums[w];
        if (w < warp) before += s;
        all += s;
    }
    __syncthreads();
    *total = all;
    return v + before;
}

__device__ __forceinline__ uint32_t saturate32(uint64_t v) { return v > 0xFFFFFFFFull ? 0xFFFFFFFFu : (uint32_t)v; }

#endif

}  // namespace gift
