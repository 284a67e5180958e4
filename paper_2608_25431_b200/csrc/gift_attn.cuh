// Attention of a step's rows over the labelled paged cache: how the work is cut, and the pieces
// that the kernels share.
//
// An ITEM is one (request, K/V head, tile of query rows); the query rows of a K/V head are the
// request's tokens times the group of query heads that share the head.  An item costs the
// token tiles of its context and, before the first of them, some tiles' time for its start and end
// (`extra`): a batch whose shortest contexts are a few tiles would otherwise give one CTA
// many more items than the others.  Contexts differ by orders of magnitude, so the items'
// tiles are laid end to end and cut into equal slices, one per resident CTA (the split the
// cipher kernel uses).  A CTA walks its slice; an item that lies inside it is finished there, an
// item that a slice boundary cuts leaves its pieces' maxima, sums and unnormalised rows in
// scratch, to be joined: where the rows are few by the CTA whose piece is ready last, where they are
// many (128 rows are 64 KiB a piece) by a second kernel.  A slice has at most two such pieces (it enters one
// item in the middle and leaves one in the middle), so the scratch does not depend on the call.
//
// Where the rows of a K/V head fill several tiles, two CTAs walk one slice together (`ways` 2): its
// units are then those of pairs of a request's items (2 k, 2 k + 1), and each CTA takes its own of
// every pair.  Neighbouring items are tiles of query rows of one K/V head, so the second reader
// of every token finds it in L2.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gift_batch.cuh"

namespace gift {

// What the joining kernel has to know of a piece.  The first piece of a cut item describes the item.
struct PartHead {
    uint32_t pieces;                 // of the item, this one included; 0: this slot is not a first piece
    uint32_t bits;                   // status bits of the piece's pages
    uint32_t r, row0, rows_m;        // request, its first row, its rows
    uint32_t h, q0, nr;              // K/V head, the item's first query row and number of query rows
};

struct AttnArgs {
    BatchArgs b;
    const char* pages;
    uint64_t token_bytes;            // K and V of one token
    uint32_t kv_heads, heads, group;
    FixedDiv by_group, by_tile_rows;
    const char* q;
    uint64_t q_row, q_head;          // strides in bytes
    char* out;
    uint64_t out_row, out_head;
    uint32_t n_rows;
    float scale_log2;                // scale * log2(e): scores are kept in base 2
    uint32_t run;                    // tcgen05 kernel: tokens that are one copy (see there); below 8: gathered
    uint32_t negate;                 // tcgen05 kernel: scale_log2 is the positive one, q is negated
    const uint32_t* mask;
    uint32_t mask_words;
    float* lse;
    int32_t* row_owner;
    const int32_t* owner_map;
    uint32_t* status;
    uint32_t tile_rows;              // query rows of an item, at most
    uint32_t least;                  // smallest slice, in tiles
    uint32_t extra;                  // tiles that an item costs beyond its own
    uint32_t tile_tokens;            // few rows over codes: tokens of a tile; many rows over codes: step tokens of a tile of query rows
    uint32_t window;                 // tokens that a row may see, its own included; 0: all (kernels with WIN alone look at it)
    uint32_t n_slices, ways;         // slices, and CTAs that share one
    uint32_t wait_tries, wait_ns;    // tcgen05 kernel: further attempts of a wait, and the longest single one
    float* part_o;                   // [2 CTAs][rows][D]
    float2* part_ml;                 // [2 CTAs][rows] running maximum, sum
    PartHead* part_head;             // [2 CTAs]
    uint4* part_stall;               // [CTAs] many rows: requests x .. y - 1, which have rows z .. w - 1, were not all done
    uint32_t* tickets;               // few rows: [CTAs] pieces of the item that begins in a slice which are ready; [1] CTAs that are done
};

constexpr float NEG_INF = -__builtin_huge_valf();

// Shape of a request's items.
struct ItemShape {
    uint32_t rows_m;                 // step tokens
    uint32_t nqt;                    // tiles of query rows
    uint32_t tiles;                  // token tiles of the context, or (WIN) of what of it the rows may see
    uint32_t first;                  // WIN: the first of them
    uint32_t items;                  // nqt for every K/V head
    uint32_t cost;                   // units of one item (or pair of items): extra, then its tiles
    uint64_t units;                  // units of all its items
};

// The first token that a request's rows may see: its first row, at position have, sees the furthest back.
__device__ __forceinline__ uint32_t first_seen(const AttnArgs& a, uint32_t have) { return a.window && have >= a.window ? have - a.window + 1u : 0u; }

template <bool WIN = false>
__device__ __forceinline__ ItemShape item_shape(const AttnArgs& a, const ReqShape& s, uint32_t tile_tokens)
{
    ItemShape i;
    i.rows_m = s.rows;
    // rows * group fits 31 bits unless the step has more rows than the call, which is refused on the rows alone
    i.nqt = a.by_tile_rows.cover(s.rows * a.group & 0x7FFFFFFFu);
    i.tiles = (s.want + tile_tokens - 1) / tile_tokens;      // >= 1 when rows > 0
    if constexpr (WIN) {
        i.first = first_seen(a, s.have) / tile_tokens;
        i.tiles -= i.first;
    }
    i.cost = i.tiles + a.extra;
    i.items = i.nqt * a.kv_heads;
    i.units = (uint64_t)((i.items + a.ways - 1) / a.ways) * i.cost;
    return i;
}

// Where a unit lies.
struct Place {
    uint32_t r;                      // request
    uint32_t row0;                   // its first row
    uint32_t k, u;                   // the request's item (or pair), the unit's index within it
};

struct PlaceShared {
    uint64_t sums[32];
    Place at;
};

// Block-wide: the total of the requests' units and the place of unit w * slice.  Returns false
// (for every thread) when that unit does not exist, or the step has more rows than the caller
// gave; `first` marks the CTA that writes the status of requests without items.
template <int THREADS, bool WIN = false>
__device__ bool place_unit(const AttnArgs& a, uint32_t w, uint32_t tile_tokens, bool first,
                           PlaceShared* sh, uint64_t* total_out, uint64_t* slice_out)
{
    const uint32_t n = a.b.n_req, per = (n + THREADS - 1) / THREADS;
    const uint32_t r0 = threadIdx.x * per, r1 = r0 + per < n ? r0 + per : n;
    uint64_t rows = 0, units = 0;
#pragma unroll 1
    for (uint32_t r = r0; r < r1; r++) {
        const ReqShape s = load_shape(a.b, r);
        rows += s.rows;
        units += item_shape<WIN>(a, s, tile_tokens).units;
        if (first && s.rows == 0) a.status[r] = s.ok ? 0u : GIFT_ST_BAD_DESC;
    }
    uint64_t all_rows, total;
    const uint64_t incl_rows = block_scan<THREADS>(rows, sh->sums, &all_rows);
    const uint64_t incl = block_scan<THREADS>(units, sh->sums, &total);
    if (all_rows > a.n_rows) {
        if (first)
            for (uint32_t r = threadIdx.x; r < n; r += THREADS) a.status[r] = GIFT_ST_BAD_TABLE;
        return false;
    }
    const uint64_t slice = slice_units(total, a.n_slices, a.least);
    const uint64_t u = slice * w;
    *total_out = total;
    *slice_out = slice;
    if (u >= total) return false;
    uint64_t before = incl - units, row = incl_rows - rows;
    if (u >= before && u < incl) {
#pragma unroll 1
        for (uint32_t r = r0; r < r1; r++) {
            const ReqShape s = load_shape(a.b, r);
            const ItemShape it = item_shape<WIN>(a, s, tile_tokens);
            if (u < before + it.units) {
                sh->at.r = r;
                sh->at.row0 = (uint32_t)row;
                sh->at.k = (uint32_t)((u - before) / it.cost);
                sh->at.u = (uint32_t)((u - before) - (uint64_t)sh->at.k * it.cost);
                break;
            }
            before += it.units;
            row += s.rows;
        }
    }
    __syncthreads();
    return true;
}

// The pieces of a CTA's slice, in order.  TILE 0: tiles of a.tile_tokens.
template <uint32_t TILE, bool WIN = false> struct Walk {
    ReqShape s;
    ItemShape it;
    uint32_t r, row0;
    uint32_t way, k, u;              // which of the CTAs that share the slice; item (or pair); its units that are done
    uint64_t left;                   // units to go
    int32_t next_owner, next_have, next_want;       // of request r + 1, fetched ahead
    // the current piece: K/V head, tile of query rows, token tiles (WIN: counted from it.first)
    uint32_t h, qt, tb, n_tiles, all_q;

    __device__ __forceinline__ void fetch(const AttnArgs& a)
    {
        const uint32_t k = r + 1 < a.b.n_req ? r + 1 : r;
        next_owner = a.b.owner[k]; next_have = a.b.have[k]; next_want = a.b.want[k];
    }
    __device__ __forceinline__ void start(const AttnArgs& a, const Place& p, uint32_t which, uint64_t units)
    {
        way = which; k = p.k; u = p.u;
        r = p.r; row0 = p.row0; left = units;
        s = load_shape(a.b, r);
        it = item_shape<WIN>(a, s, TILE ? TILE : a.tile_tokens);
        fetch(a);
        all_q = it.rows_m * a.group;
    }
    __device__ __forceinline__ bool next(const AttnArgs& a)
    {
        while (left > 0) {
            if (u >= it.cost) {
                u = 0;
                if (++k * a.ways >= it.items) {
                    k = 0;
                    do {
                        row0 += it.rows_m;
                        r++;
                        s = req_shape(next_owner, next_have, next_want, a.b.page, a.b.max_blocks);
                        it = item_shape<WIN>(a, s, TILE ? TILE : a.tile_tokens);
                        fetch(a);
                    } while (it.nqt == 0);
                    all_q = it.rows_m * a.group;
                }
            }
            const uint32_t used = (uint64_t)(it.cost - u) < left ? it.cost - u : (uint32_t)left;
            const uint32_t end = u + used;
            tb = u > a.extra ? u - a.extra : 0u;
            n_tiles = (end > a.extra ? end - a.extra : 0u) - tb;       // none when the units end in the item's extra
            u = end;
            left -= used;
            const uint32_t item = k * a.ways + way;
            if (n_tiles == 0 || item >= it.items) continue;            // an odd last item has no partner
            h = item / it.nqt;
            qt = item - h * it.nqt;
            return true;
        }
        return false;
    }
    // Whether the piece is the whole item, and the scratch slot of one that is not: a slice's last piece, if
    // it starts an item, or its first one.
    __device__ __forceinline__ bool whole() const { return tb == 0 && n_tiles == it.tiles; }
    __device__ __forceinline__ uint32_t slot() const { return blockIdx.x * 2u + (tb == 0 ? 1u : 0u); }
    // One thread, after a piece that is not whole: what the joining kernel needs.  The item goes on in the
    // slices behind this one.
    __device__ __forceinline__ void write_head(const AttnArgs& a, uint32_t bits, uint64_t slice) const
    {
        PartHead p;
        const uint32_t rest = it.cost - u;
        p.pieces = tb == 0 ? 1u + (uint32_t)((rest + slice - 1) / slice) : 0u;
        p.bits = bits;
        p.r = r; p.row0 = row0; p.rows_m = it.rows_m;
        p.h = h; p.q0 = qt * a.tile_rows;
        p.nr = all_q - p.q0 < a.tile_rows ? all_q - p.q0 : a.tile_rows;
        a.part_head[slot()] = p;
    }
    // One thread, after a piece that could not be done: nor will any behind it in the slice.
    __device__ __forceinline__ void note_stall(const AttnArgs& a) const
    {
        uint4 s = a.part_stall[blockIdx.x];
        if (s.y == 0u) { s.x = r; s.z = row0; }
        s.y = r + 1u;
        s.w = row0 + it.rows_m;
        a.part_stall[blockIdx.x] = s;
    }
    // more step tokens than the mask has bits: the request is refused without looking at the mask
    __device__ __forceinline__ bool masked_short(const AttnArgs& a) const { return a.mask && it.rows_m > a.mask_words * 32u; }
};

// The kernel that joins this one's pieces may be launched.
__device__ __forceinline__ void join_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Which of the 64 tokens from t0 a request's i-th row (row `row` of the step) sees, as bits.
static __device__ __noinline__ uint64_t row_sees64(const AttnArgs& a, uint32_t have, uint32_t want, uint32_t row, uint32_t i, uint32_t t0)
{
    const uint32_t j0 = t0 > have ? t0 - have : 0u;            // first step token at or after t0
    const uint32_t cached = t0 < have ? have - t0 : 0u;
    if (cached >= 64u) return ~0ull;
    uint64_t own;                                                      // bit b: step token j0 + b
    if (a.mask) {
        const uint32_t* words = a.mask + (uint64_t)row * a.mask_words;
        const uint32_t k = j0 >> 5, sh = j0 & 31u;
        const uint64_t lo = k < a.mask_words ? words[k] : 0u, mid = k + 1 < a.mask_words ? words[k + 1] : 0u;
        const uint64_t hi = k + 2 < a.mask_words ? words[k + 2] : 0u;
        own = ((lo | (mid << 32)) >> sh) | (sh ? hi << (64u - sh) : 0ull);
    } else {
        const uint32_t n = i >= j0 ? i - j0 + 1u : 0u;
        own = n >= 64u ? ~0ull : (1ull << n) - 1ull;
    }
    uint64_t sees = (own << cached) | ((1ull << cached) - 1ull);
    const uint32_t there = want - t0;                              // tokens from t0 to the end, > 0
    if (there < 64u) sees &= (1ull << there) - 1ull;
    return sees;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }


template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }

// Whether either half of a pair is infinite or NaN.
template <class T> __device__ __forceinline__ bool pair_not_finite(uint32_t x)
{
    const uint32_t e = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    return (x & e) == e || ((x >> 16) & e) == e;
}

// BAD_DESC stands alone (no other bit is evaluated for a bad descriptor).
__device__ __forceinline__ uint32_t final_status(uint32_t bits) { return bits & GIFT_ST_BAD_DESC ? GIFT_ST_BAD_DESC : bits; }

// What one item's end writes besides its rows: by the first item of a request.
template <int THREADS>
__device__ __forceinline__ void write_request(const AttnArgs& a, uint32_t r, uint32_t row0, uint32_t rows_m, uint32_t bits)
{
    if (threadIdx.x == 0) a.status[r] = final_status(bits);
    if (a.row_owner) {
        const int32_t o = bits ? GIFT_OWNER_CONFLICT : a.b.owner[r];
        for (uint32_t t = threadIdx.x; t < rows_m; t += THREADS) a.row_owner[row0 + t] = o;
    }
}

}  // namespace gift
