// Attention over labelled pages of 8 bits, many query rows per K/V head: tcgen05 products.
//
// The roles and barriers of the 16-bit kernel: a tile of 128 query rows (or what whole tokens fit) meets tiles of 64
// tokens, S = Q K^T lands in tensor memory, one row per thread of four softmax warps, P goes back into the columns of
// its S and is the A operand of O += P V.  What differs:
//   warps 6, 7 fetch the codes (and scales) of K and of V into shared memory, two tiles ahead, judge the labels of the pages that
//              they read, and issue the products.
//   warps 4, 5 put the codes as fp16 numbers (exact) where the products read them.  (A product of codes
//              would need q and the weights as codes too.)
//   softmax    K's scale multiplies the score, V's the weight, in 32 bits.  Weights go to fp16 by a power of two of the row's
//              own, which follows the largest p * scale as the maximum follows the scores; O is in its units.
//              bf16 queries become fp16 in place, by a power of two of the row's own too.
// A code of NaN in a V whose token may be hidden from some row becomes 0, and the rows that see the token get their NaN at the piece's end: what
// a hidden token holds does not matter.
// 48 trees of 1 to 64 rows, 4 query heads to one, contexts of up to 16 384 tokens: 531 to 560 us, 373 to 393 TFLOP/s of the
// rows that exist; all of 64 rows: 740 us, 561 TFLOP/s; prompt chunks of 300 to 512 tokens, 8 requests: 194 us, capped 259 to 268, with scores that reach
// the cap 370.  What bounds it is a tile's
// chain through the softmax: of 128 rows and 64 tokens it takes a warp 2 200 to 3 300 clocks, with two such warps on
// a scheduler; issue slots are 43 % taken, the tensor pipe 30 %, HBM 36 %.
// Every wait is bounded; a CTA whose wait runs out notes its unfinished requests, and the joining kernel makes them zero.
#pragma once
#include "gift_attn8.cuh"
#include "gift_tc.cuh"

namespace gift {

constexpr int TC8_ROWS = 128;
constexpr int TC8_TILE = 64;
constexpr int TC8_THREADS = 256;
constexpr int TC8_AHEAD = 2;             // tiles whose codes are on their way
constexpr uint32_t SMALL_QUERY = 127u - 16u;     // exponent field of a row's largest element: S * K's scale is 2^24 q . k at most from it on
constexpr int TC8_BITS_RING = 8;         // pieces whose page verdicts are kept: no warp is more than three ahead of the softmax

template <int D> struct Tc8Smem {
    static constexpr uint32_t q = 0;                                                  // [D/64][128][64]
    static constexpr uint32_t k = TC8_ROWS * D * 2;                                   // [D/64][64][64]
    static constexpr uint32_t v = k + TC8_TILE * D * 2;
    static constexpr uint32_t o = v + TC8_TILE * D * 2;                               // [4 warps][32 rows][64 bytes]
    static constexpr uint32_t codes = o + 4 * 32 * 64;                                // of K, of V: [2 tiles][64][D]
    static constexpr uint32_t bytes = codes + 2 * TC8_AHEAD * TC8_TILE * D;
};


// One lane of a converged warp, in a way that lets the compiler see that one it is (products issued by it instead of by
// "lane 0": 612 -> 572 us for trees of up to 64 rows, at the time).
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0u;
}

// Items, slices and pieces as gift_attn.cuh has them, but an item has the tiles that its rows see: a prompt's early rows
// stop at their diagonal, and under a window late ones begin behind what they see.  With `ways` 2 the CTAs that share a
// slice take the two tiles of query rows of a group.  Where a head's tiles are odd in number its last one shares a group with
// that of the next head, whose own groups come behind it (with nobody beside it 733 us for trees of up to 64 rows,
// this way 581, at the time).
__device__ __forceinline__ GroupShape group_shape(const Attn8Args& a, const ReqShape& s)
{
    GroupShape p;
    p.have = s.have; p.want = s.want; p.rows = s.rows;
    p.per = a.tile_tokens * a.ways;
    // rows * group fits 31 bits unless the step has more rows than the call, which is refused on the rows alone
    p.groups = (a.by_tile_rows.cover(s.rows * a.group & 0x7FFFFFFFu) + a.ways - 1u) / a.ways;
    p.window = a.window;
    p.tree = a.mask != nullptr;
    return p;
}

// Whether heads come in such pairs, and the groups of head h.
__device__ __forceinline__ bool paired_heads(const Attn8Args& a, const GroupShape& p) { return a.ways == 2u && p.rows > 0 && ((p.rows + a.tile_tokens - 1u) / a.tile_tokens & 1u); }
__device__ __forceinline__ uint32_t groups_of(const GroupShape& p, bool pairs, uint32_t h) { return pairs && (h & 1u) ? p.groups - 1u : p.groups; }

struct Place8 {
    uint64_t sums[32];
    uint32_t r, row0, h, g, u;       // where a slice begins: request, its first row, K/V head, group, units of the item done
};

// As place_unit: the total of the requests' units and the place of unit w * slice.
template <int THREADS>
__device__ bool place_unit8(const Attn8Args& a, uint32_t w, bool first, Place8* sh, uint64_t* total_out, uint64_t* slice_out)
{
    const uint32_t n = a.b.n_req, per = (n + THREADS - 1) / THREADS;
    const uint32_t r0 = threadIdx.x * per, r1 = r0 + per < n ? r0 + per : n;
    uint64_t rows = 0, units = 0;
#pragma unroll 1
    for (uint32_t r = r0; r < r1; r++) {
        const ReqShape s = load_shape(a.b, r);
        rows += s.rows;
        if (s.rows) {
            const GroupShape p = group_shape(a, s);
            const uint64_t head = group_units_before(p, p.groups, a.extra);
            units += paired_heads(a, p) ? (a.kv_heads + 1u) / 2 * head + a.kv_heads / 2 * group_units_before(p, p.groups - 1u, a.extra) : a.kv_heads * head;
        } else if (first) {
            a.status[r] = s.ok ? 0u : GIFT_ST_BAD_DESC;
        }
    }
    uint64_t all_rows, total;
    const uint64_t incl_rows = block_scan<THREADS>(rows, sh->sums, &all_rows);
    const uint64_t incl = block_scan<THREADS>(units, sh->sums, &total);
    if (all_rows > a.n_rows) {
        if (first)
            for (uint32_t r = threadIdx.x; r < n; r += THREADS) a.status[r] = GIFT_ST_BAD_TABLE;
        return false;
    }
    const uint64_t slice = slice_units(total, a.n_slices, a.least), u = slice * w;
    *total_out = total;
    *slice_out = slice;
    if (u >= total) return false;
    uint64_t before = incl - units, row = incl_rows - rows;
    if (u >= before && u < incl) {
#pragma unroll 1
        for (uint32_t r = r0; r < r1; r++) {
            const ReqShape s = load_shape(a.b, r);
            if (s.rows == 0) continue;
            const GroupShape p = group_shape(a, s);
            const bool pairs = paired_heads(a, p);
            const uint64_t head = group_units_before(p, p.groups, a.extra), two = pairs ? head + group_units_before(p, p.groups - 1u, a.extra) : 2 * head;
            const uint64_t all = a.kv_heads / 2 * two + a.kv_heads % 2 * head;
            if (u < before + all) {
                uint32_t h = 2 * (uint32_t)((u - before) / two);
                uint64_t off = (u - before) % two;
                if (off >= head) {
                    h++;
                    off -= head;
                }
                uint32_t lo = 0, hi = groups_of(p, pairs, h);      // units before lo <= off < units before hi
                while (hi - lo > 1) {
                    const uint32_t mid = (lo + hi) >> 1;
                    if (group_units_before(p, mid, a.extra) <= off) lo = mid; else hi = mid;
                }
                sh->r = r; sh->row0 = (uint32_t)row;
                sh->h = h; sh->g = lo;
                sh->u = (uint32_t)(off - group_units_before(p, lo, a.extra));
                break;
            }
            before += all;
            row += s.rows;
        }
    }
    __syncthreads();
    return true;
}

struct Tc8Shared {
    uint64_t fetched[2][TC8_AHEAD], full[2], judged[2][TC8_BITS_RING];                 // of K, of V
    uint64_t scaled[4], checked[4], s_full[2], p_full[2], o_done[2], s_done, q_full, q_ready, last;
    float k_scale[4][TC8_TILE], v_scale[4][TC8_TILE];                                 // by tile
    uint32_t tmem;
    uint32_t bits[TC8_BITS_RING];
    int dead;
    Place8 place;
};

struct Walk8 {
    ReqShape s;
    GroupShape p;
    uint32_t r, row0;
    uint32_t way, at, g, u;          // which of the CTAs that share the slice; K/V head, group, its units that are done
    bool pairs;
    uint32_t cost;                   // of the group's items
    uint64_t left;                   // units to go
    int32_t next_owner, next_have, next_want;              // of request r + 1, fetched ahead
    // the current piece: K/V head, tile of query rows, first token tile, token tiles, whether it is the item's first or last one
    uint32_t h, qt, tb, n_tiles, all_q;
    bool starts, ends;

    __device__ __forceinline__ void fetch(const Attn8Args& a)
    {
        const uint32_t k = r + 1 < a.b.n_req ? r + 1 : r;
        next_owner = a.b.owner[k]; next_have = a.b.have[k]; next_want = a.b.want[k];
    }
    __device__ __forceinline__ void start(const Attn8Args& a, const Place8& x, uint32_t which, uint64_t units)
    {
        way = which; at = x.h; g = x.g; u = x.u;
        r = x.r; row0 = x.row0; left = units;
        s = load_shape(a.b, r);
        p = group_shape(a, s);
        pairs = paired_heads(a, p);
        cost = group_tiles(p, g) + a.extra;
        fetch(a);
    }
    __device__ __forceinline__ bool next(const Attn8Args& a)
    {
        while (left > 0) {
            if (u >= cost) {
                u = 0;
                if (++g >= groups_of(p, pairs, at)) {
                    g = 0;
                    at += pairs && p.groups == 1u ? 2u : 1u;       // a head with nothing of its own is passed over
                    if (at >= a.kv_heads) {
                        at = 0;
                        do {
                            row0 += s.rows;
                            r++;
                            s = req_shape(next_owner, next_have, next_want, a.b.page, a.b.max_blocks);
                            fetch(a);
                        } while (s.rows == 0);
                        p = group_shape(a, s);
                        pairs = paired_heads(a, p);
                    }
                }
                cost = group_tiles(p, g) + a.extra;
            }
            const uint32_t used = (uint64_t)(cost - u) < left ? cost - u : (uint32_t)left, end = u + used;
            const uint32_t done = u > a.extra ? u - a.extra : 0u;
            n_tiles = (end > a.extra ? end - a.extra : 0u) - done;     // none when the units end in the item's extra
            tb = group_first_tile(p, g) + done;
            starts = done == 0;
            ends = end == cost;
            u = end;
            left -= used;
            all_q = s.rows * a.group;
            h = at;
            qt = g * a.ways + way;
            if (pairs && way && g + 1u == p.groups) {              // the next head's last tile of rows, if there is one
                h = at + 1u;
                qt--;
            }
            if (n_tiles == 0 || h >= a.kv_heads) continue;
            return true;
        }
        return false;
    }
    // Whether the piece is the whole item, and the scratch slot of one that is not: a slice's last piece, if
    // it starts an item, or its first one.
    __device__ __forceinline__ bool whole() const { return starts && ends; }
    __device__ __forceinline__ uint32_t slot() const { return blockIdx.x * 2u + (starts ? 1u : 0u); }
    // One thread, after a piece that is not whole: what the joining kernel needs.  The item goes on in the
    // slices behind this one.
    __device__ __forceinline__ void write_head(const Attn8Args& a, uint32_t bits, uint64_t slice) const
    {
        PartHead x;
        x.pieces = starts ? 1u + (uint32_t)((cost - u + slice - 1) / slice) : 0u;
        x.bits = bits;
        x.r = r; x.row0 = row0; x.rows_m = s.rows;
        x.h = h; x.q0 = qt * a.tile_rows;
        x.nr = all_q - x.q0 < a.tile_rows ? all_q - x.q0 : a.tile_rows;
        a.part_head[slot()] = x;
    }
    // One thread, after a piece that could not be done: nor will any behind it in the slice.
    __device__ __forceinline__ void note_stall(const Attn8Args& a) const
    {
        uint4 x = a.part_stall[blockIdx.x];
        if (x.y == 0u) { x.x = r; x.z = row0; }
        x.y = r + 1u;
        x.w = row0 + s.rows;
        a.part_stall[blockIdx.x] = x;
    }
    // more step tokens than the mask has bits: the request is refused without looking at the mask
    __device__ __forceinline__ bool masked_short(const Attn8Args& a) const { return a.mask && s.rows > a.mask_words * 32u; }
};

// A role's walk lies in shared memory: its two dozen words are used at a piece's ends, registers in between.
static __device__ __noinline__ bool walk8_next(Walk8& w, const Attn8Args& a, uint32_t lane)
{
    Walk8 x = w;
    const bool more = x.next(a);
    __syncwarp();
    if (lane == 0) w = x;
    __syncwarp();
    return more;
}

// A softmax warp's rows of a piece whose results are written: their NaN from the tiles that some row does not see all of.
template <int D>
static __device__ __noinline__ void put_nan_piece(const Attn8Args& a, const Walk8& w, bool none)
{
    const uint32_t row = threadIdx.x, rho = w.qt * a.tile_rows + row;
    const bool there = rho < w.all_q && row < a.tile_rows && !(w.whole() && none);
    const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = w.h * a.group + (there ? rho - i * a.group : 0u);
    char* whole = a.out + (uint64_t)(w.row0 + i) * a.out_row + (uint64_t)hq * a.out_head;
    float* part = a.part_o + ((uint64_t)w.slot() * TC8_ROWS + row) * D;
#pragma unroll 1
    for (uint32_t x = 0; x < 2 * w.n_tiles; x++) {
        const uint32_t tile = (w.tb + x / 2) * TC8_TILE, t = tile + x % 2 * 32;
        if (tile + TC8_TILE <= w.s.have && !(a.window && tile + a.window < w.s.want)) continue;
        if (w.whole()) put_nan<D>(a, w.r, w.h, w.s.have, w.s.want, w.row0 + i, i, t, 32u, there, reinterpret_cast<uint16_t*>(whole));
        else put_nan<D>(a, w.r, w.h, w.s.have, w.s.want, w.row0 + i, i, t, 32u, there, part);
    }
}

// Waits until another role's generic writes may be read by the tensor cores' proxy.
__device__ __forceinline__ void publish_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int D, bool NEAR>
__global__ void __launch_bounds__(TC8_THREADS, 2)
attn8_tc_kernel(const __grid_constant__ Attn8Args a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap code_map)
{
    constexpr uint32_t TMEM_COLS = 256;                    // 2 S, O; a power of two, half of what an SM has
    constexpr uint32_t S_COL = 0, O_COL = 2 * TC8_TILE;
    extern __shared__ __align__(1024) char smem[];
    __shared__ __align__(16) Tc8Shared sh;
    __shared__ Walk8 walks[TC8_THREADS / 32 + 2];       // of the warps, and of the codes that two of them fetch
    using L = Tc8Smem<D>;

    join_may_start();
    if (threadIdx.x == 0) {
        a.part_head[blockIdx.x * 2u + 1u].pieces = 0u;
        a.part_stall[blockIdx.x] = make_uint4(0u, 0u, 0u, 0u);
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int kv = 0; kv < 2; kv++) {
            for (int i = 0; i < TC8_AHEAD; i++) bar_init(&sh.fetched[kv][i], 32);
            for (int i = 0; i < TC8_BITS_RING; i++) bar_init(&sh.judged[kv][i], 1);
            bar_init(&sh.full[kv], 1);
        }
        for (int i = 0; i < 4; i++) { bar_init(&sh.scaled[i], 32); bar_init(&sh.checked[i], 1); }
        for (int i = 0; i < 2; i++) { bar_init(&sh.s_full[i], 1); bar_init(&sh.p_full[i], 4); bar_init(&sh.o_done[i], 1); }
        bar_init(&sh.q_full, 1); bar_init(&sh.q_ready, 4); bar_init(&sh.s_done, 1); bar_init(&sh.last, 2);
        for (int i = 0; i < TC8_BITS_RING; i++) sh.bits[i] = 0u;
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    uint64_t total, slice;
    // ends with a barrier for every thread, taken or not
    const bool some = place_unit8<TC8_THREADS>(a, blockIdx.x / a.ways, blockIdx.x == 0, &sh.place, &total, &slice);
    if (!some) return;
    if (warp == 6) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem;
    volatile int* dead = &sh.dead;
    const uint64_t begin = slice * (blockIdx.x / a.ways), units = slice < total - begin ? slice : total - begin;
    const uint32_t sm = smem_u32(smem);
    Walk8& w = walks[warp];
    {
        Walk8 x;
        x.start(a, sh.place, blockIdx.x % a.ways, units);
        if (lane == 0) {
            w = x;
            if (warp >= 6) walks[warp + 2] = x;
        }
        __syncwarp();
    }

    // Of a tile's codes a lane fetches 16 from 16 chunk of every ROWS_AT_ONCE-th token.
    constexpr int ROW_LANES = D / 16, ROWS_AT_ONCE = 32 / ROW_LANES, LOADS = TC8_TILE / ROWS_AT_ONCE, PARTS = 4;
    const uint32_t chunk = lane % ROW_LANES, sub = lane / ROW_LANES;
    if (warp == 4 || warp == 5) {
        // ------------------------------------------------------------------ codes to fp16
        const uint32_t kv = warp - 4;
        const uint32_t raw = sm + L::codes + kv * (TC8_AHEAD * TC8_TILE * D) + lane * 16;
        // 16 codes are two 16-byte chunks of their row; lanes of the second block of 64 columns begin with the
        // second one, for other banks than those of the first
        const uint32_t block = chunk >> 2, dst = sm + (kv ? L::v : L::k) + block * (TC8_TILE * 128);
        uint32_t n = 0, piece = 0;
        bool ok = true;
        for (; ok && walk8_next(w, a, lane); piece++) {
            const uint32_t n_tiles = w.n_tiles, have = w.s.have, want = w.s.want, tb = w.tb;
#pragma unroll 1
            for (uint32_t j = 0; j < n_tiles; j++, n++) {
                const uint32_t t0 = (tb + j) * TC8_TILE, place = raw + (n % TC8_AHEAD) * (TC8_TILE * D);
                ok = warp_wait(&sh.fetched[kv][n % TC8_AHEAD], (n / TC8_AHEAD) & 1u, dead, a);
                if (!ok) break;
                if (kv) {
                    if (t0 + TC8_TILE > have || (NEAR && a.window && t0 + a.window < want)) {
#pragma unroll 1
                        for (int i = 0; i < LOADS; i++) {
                            const uint4 x = lds128(place + i * 512);
                            if (codes_nan(x.x) || codes_nan(x.y) || codes_nan(x.z) || codes_nan(x.w)) {
                                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(place + i * 512), "r"(codes_without_nan(x.x)),
                                             "r"(codes_without_nan(x.y)), "r"(codes_without_nan(x.z)), "r"(codes_without_nan(x.w)) : "memory");
                                atomicOr(&sh.bits[piece % TC8_BITS_RING], FOUND_NAN);
                            }
                        }
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sh.checked[n & 3u]);
                }
                // the product with the tile before is complete
                ok = n == 0 || (kv ? warp_wait(&sh.o_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, dead, a) : warp_wait(&sh.s_done, (n - 1) & 1u, dead, a));
                if (!ok) break;
                // A part's codes are loaded at once (one by one it is a chain of latencies), but the parts share their instructions: the
                // roles' loops together are about what the instruction cache holds (whole tiles of rows 710 -> 694 us at the time).
#pragma unroll 1
                for (int part = 0; part < PARTS; part++) {
                    uint4 x[LOADS / PARTS];
#pragma unroll
                    for (int i = 0; i < LOADS / PARTS; i++) x[i] = lds128(place + (part * (LOADS / PARTS) + i) * 512);
#pragma unroll
                    for (int i = 0; i < LOADS / PARTS; i++) {
                        const uint32_t row = (part * (LOADS / PARTS) + i) * ROWS_AT_ONCE + sub;
                        const uint32_t first[2] = {block ? x[i].z : x[i].x, block ? x[i].w : x[i].y}, second[2] = {block ? x[i].x : x[i].z, block ? x[i].y : x[i].w};
                        const uint32_t at = dst + row * 128 + (((chunk & 3u) * 2 + block ^ (row & 7u)) << 4);
                        uint32_t f[4];
                        four_codes(first[0], f[0], f[1]);
                        four_codes(first[1], f[2], f[3]);
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                        four_codes(second[0], f[0], f[1]);
                        four_codes(second[1], f[2], f[3]);
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at ^ 16u), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                    }
                }
                publish_smem();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.full[kv]);
            }
        }
    } else if (warp >= 6) {
        // ------------------------------------------------------------------ codes from the pages, and the products
        // Warp 6: K, and Q K^T; warp 7: V, and P V.  When a tile is converted the place that its codes had is free for those of
        // two tiles later, perhaps of another piece: what is fetched has a walk of its own.
        const uint32_t kv = warp - 6;
        const uint32_t raw = sm + L::codes + kv * (TC8_AHEAD * TC8_TILE * D);
        Walk8& f = walks[warp + 2];
        uint32_t fetched = 0, judged = 0, left = 0;            // tiles so far, pieces judged; tiles of the piece to go
        bool more = true, begun = false;
        uint32_t slot[2] = {0, 0}, slot_head = 0;              // of the next tile's tokens lane and lane + 32; its K/V head
        // The next tile's scales go where the softmax reads them: four tiles' places (the tile whose scales were here is
        // done, since V of the one behind it was converted).
        auto fetch_scales = [&]() {
            const char* scales = a.pages + 2ull * a.codes + slot_head * 8u;
            const uint32_t at = fetched & 3u;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const bool there = slot[e] != 0xFFFFFFFFu;
                const char* p = scales + (there ? slot[e] * a.token_bytes : 0ull);
                cp_async4(smem_u32(&sh.k_scale[at][e * 32 + lane]), p, there ? 4u : 0u);
                cp_async4(smem_u32(&sh.v_scale[at][e * 32 + lane]), p + 4, there ? 4u : 0u);
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.scaled[at])) : "memory");
        };
        auto fetch_codes = [&]() {
            const uint32_t at_place = fetched % TC8_AHEAD, place = raw + at_place * (TC8_TILE * D);
            uint64_t* bar = &sh.fetched[kv][at_place];
            if (a.copy_run >= 8) {
                // A run is one copy, by the lane that has its first token.  What it holds past the context, or before
                // a window, is hidden from every row; runs that nobody sees are sent outside the map, and are zeros.
                if (lane == 0) asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(TC8_TILE * D) : "memory");
                __syncwarp();
#pragma unroll
                for (uint32_t e = 0; e < 2; e++)
                    if (((e * 32 + lane) & (a.copy_run - 1u)) == 0u)
                        copy_run(place + (e * 32 + lane) * D, &code_map, (int32_t)(kv * a.codes + slot_head * D),
                                 slot[e] == 0xFFFFFFFFu ? -(int32_t)TC8_TILE : (int32_t)slot[e], bar);
                bar_arrive(bar);
            } else {
                // tokens that nobody sees are zeros: what memory holds there does not matter
                const char* from = a.pages + (uint64_t)kv * a.codes + (uint64_t)slot_head * D + chunk * 16;
#pragma unroll 4
                for (int i = 0; i < LOADS; i++) {
                    const uint32_t row = i * ROWS_AT_ONCE + sub;
                    const uint32_t at = __shfl_sync(0xFFFFFFFFu, i * ROWS_AT_ONCE < 32 ? slot[0] : slot[1], row & 31u);
                    const bool there = at != 0xFFFFFFFFu;
                    cp_async16(place + (i * 32 + lane) * 16, there ? from + at * a.token_bytes : from, there ? 16u : 0u);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
            }
            fetched++;
        };
        int32_t owner = 0, label[2] = {GIFT_OWNER_PARAM, GIFT_OWNER_PARAM}, page[2] = {-1, -1};
        const int32_t* table = nullptr;
        uint32_t want = 0, begin_t = 0, end_t = 0, from_t = 0, run_low = 0, base = 0, bits = 0;
        // Pages of 8 or more tokens: the lanes hold the table's entries of 32 pages (page[0]) and of the next 32, which are asked
        // for 32 pages ahead.  Every load waits for the copies of scales that were started before it, on the whole SM.
        // Smaller pages: the entries of tokens lane and lane + 32, asked for one tile ahead, labels judged a tile later.
        auto used = [&](uint32_t p) { return p * a.b.page_tokens < end_t && (p + 1u) * a.b.page_tokens > from_t; };
        auto entry = [&](uint32_t p) -> int32_t { return used(p) ? table[p] : -1; };
        auto entry_of = [&](uint32_t t) -> int32_t { return t < end_t && t >= from_t ? table[a.b.page.quot(t)] : -1; };
        auto judge = [&]() {
#pragma unroll
            for (int e = 0; e < 2; e++) {
                bits |= label_read_status(label[e], owner);
                label[e] = GIFT_OWNER_PARAM;
            }
        };
        auto ask = [&](int32_t p, bool there, int32_t& l) {    // for a page's label
            if (!there) return;
            if ((uint32_t)p >= a.b.n_pages) bits |= GIFT_ST_BAD_DESC;
            else if (a.owner_map) l = a.owner_map[p];
        };
        // the pages with tokens from lo to hi
        auto judge_pages = [&](uint32_t lo, uint32_t hi) {
            if (lo >= hi) return;
#pragma unroll 4
            for (uint32_t p = a.b.page.quot(lo) + lane; p * a.b.page_tokens < hi; p += 32) {
                int32_t l = GIFT_OWNER_PARAM;
                ask(table[p], true, l);
                bits |= label_read_status(l, owner);
            }
        };
        // The next tile's slots, and its scales.
        auto advance = [&]() {
            if (left == 0) {
                if (begun) {
                    // the piece's verdict
                    if (a.copy_run >= 8) ask(page[1], used(base + 32u + lane), label[1]);
                    judge();
                    bits = __reduce_or_sync(0xFFFFFFFFu, bits);
                    if (lane == 0) {
                        if (bits) atomicOr(&sh.bits[judged % TC8_BITS_RING], bits);
                        bar_arrive(&sh.judged[kv][judged % TC8_BITS_RING]);
                    }
                    judged++;
                }
                more = walk8_next(f, a, lane);
                if (!more) return;
                begun = true;
                left = f.n_tiles;
                owner = a.b.owner[f.r];
                table = a.b.table + (uint64_t)f.r * a.b.max_blocks;
                want = f.s.want;
                begin_t = f.tb * TC8_TILE;
                end_t = want - begin_t < left * TC8_TILE ? want : begin_t + left * TC8_TILE;
                const uint32_t low = NEAR ? first_seen(a, f.s.have) : 0u;
                from_t = NEAR && begin_t < low ? low : begin_t;
                run_low = low & ~(a.copy_run - 1u);
                bits = f.masked_short(a) ? GIFT_ST_BAD_DESC : 0u;
                // a request is served or refused as a whole: pages that other rows see and these do not are judged with the
                // item's first and last piece
                if (kv == 0 && f.starts) judge_pages(low, begin_t);
                if (kv == 0 && f.ends) judge_pages(end_t, want);
                if (a.copy_run >= 8) {
                    base = a.b.page.quot(from_t);
                    page[0] = entry(base + lane);
                    page[1] = entry(base + 32u + lane);
                    ask(page[0], used(base + lane), label[0]);
                } else {
#pragma unroll
                    for (int e = 0; e < 2; e++) page[e] = entry_of(begin_t + e * 32 + lane);
                }
            }
            if (a.copy_run >= 8) {
                if (begin_t > from_t && a.b.page.quot(begin_t) >= base + 32u) {
                    judge();
                    page[0] = page[1];
                    base += 32u;
                    page[1] = entry(base + 32u + lane);
                    ask(page[0], used(base + lane), label[0]);
                }
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const uint32_t t = begin_t + e * 32 + lane, p = a.b.page.quot(t), k = p - base;
                    const int32_t p0 = __shfl_sync(0xFFFFFFFFu, page[0], k & 31u), p1 = __shfl_sync(0xFFFFFFFFu, page[1], k & 31u);
                    const uint32_t at = (uint32_t)(k < 32u ? p0 : p1);
                    slot[e] = t < want && (!NEAR || t >= run_low) && at < a.b.n_pages ? at * a.b.page_tokens + (t - p * a.b.page_tokens) : 0xFFFFFFFFu;
                }
            } else {
                judge();
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const uint32_t t = begin_t + e * 32 + lane;
                    const bool there = t < end_t && t >= from_t;
                    ask(page[e], there, label[e]);
                    slot[e] = there && (uint32_t)page[e] < a.b.n_pages ? (uint32_t)page[e] * a.b.page_tokens + (t - a.b.page.quot(t) * a.b.page_tokens) : 0xFFFFFFFFu;
                    page[e] = entry_of(t + TC8_TILE);
                }
            }
            begin_t += TC8_TILE;
            left--;
            slot_head = f.h;
            if (kv) fetch_scales();
        };
        // The next tile's codes, and what the one behind it needs first.
        auto fetch = [&]() {
            if (!more) return;
            fetch_codes();
            advance();
        };
        // a negative scale: the products negate q, so that the scale used on the scores is positive
        const uint32_t id_s = instr_desc<__half>(TC8_ROWS, TC8_TILE, 0) | (a.negate << 13);
        constexpr uint32_t id_o = instr_desc<__half>(TC8_ROWS, D, 1);
        const uint64_t q_desc = smem_desc(sm + L::q, 16, 1024), k_desc = smem_desc(sm + L::k, 16, 1024);
        const uint64_t v_desc = smem_desc(sm + L::v, TC8_TILE * 128, 1024);
        uint32_t n = 0, piece = 0, q_loads = 0;
        bool ok = true;
        advance();
#pragma unroll 1
        for (int i = 0; i < TC8_AHEAD; i++) fetch();
        while (ok && walk8_next(w, a, lane)) {
            const uint32_t n_tiles = w.n_tiles;
            if (kv == 0) {
                // Q, once the products of the piece before have read the old rows.  What the box holds past the request's rows
                // is another request's: rows that nobody asks for.
                ok = n == 0 || warp_wait(&sh.s_done, (n - 1) & 1u, dead, a);
                if (!ok) break;
                q_loads++;
                if (lane == 0) {
                    bar_expect(&sh.q_full, a.tile_rows * D * 2);
#pragma unroll
                    for (int c = 0; c < D / 64; c++)
                        copy_q(sm + L::q + c * (TC8_ROWS * 128), &q_map, c * 64, (int32_t)(w.h * a.group),
                               (int32_t)(w.row0 + a.by_group.quot(w.qt * a.tile_rows)), &sh.q_full);
                }
                ok = warp_wait(&sh.q_ready, piece & 1u, dead, a);
            }
#pragma unroll 1
            for (uint32_t j = 0; ok && j < n_tiles; j++, n++) {
                ok = warp_wait(&sh.full[kv], n & 1u, dead, a);
                if (!ok) break;
                // S's columns, which held P of tile n - 2; or P
                ok = kv ? warp_wait(&sh.p_full[n & 1u], (n >> 1) & 1u, dead, a) : n < 2 || warp_wait(&sh.o_done[n & 1u], ((n - 2) >> 1) & 1u, dead, a);
                if (!ok) break;
                if (elect_one()) {
                    tc_after();
                    const uint32_t s_at = tmem + S_COL + (n & 1u) * TC8_TILE;
                    if (kv == 0) {
#pragma unroll
                        for (uint32_t ks = 0; ks < D / 16; ks++)       // 16 columns are 32 bytes; 64 columns a block
                            mma_ss(s_at, q_desc + (ks >> 2) * (TC8_ROWS * 128 / 16) + (ks & 3u) * 2,
                                   k_desc + (ks >> 2) * (TC8_TILE * 128 / 16) + (ks & 3u) * 2, id_s, ks > 0);
                        mma_commit(&sh.s_full[n & 1u]);
                        mma_commit(&sh.s_done);
                    } else {
#pragma unroll
                        for (uint32_t ks = 0; ks < TC8_TILE / 16; ks++)      // 16 tokens are 8 columns of P, 2048 bytes of V
                            mma_ts(tmem + O_COL, s_at + ks * 8, v_desc + ks * (2048 / 16), id_o, j > 0 || ks > 0);
                        mma_commit(&sh.o_done[n & 1u]);
                    }
                }
                __syncwarp();
                fetch();
            }
            piece++;
        }
        // the copies and products under way end before the CTA does, whether or not anybody is left to wait for them
        cp_commit();
        cp_wait<0>();
        for (uint32_t k = fetched > TC8_AHEAD ? fetched - TC8_AHEAD : 0; k < fetched; k++) bar_drain(&sh.fetched[kv][k % TC8_AHEAD], (k / TC8_AHEAD) & 1u);
        if (q_loads > 0) bar_drain(&sh.q_full, (q_loads - 1) & 1u);
        // nothing may be in flight when the tensor memory is given back (the lane that issued products commits them)
        if (elect_one()) mma_commit(&sh.last);
        __syncwarp();
        bar_drain(&sh.last, 0);
    } else {
        // ------------------------------------------------------------------ softmax
        const uint32_t row = threadIdx.x, lane_base = (warp * 32u) << 16;
        uint32_t n = 0, piece = 0;
        char* stage_o = smem + L::o + warp * (32 * 64);
        bool alive = true;
        while (walk8_next(w, a, lane)) {
            const uint32_t rho = w.qt * a.tile_rows + row;
            const bool there = rho < w.all_q && row < a.tile_rows;
            const bool warp_there = w.qt * a.tile_rows + warp * 32 < w.all_q && warp * 32 < a.tile_rows;
            const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = w.h * a.group + (there ? rho - i * a.group : 0u);
            const bool masked_short = w.masked_short(a);
            float scale = NEAR && a.cap_out != 0.f ? a.cap_in : a.scale_log2;
            if (alive && warp_wait(&sh.q_full, piece & 1u, dead, a)) {
                if (!a.half && warp_there) {
                    // this row as fp16 numbers, by a power of two
                    char* q = smem + L::q + row * 128;
                    uint32_t top = 0u;
#pragma unroll 4
                    for (uint32_t x = 0; x < D / 8; x++) {
                        const uint4 v = *reinterpret_cast<const uint4*>(q + (x >> 3) * (TC8_ROWS * 128) + (((x & 7u) ^ (row & 7u)) << 4));
                        const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int y = 0; y < 4; y++) top = max(top, max(word[y] << 16 & 0x7FFFFFFFu, word[y] & 0x7FFF0000u));
                    }
                    const uint32_t e = top_exponent(top);
                    // S meets K's scale before it meets the row's own, and q as large as that would let it leave 32 bits where q is small and
                    // K large, although q . k is ordinary.  Rows that far from one go to 2^-8, so that S is below 448; what that rounds is
                    // 2^-17 of the row's largest element.
                    const bool small = e < SMALL_QUERY;
                    const float f = to_half_range(e) * (small ? 0x1p-16f : 1.f);
                    scale *= from_half_range(e) * (small ? 0x1p16f : 1.f);
#pragma unroll 4
                    for (uint32_t x = 0; x < D / 8; x++) {
                        uint4* at = reinterpret_cast<uint4*>(q + (x >> 3) * (TC8_ROWS * 128) + (((x & 7u) ^ (row & 7u)) << 4));
                        uint4 v = *at;
                        v.x = pack2<__half>(__uint_as_float(v.x << 16) * f, __uint_as_float(v.x & 0xFFFF0000u) * f);
                        v.y = pack2<__half>(__uint_as_float(v.y << 16) * f, __uint_as_float(v.y & 0xFFFF0000u) * f);
                        v.z = pack2<__half>(__uint_as_float(v.z << 16) * f, __uint_as_float(v.z & 0xFFFF0000u) * f);
                        v.w = pack2<__half>(__uint_as_float(v.w << 16) * f, __uint_as_float(v.w & 0xFFFF0000u) * f);
                        *at = v;
                    }
                    publish_smem();
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.q_ready);
            } else {
                alive = false;
            }
            // the factor is positive (q's sign carries the scale's), and not 0, so that a hidden token's minus infinity stays
            scale = fmaxf(scale, __uint_as_float(1u));
            const float slope = NEAR && a.slopes && there ? a.slopes[hq] * LOG2_E : 0.f;
            float m = NOTHING, l = 0.f;                    // the maximum in use, the sum relative to it
            float most = 0.f, to_half = to_half_range(9u), room = half_range_end(9u);
            const uint32_t have = w.s.have;
            uint32_t t0 = w.tb * TC8_TILE, left = w.n_tiles;
            bool begun = false;
#pragma unroll 1
            for (; alive && left > 0; left--, n++, t0 += TC8_TILE, begun = true) {
                const uint32_t s_at = tmem + lane_base + S_COL + (n & 1u) * TC8_TILE;
                const bool mixed = t0 + TC8_TILE > have || (NEAR && a.window && t0 + a.window < w.s.want);
                uint64_t sees = ~0ull;
                if (mixed) {
                    sees = there && !masked_short ? row_sees64(a, have, w.s.want, w.row0 + i, i, t0) : 0ull;
                    if (NEAR && a.window) sees &= in_window64(a.window, have + i, t0);
                }
                // those of tile n + 4 are fetched when V of tile n + 1 is converted, so after P V of tile n
                if (!warp_wait(&sh.scaled[n & 3u], (n >> 2) & 1u, dead, a) || !warp_wait(&sh.s_full[n & 1u], (n >> 1) & 1u, dead, a)) {
                    alive = false;
                    break;
                }
                if (mixed && !warp_wait(&sh.checked[n & 3u], (n >> 2) & 1u, dead, a)) { alive = false; break; }      // for FOUND_NAN
                if (!warp_there) {                         // rows that do not exist: whatever P holds stays in them
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sh.p_full[n & 1u]);
                    continue;
                }
                tc_after();
                uint32_t sc[2][32];
                tc_ld32(sc[0], s_at);
                tc_ld32(sc[1], s_at + 32);
                tc_wait_ld();
                tc_pin32(sc[0]);
                tc_pin32(sc[1]);
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float4 ks = *reinterpret_cast<const float4*>(&sh.k_scale[n & 3u][32 * x + c]);
                        float y[4];
                        split2(mul2(pair2(__uint_as_float(sc[x][c]), __uint_as_float(sc[x][c + 1])), pair2(ks.x, ks.y)), y[0], y[1]);
                        split2(mul2(pair2(__uint_as_float(sc[x][c + 2]), __uint_as_float(sc[x][c + 3])), pair2(ks.z, ks.w)), y[2], y[3]);
#pragma unroll
                        for (int e = 0; e < 4; e++) sc[x][c + e] = __float_as_uint(y[e]);
                    }
                float by = scale;                          // what the scores still lack
                if constexpr (NEAR) {
                    if (a.cap_out != 0.f) {
                        float far[2] = {0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 2; x++)
#pragma unroll
                            for (int c = 0; c < 32; c += 2)
                                far[x] = max3(far[x], fabsf(__uint_as_float(sc[x][c])), fabsf(__uint_as_float(sc[x][c + 1])));
                        if (__any_sync(0xFFFFFFFFu, !(fmaxf(far[0], far[1]) * scale <= TANH_NEAR))) {
                            const uint64_t in2 = pair2(scale, scale), cap2 = pair2(a.cap_out, a.cap_out);
#pragma unroll
                            for (int x = 0; x < 2; x++)
#pragma unroll
                                for (int c = 0; c < 32; c++) sc[x][c] = __float_as_uint(capped(__uint_as_float(sc[x][c]) * scale, a.cap_out));
                        } else {
                            const uint64_t in2 = pair2(scale, scale), cap2 = pair2(a.cap_out, a.cap_out);
#pragma unroll
                            for (int x = 0; x < 2; x++)
#pragma unroll
                                for (int c = 0; c < 32; c += 2) {
                                    float lo, hi;
                                    split2(capped_near(mul2(pair2(__uint_as_float(sc[x][c]), __uint_as_float(sc[x][c + 1])), in2), cap2), lo, hi);
                                    sc[x][c] = __float_as_uint(lo);
                                    sc[x][c + 1] = __float_as_uint(hi);
                                }
                        }
                        by = 1.f;
                    }
                    if (a.slopes) {
                        const float away = (float)((int32_t)t0 - (int32_t)(have + i));
#pragma unroll
                        for (int x = 0; x < 2; x++)
#pragma unroll
                            for (int c = 0; c < 32; c++)
                                sc[x][c] = __float_as_uint(__uint_as_float(sc[x][c]) * by + slope * (away + (float)(32 * x + c)));
                        by = 1.f;
                    }
                }
                if (mixed) {
#pragma unroll
                    for (int x = 0; x < 2; x++)
#pragma unroll
                        for (int c = 0; c < 32; c++)
                            if (!((uint32_t)(sees >> (32 * x)) >> c & 1u)) sc[x][c] = 0xFF800000u;      // minus infinity
                }
                float tops[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int c = 0; c < 32; c += 2)
                        tops[(c >> 1) & 3] = max3(tops[(c >> 1) & 3], __uint_as_float(sc[x][c]), __uint_as_float(sc[x][c + 1]));
                // the scale is positive here (q's sign carries it), so the largest score stays the largest
                const float top = max3(tops[0], tops[1], fmaxf(tops[2], tops[3])) * by;
                const bool grow = top > m + 8.f;           // also when nothing has been seen yet
                float alpha = 1.f;
                if (grow) {
                    alpha = fast_exp2(m - top);
                    m = top;
                }
                const uint64_t by2 = pair2(by, by), minus2 = pair2(-m, -m);
                uint64_t sums[2] = {0ull, 0ull};
                float bigs[2] = {0.f, 0.f};
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float4 vs = *reinterpret_cast<const float4*>(&sh.v_scale[n & 3u][32 * x + c]);
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            float lo, hi;
                            split2(fma2(pair2(__uint_as_float(sc[x][c + e]), __uint_as_float(sc[x][c + e + 1])), by2, minus2), lo, hi);
                            lo = fast_exp2(lo);
                            hi = fast_exp2(hi);
                            const uint64_t p = pair2(lo, hi);
                            sums[e >> 1] = add2(sums[e >> 1], p);
                            split2(mul2(p, e ? pair2(vs.z, vs.w) : pair2(vs.x, vs.y)), lo, hi);
                            bigs[e >> 1] = max3(bigs[e >> 1], lo, hi);
                            sc[x][c + e] = __float_as_uint(lo);
                            sc[x][c + e + 1] = __float_as_uint(hi);
                        }
                    }
                if (mixed) {                               // 0 times a scale that is NaN (which no maximum takes up)
#pragma unroll
                    for (int x = 0; x < 2; x++)
#pragma unroll
                        for (int c = 0; c < 32; c++)
                            if (!((uint32_t)(sees >> (32 * x)) >> c & 1u)) sc[x][c] = 0u;
                }
                {
                    float lo, hi;
                    split2(add2(sums[0], sums[1]), lo, hi);
                    l = l * alpha + (lo + hi);
                }
                const float big = fmaxf(bigs[0], bigs[1]);
                float ratio = 1.f;
                if (grow || big > room) {
                    most = fmaxf(most * alpha, big);
                    const uint32_t e = top_exponent(__float_as_uint(most));
                    const float f = to_half_range(e);
                    ratio = alpha * inverse_power(to_half) * f;
                    to_half = f;
                    room = half_range_end(e);
                }
                const uint64_t half2 = pair2(to_half, to_half);
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    // P into the first 32 columns of its S
                    uint32_t pk[16];
#pragma unroll
                    for (int c = 0; c < 16; c++) {
                        float lo, hi;
                        split2(mul2(pair2(__uint_as_float(sc[x][2 * c]), __uint_as_float(sc[x][2 * c + 1])), half2), lo, hi);
                        pk[c] = pack2<__half>(lo, hi);
                    }
                    tc_st16(s_at + x * 16, pk);
                }
                if (begun && __any_sync(0xFFFFFFFFu, ratio != 1.f && there)) {
                    // Every product so far is in O (the one of tile n is not issued before p_full).  That
                    // the barrier is no more than one phase behind follows from S of tile n - 1, whose
                    // product waited for tile n - 3's P V.
                    if (!warp_wait(&sh.o_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, dead, a)) { tc_wait_st(); alive = false; break; }
                    tc_after();
#pragma unroll 1
                    for (uint32_t c0 = 0; c0 < (uint32_t)D; c0 += 32) {
                        uint32_t o[32];
                        tc_ld32(o, tmem + lane_base + O_COL + c0);
                        tc_wait_ld();
                        tc_pin32(o);
#pragma unroll
                        for (int c = 0; c < 32; c++) o[c] = __float_as_uint(__uint_as_float(o[c]) * ratio);
                        tc_st32(tmem + lane_base + O_COL + c0, o);
                    }
                }
                tc_wait_st();
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.p_full[n & 1u]);
            }
            // ---------------------------------------------------------- the piece's end
            if (alive) alive = warp_wait(&sh.o_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, dead, a);
            // both verdicts: the warps that fetch are four tiles ahead at most
            for (int kv = 0; alive && kv < 2; kv++)
                alive = warp_wait(&sh.judged[kv][piece % TC8_BITS_RING], (piece / TC8_BITS_RING) & 1u, dead, a);
            tc_after();
            // The four warps agree on how the piece ended: it is complete when each of them saw its last
            // product, whatever the other roles come to.  The verdict of the piece before, which all have read
            // by now, makes room.
            alive = !any_softmax(!alive);
            uint32_t bits = alive ? *(volatile uint32_t*)&sh.bits[piece % TC8_BITS_RING] : (uint32_t)GIFT_ST_STALLED;
            if (!alive && row == 0) w.note_stall(a);
            const bool odd = bits & FOUND_NAN;
            bits &= ~FOUND_NAN;
            if (row == 0) *(volatile uint32_t*)&sh.bits[(piece + TC8_BITS_RING - 1) % TC8_BITS_RING] = 0u;
            const bool whole = w.whole();
            const uint32_t slot = w.slot();
            const bool none = bits != 0u || l == 0.f;
            const float unit = inverse_power(to_half), inv = none ? 0.f : 1.f / l;
            if (warp_there) {
                // Rows leave by way of shared memory, 64 bytes of 32 rows at a time, so that four lanes write
                // a row's 64 bytes.
                char* mine = whole ? a.out + (uint64_t)(w.row0 + i) * a.out_row + (uint64_t)hq * a.out_head
                                   : reinterpret_cast<char*>(a.part_o + ((uint64_t)slot * TC8_ROWS + row) * D);
                const uint32_t last = w.all_q - w.qt * a.tile_rows < a.tile_rows ? w.all_q - w.qt * a.tile_rows : a.tile_rows;
                const uint32_t rows = last - warp * 32;                         // rows of this warp that exist, if below 32
#pragma unroll 1
                for (uint32_t c0 = 0; c0 < (uint32_t)D; c0 += 32) {
                    uint32_t o[32];
                    tc_ld32(o, tmem + lane_base + O_COL + c0);
                    tc_wait_ld();
                    tc_pin32(o);
#pragma unroll
                    for (int x = 0; x < 32; x++) o[x] = __float_as_uint(__uint_as_float(o[x]) * unit);
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 16; x++)
                            o[x] = none ? 0u : pack_out(a, __uint_as_float(o[2 * x]) * inv, __uint_as_float(o[2 * x + 1]) * inv);
                    }
                    const uint32_t parts = whole ? 1 : 2;                       // 32 columns are 64 or 128 bytes
#pragma unroll
                    for (uint32_t part = 0; part < 2; part++) {
                        if (part >= parts) break;
#pragma unroll
                        for (uint32_t x = 0; x < 4; x++)
                            *reinterpret_cast<uint4*>(stage_o + lane * 64 + ((x ^ ((lane >> 1) & 3u)) << 4)) =
                                make_uint4(o[part * 16 + 4 * x], o[part * 16 + 4 * x + 1], o[part * 16 + 4 * x + 2], o[part * 16 + 4 * x + 3]);
                        __syncwarp();
#pragma unroll
                        for (uint32_t y = 0; y < 4; y++) {
                            const uint32_t other = y * 8 + (lane >> 2), x = lane & 3u;
                            char* to = reinterpret_cast<char*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)mine, other));
                            const uint4 v = *reinterpret_cast<const uint4*>(stage_o + other * 64 + ((x ^ ((other >> 1) & 3u)) << 4));
                            if (other < rows) *reinterpret_cast<uint4*>(to + (whole ? c0 * 2 : c0 * 4 + part * 64) + x * 16) = v;
                        }
                        __syncwarp();
                    }
                }
                if (there) {
                    if (!whole) a.part_ml[(uint64_t)slot * TC8_ROWS + row] = make_float2(m, l);
                    else if (a.lse) a.lse[(uint64_t)(w.row0 + i) * a.heads + hq] = none ? NEG_INF : (m + log2f(l)) * 0.6931471805599453f;
                }
            }
            if (odd) put_nan_piece<D>(a, w, none);
            if (whole) {
                if (w.h == 0 && w.qt == 0) write_request<128>(a, w.r, w.row0, w.s.rows, bits);
            } else if (row == 0) {
                w.write_head(a, bits, slice);
            }
            tc_before();
            piece++;
        }
    }
    __syncthreads();
    if (warp == 6) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

}  // namespace gift
