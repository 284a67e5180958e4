// Attention over the labelled paged cache, many query rows per K/V head: tcgen05 products.
//
// A tile of 128 query rows (or what whole tokens fit) meets tiles of 64 tokens.  S = Q K^T (128 x 64,
// 32-bit) lands in tensor memory, one row per thread of four softmax warps; P, rounded to the pool's type, goes back
// into the tensor-memory columns of its S and is the A operand of O += P V, whose accumulator
// (128 x D) stays in tensor memory for the whole piece.  Roles, which meet on mbarriers alone:
//   warps 0-3  softmax: thread = query row; running maximum and sum in registers
//   warp 4     brings Q and the K tiles into swizzled shared memory, warp 5 the V tiles, by TMA.  What
//              is contiguous in a page is a run of tokens: the largest power of two, up to a tile,
//              that divides the page.  A run of 8 or more is one copy of 64 columns; shorter ones are
//              gathered, 4 tokens to a copy, which costs some 37 clocks of the SM's one TMA unit
//              however little it brings (32 requests of 8192 tokens, 8 K/V heads, 128 rows each: 204
//              us with pages of 16, 279 us with pages of 4).  Rows outside the map read as zeros:
//              that is where the runs past the context are sent.  Each of the two judges the
//              labels of the pages that it copies from: both look a page up for themselves, and a table
//              that is rewritten meanwhile must not give K of one page and V of another.
//   warp 6     one thread issues Q K^T: tile j + 1's runs while the softmax of tile j does.
//   warp 7     looks over the V tiles that hold step tokens (below), and one thread issues P V.  Two
//              issuers, because what one thread spends on a tile (waits, descriptors, commits) was
//              the longest part of the cycle.
// O is rescaled only when a row's maximum has grown by more than 2^8 over the one in use: p is then at
// most 2^8, which neither 16-bit type minds, and nearly all tiles leave O alone.
// 2 CTAs per SM share its tensor memory (256 of 512 columns each) and hide each other's waits.
//
// What bounds it: with one tile of query rows per K/V head, HBM (24 drafted tokens of 32 heads over
// contexts of 256 to 8192, 64 requests: 716 us, 6.3 TB/s; 32 requests as above: 204 us, 5.4 TB/s and 675
// TFLOP/s).  With several (48 requests, trees of 1 to 64, up to 16384 tokens, 8 of 32 heads) it takes 389 us at
// 1965 MHz, 3 000 clocks per tile and CTA, where the chain of a tile through softmax and products takes
// 1 900 with K/V in L2: the rest, waits for K and V among it, is not accounted for.  Under a long load the
// power cap takes the clock to 1390 MHz and the time to 464 us.  The
// whole kernel is written small: items of a few tiles meet its cold parts at every end, and
// fetching those past the instruction cache cost as much as the tiles (code of 105 KB: 505 us
// where 66 KB take 442, contexts of 64 to 1024 tokens 261 and 169 us).
// Eight softmax warps, two to a row's columns, were no faster (406 against 388 us).
//
// Every wait is bounded (gift_ctx_wait_limit).  A CTA whose wait runs out leaves the rest of its slice undone and
// notes which requests that concerns (part_stall): the joining kernel makes all their rows zero, those of
// other CTAs too, and their status GIFT_ST_STALLED.  It ends only when its own copies and products have: the warps that started them wait
// for the last of them, with a limit of their own.
#pragma once
#include "gift_tc.cuh"

namespace gift {

constexpr int TC_ROWS = 128;
constexpr int TC_TILE = 64;
constexpr int TC_THREADS = 256;
constexpr int TC_STAGES = 2;
// Pieces whose page verdicts are kept: warp 4 is at most three pieces ahead of the softmax (Q of the fourth
// waits for S of the third, that for P V of the first, that for the softmax), warp 5 at most two (its stages
// are freed by P V), and a verdict is cleared one piece after it was read.
constexpr int TC_BITS_RING = 8;

template <int D> struct TcSmem {
    static constexpr uint32_t q = 0;                                                  // [D/64][128][64]
    static constexpr uint32_t k = TC_ROWS * D * 2;                                    // [stage][D/64][64][64]
    static constexpr uint32_t v = k + TC_STAGES * TC_TILE * D * 2;
    static constexpr uint32_t o = v + TC_STAGES * TC_TILE * D * 2;                    // [4 warps][32 rows][64 bytes]
    static constexpr uint32_t bytes = o + 4 * 32 * 64;
};

struct TcShared {
    uint64_t k_full[TC_STAGES], k_empty[TC_STAGES], v_full[TC_STAGES], v_empty[TC_STAGES];
    uint64_t s_full[2], p_full[2], o_done[2], checked[2], q_full, q_empty, last;
    uint32_t tmem;
    uint32_t bits[TC_BITS_RING];
    int odd[2];                      // P V of the tile with step tokens in this stage is done by the softmax warps
    int dead;
    PlaceShared place;
};

using TcWalk = Walk<TC_TILE>;

// A role's walk lies in shared memory: its two dozen words are used at a piece's ends, and the softmax
// threads need every register in between (spills go through what little L1 the tiles leave, and made
// an item's end several times as long).
__device__ __noinline__ bool walk_next(TcWalk& w, const AttnArgs& a, uint32_t lane)
{
    TcWalk x = w;
    const bool more = x.next(a);
    __syncwarp();
    if (lane == 0) w = x;
    __syncwarp();
    return more;
}

template <class T, int D>
__global__ void __launch_bounds__(TC_THREADS, 2) attn_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map)
{
    constexpr uint32_t CH = D / 8;                         // 16-byte chunks of a row
    constexpr uint32_t TMEM_COLS = 256;                    // 2 S, O; a power of two, half of what an SM has
    constexpr uint32_t S_COL = 0, O_COL = 2 * TC_TILE;
    extern __shared__ __align__(1024) char smem[];
    __shared__ TcShared sh;
    __shared__ TcWalk walks[TC_THREADS / 32];
    using L = TcSmem<D>;

    join_may_start();
    if (threadIdx.x == 0) {
        a.part_head[blockIdx.x * 2u + 1u].pieces = 0u;
        a.part_stall[blockIdx.x] = make_uint4(0u, 0u, 0u, 0u);
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < TC_STAGES; i++) {
            bar_init(&sh.k_full[i], 1); bar_init(&sh.k_empty[i], 1);
            bar_init(&sh.v_full[i], 1); bar_init(&sh.v_empty[i], 1);
        }
        for (int i = 0; i < 2; i++) { bar_init(&sh.s_full[i], 1); bar_init(&sh.p_full[i], 4); bar_init(&sh.o_done[i], 1); bar_init(&sh.checked[i], 1); sh.odd[i] = 0; }
        bar_init(&sh.q_full, 1); bar_init(&sh.q_empty, 1); bar_init(&sh.last, 2);
        for (int i = 0; i < TC_BITS_RING; i++) sh.bits[i] = 0u;
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    uint64_t total, slice;
    // ends with a barrier for every thread, taken or not
    const bool some = place_unit<TC_THREADS>(a, blockIdx.x / a.ways, TC_TILE, blockIdx.x == 0, &sh.place, &total, &slice);
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
    TcWalk& w = walks[warp];
    {
        TcWalk x;
        x.start(a, sh.place.at, blockIdx.x % a.ways, units);
        if (lane == 0) w = x;
        __syncwarp();
    }

    if (warp == 4 || warp == 5) {
        // ------------------------------------------------------------------ copies
        // Lane l brings run l % runs of a tile (or gathers 4 tokens), columns 64 (l / runs) .. + 63.
        const uint32_t kv = warp - 4, runs = TC_TILE / (a.run > 4 ? a.run : 4), col = lane / runs, first = (lane & (runs - 1)) * (TC_TILE / runs);
        const bool active = col < D / 64, gather = a.run < 8;
        uint64_t* full = kv ? sh.v_full : sh.k_full;
        uint64_t* empty = kv ? sh.v_empty : sh.k_empty;
        uint32_t n = 0, piece = 0, q_loads = 0;            // tiles and pieces so far
        bool ok = true;
        while (ok && walk_next(w, a, lane)) {
            const int32_t owner = a.b.owner[w.r];
            const int32_t* table = a.b.table + (uint64_t)w.r * a.b.max_blocks;
            const int32_t x = (int32_t)((kv * a.kv_heads + w.h) * D + col * 64);
            uint32_t bits = w.masked_short(a) ? GIFT_ST_BAD_DESC : 0u;
            if (kv == 0) {
                // Q, once the products of the piece before have read the old rows.  What the box holds past
                // the request's rows is another request's: rows that nobody asks for.
                ok = piece == 0 || warp_wait(&sh.q_empty, (piece - 1) & 1u, dead, a);
                if (!ok) break;
                q_loads++;
                if (lane == 0) {
                    bar_expect(&sh.q_full, a.tile_rows * D * 2);
#pragma unroll
                    for (int c = 0; c < D / 64; c++)
                        copy_q(sm + L::q + c * (TC_ROWS * 128), &q_map, c * 64, (int32_t)(w.h * a.group),
                               (int32_t)(w.row0 + a.by_group.quot(w.qt * a.tile_rows)), &sh.q_full);
                }
            }
            // Where runs are copied, lane l looks up its run's first token; where tokens are gathered, tokens
            // l and l + 32.  Table entries are fetched a tile ahead, labels judged a tile later.
            int32_t next[2] = {-1, -1}, label[2] = {GIFT_OWNER_PARAM, GIFT_OWNER_PARAM};
            const uint32_t mine = gather ? lane : first;
#pragma unroll 1
            for (uint32_t j = 0; j <= w.n_tiles; j++) {
                int32_t slot[2], page[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    // the slots of tile j - 1, and the entries of tile j
                    const uint32_t t_next = (w.tb + j) * TC_TILE + mine + e * 32, t = t_next - TC_TILE;
                    const bool used = e == 0 || gather;
                    bits |= label_read_status(label[e], owner);
                    page[e] = -1;
                    if (j > 0 && used && t < w.s.want) {
                        page[e] = (uint32_t)next[e] < a.b.n_pages ? next[e] : -1;
                        if (page[e] < 0) bits |= GIFT_ST_BAD_DESC;
                    }
                    slot[e] = page[e] >= 0 ? (int32_t)((uint32_t)page[e] * a.b.page_tokens + (t - a.b.page.quot(t) * a.b.page_tokens)) : -(int32_t)TC_TILE;
                    next[e] = j < w.n_tiles && used && t_next < w.s.want ? table[a.b.page.quot(t_next)] : -1;
                    label[e] = a.owner_map && page[e] >= 0 ? a.owner_map[page[e]] : GIFT_OWNER_PARAM;
                }
                if (j == 0) continue;
                const uint32_t stage = n % TC_STAGES, round = n / TC_STAGES;
                ok = round == 0 || warp_wait(&empty[stage], (round - 1) & 1u, dead, a);
                if (!ok) break;
                const uint32_t dst = sm + (kv ? L::v : L::k) + stage * (TC_TILE * D * 2) + col * (TC_TILE * 128) + first * 128;
                if (gather) {
                    int32_t four[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int32_t lo = __shfl_sync(0xFFFFFFFFu, slot[0], (first + e) & 31u), hi = __shfl_sync(0xFFFFFFFFu, slot[1], (first + e) & 31u);
                        four[e] = first < 32 ? lo : hi;
                    }
                    if (active) gather4(dst, &map, x, four, &full[stage]);
                } else if (active) {
                    copy_run(dst, &map, x, slot[0], &full[stage]);
                }
                if (j == w.n_tiles) {
                    // this warp's verdict on the piece, before its last tile is announced
                    bits |= label_read_status(label[0], owner) | label_read_status(label[1], owner);
                    bits = __reduce_or_sync(0xFFFFFFFFu, bits);
                    if (lane == 0 && bits) atomicOr(&sh.bits[piece % TC_BITS_RING], bits);
                }
                __syncwarp();
                if (lane == 0) bar_expect(&full[stage], TC_TILE * D * 2);
                n++;
            }
            piece++;
        }
        // The copies under way end before the CTA does, whether or not anybody is left to wait for them: one of
        // the others may still give up after this warp has issued its last.
        for (uint32_t k = n > TC_STAGES ? n - TC_STAGES : 0; k < n; k++) bar_drain(&full[k % TC_STAGES], (k / TC_STAGES) & 1u);
        if (kv == 0 && q_loads > 0) bar_drain(&sh.q_full, (q_loads - 1) & 1u);
    } else if (warp == 6) {
        // ------------------------------------------------------------------ Q K^T
        // a negative scale: the products negate q, so that the scale used on the scores is positive
        const uint32_t id_s = instr_desc<T>(TC_ROWS, TC_TILE, 0) | (a.negate << 13);
        const uint64_t q_desc = smem_desc(sm + L::q, 16, 1024), k_desc = smem_desc(sm + L::k, 16, 1024);
        uint32_t n = 0, piece = 0;
        bool ok = true;
        while (ok && walk_next(w, a, lane)) {
            const uint32_t n_tiles = w.n_tiles;
            if (lane == 0) {
                ok = bar_wait(&sh.q_full, piece & 1u, dead, a);
#pragma unroll 1
                for (uint32_t j = 0; ok && j < n_tiles; j++) {
                    const uint32_t t = n + j, stage = t % TC_STAGES;
                    // S takes the columns that held P of tile t - 2
                    ok = bar_wait(&sh.k_full[stage], (t / TC_STAGES) & 1u, dead, a) &&
                         (t < 2 || bar_wait(&sh.o_done[t & 1u], ((t - 2) >> 1) & 1u, dead, a));
                    if (!ok) break;
                    tc_after();
                    const uint64_t kb = k_desc + stage * (TC_TILE * D * 2 / 16);
                    const uint32_t d = tmem + S_COL + (t & 1u) * TC_TILE;
#pragma unroll
                    for (uint32_t ks = 0; ks < D / 16; ks++)       // 16 columns are 32 bytes; 64 columns a block
                        mma_ss(d, q_desc + (ks >> 2) * (TC_ROWS * 128 / 16) + (ks & 3u) * 2,
                               kb + (ks >> 2) * (TC_TILE * 128 / 16) + (ks & 3u) * 2, id_s, ks > 0);
                    mma_commit(&sh.s_full[t & 1u]);
                    mma_commit(&sh.k_empty[stage]);
                    if (j + 1 == n_tiles) mma_commit(&sh.q_empty);
                }
            }
            ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
            n += n_tiles;
            piece++;
        }
        if (lane == 0) {
            // nothing may be in flight when the tensor memory is given back
            mma_commit(&sh.last);
            bar_drain(&sh.last, 0);
        }
        __syncwarp();
    } else if (warp == 7) {
        // ------------------------------------------------------------------ P V
        // What a hidden token's V holds must not reach a row, and 0 * inf is NaN: if a step token's V in a
        // tile is not finite, the softmax warps take the tile's product token by token, over what each
        // row sees.  Tokens of the cache are seen by every row.  The rows of a run that lie past the
        // context hold what the page held: they become zeros here.
        constexpr uint32_t id_o = instr_desc<T>(TC_ROWS, D, 1);
        const uint64_t v_desc = smem_desc(sm + L::v, TC_TILE * 128, 1024);
        uint32_t n = 0;
        bool ok = true;
        while (ok && walk_next(w, a, lane)) {
#pragma unroll 1
            for (uint32_t j = 0; j < w.n_tiles; j++, n++) {
                const uint32_t stage = n % TC_STAGES, t0 = (w.tb + j) * TC_TILE;
                ok = warp_wait(&sh.v_full[stage], (n / TC_STAGES) & 1u, dead, a);
                if (!ok) break;
                bool odd = false;
                if (t0 + TC_TILE > w.s.have) {
                    const uint32_t lo = w.s.have > t0 ? w.s.have - t0 : 0u;
                    const uint32_t hi = w.s.want - t0 < (uint32_t)TC_TILE ? w.s.want - t0 : (uint32_t)TC_TILE;
                    uint4* v = reinterpret_cast<uint4*>(smem + L::v + stage * (TC_TILE * D * 2));
#pragma unroll
                    for (uint32_t b = 0; b < (uint32_t)D / 64; b++) {
#pragma unroll 2
                        for (uint32_t x = lo * 8 + lane; x < hi * 8; x += 32) {
                            const uint4 q = v[b * (TC_TILE * 8) + x];
                            odd |= pair_not_finite<T>(q.x) || pair_not_finite<T>(q.y) || pair_not_finite<T>(q.z) || pair_not_finite<T>(q.w);
                        }
                        if (a.run >= 8)
#pragma unroll 1
                            for (uint32_t x = hi * 8 + lane; x < TC_TILE * 8; x += 32) v[b * (TC_TILE * 8) + x] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    odd = __any_sync(0xFFFFFFFFu, odd);
                    if (lane == 0) {
                        *(volatile int*)&sh.odd[stage] = odd ? 1 : 0;
                        bar_arrive(&sh.checked[stage]);
                    }
                    __syncwarp();
                }
                ok = warp_wait(&sh.p_full[n & 1u], (n >> 1) & 1u, dead, a);
                if (!ok) break;
                if (lane == 0) {
                    tc_after();
                    if (!odd) {
                        const uint64_t vb = v_desc + stage * (TC_TILE * D * 2 / 16);
                        const uint32_t p = tmem + S_COL + (n & 1u) * TC_TILE;
#pragma unroll
                        for (uint32_t ks = 0; ks < TC_TILE / 16; ks++)      // 16 tokens are 8 columns of P, 2048 bytes of V
                            mma_ts(tmem + O_COL, p + ks * 8, vb + ks * (2048 / 16), id_o, j > 0 || ks > 0);
                    }
                    mma_commit(&sh.o_done[n & 1u]);
                    mma_commit(&sh.v_empty[stage]);
                }
                __syncwarp();
            }
        }
        if (lane == 0) {
            mma_commit(&sh.last);
            bar_drain(&sh.last, 0);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ softmax
        const uint32_t row = threadIdx.x, lane_base = (warp * 32u) << 16;
        uint32_t n = 0, piece = 0;
        uint32_t checks0 = 0, checks1 = 0;                 // tiles with step tokens so far, per stage
        char* stage_o = smem + L::o + warp * (32 * 64);
        bool alive = true;
        while (walk_next(w, a, lane)) {
            const uint32_t rho = w.qt * a.tile_rows + row;
            const bool there = rho < w.all_q && row < a.tile_rows;
            const bool warp_there = w.qt * a.tile_rows + warp * 32 < w.all_q && warp * 32 < a.tile_rows;
            const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = w.h * a.group + (there ? rho - i * a.group : 0u);
            const bool masked_short = w.masked_short(a);
            float m = NEG_INF, l = 0.f;                    // the maximum in use, the sum relative to it
#pragma unroll 1
            for (uint32_t j = 0; alive && j < w.n_tiles; j++, n++) {
                const uint32_t s_at = tmem + lane_base + S_COL + (n & 1u) * TC_TILE;
                const uint32_t t0 = (w.tb + j) * TC_TILE;
                const bool mixed = t0 + TC_TILE > w.s.have;
                uint64_t sees = ~0ull;
                if (mixed) sees = there && !masked_short ? row_sees64(a, w.s.have, w.s.want, w.row0 + i, i, t0) : 0ull;
                if (!warp_wait(&sh.s_full[n & 1u], (n >> 1) & 1u, dead, a)) { alive = false; break; }
                bool odd = false;
                if (mixed) {
                    const uint32_t round = n & 1u ? checks1++ : checks0++;
                    if (!warp_wait(&sh.checked[n & 1u], round & 1u, dead, a)) { alive = false; break; }
                    odd = *(volatile int*)&sh.odd[n & 1u] != 0;
                }
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
                if (mixed) {
#pragma unroll
                    for (int x = 0; x < 2; x++)
#pragma unroll
                        for (int c = 0; c < 32; c++)
                            if (!((uint32_t)(sees >> (32 * x)) >> c & 1u)) sc[x][c] = 0xFF800000u;      // minus infinity
                }
                // Three inputs to a maximum, two elements to an FMA or a sum (short contexts 170 -> 148 us; half of
                // the exponentials as polynomials on the FMA pipe instead: 402 -> 459 us).
                float tops[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int c = 0; c < 32; c += 2)
                        tops[(c >> 1) & 3] = max3(tops[(c >> 1) & 3], __uint_as_float(sc[x][c]), __uint_as_float(sc[x][c + 1]));
                // the scale is positive here (q's sign carries it), so the largest score stays the largest
                const float top = max3(tops[0], tops[1], fmaxf(tops[2], tops[3])) * a.scale_log2;
                const bool grow = top > m + 8.f;           // also when nothing has been seen yet
                float alpha = 1.f;
                if (grow) {
                    alpha = fast_exp2(m - top);            // 0 from minus infinity
                    m = top;
                }
                const float minus = m == NEG_INF ? 0.f : -m;
                const uint64_t scale2 = pair2(a.scale_log2, a.scale_log2), minus2 = pair2(minus, minus);
                uint64_t sums[2] = {0ull, 0ull};
#pragma unroll
                for (int x = 0; x < 2; x++) {
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        float lo, hi;
                        split2(fma2(pair2(__uint_as_float(sc[x][c]), __uint_as_float(sc[x][c + 1])), scale2, minus2), lo, hi);
                        lo = fast_exp2(lo);
                        hi = fast_exp2(hi);
                        sc[x][c] = __float_as_uint(lo);
                        sc[x][c + 1] = __float_as_uint(hi);
                        sums[(c >> 1) & 1] = add2(sums[(c >> 1) & 1], pair2(lo, hi));
                    }
                    if (!odd) {
                        // P into the first 32 columns of its S
                        uint32_t pk[16];
#pragma unroll
                        for (int c = 0; c < 16; c++) pk[c] = pack2<T>(__uint_as_float(sc[x][2 * c]), __uint_as_float(sc[x][2 * c + 1]));
                        tc_st16(s_at + x * 16, pk);
                    }
                }
                {
                    float lo, hi;
                    split2(add2(sums[0], sums[1]), lo, hi);
                    l = l * alpha + (lo + hi);
                }
                const bool rescale = j > 0 && __any_sync(0xFFFFFFFFu, grow && there);
                if ((rescale || odd) && n > 0) {
                    // Every product so far is in O (the one of tile n is not issued before p_full).  That
                    // the barrier is no more than one phase behind follows from S of tile n - 1, whose
                    // product waited for tile n - 3's P V.
                    if (!warp_wait(&sh.o_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, dead, a)) { tc_wait_st(); alive = false; break; }
                    tc_after();
                }
                if (odd) {
                    // p, in 32 bits, into the columns of its S; then column by column (rare: registers matter more)
                    tc_st32(s_at, sc[0]);
                    tc_st32(s_at + 32, sc[1]);
                    tc_wait_st();
#pragma unroll 1
                    for (uint32_t ch = 0; ch < CH; ch++) {
                        uint32_t o[8];
                        tc_ld8(o, tmem + lane_base + O_COL + ch * 8);
                        tc_wait_ld();
                        tc_pin8(o);
#pragma unroll
                        for (int e = 0; e < 8; e++) o[e] = j > 0 ? __float_as_uint(__uint_as_float(o[e]) * alpha) : 0u;
                        const char* v = smem + L::v + (n % TC_STAGES) * (TC_TILE * D * 2) + (ch >> 3) * (TC_TILE * 128);
#pragma unroll 1
                        for (uint32_t t = 0; t < 64; t++) {
                            const uint4 q = *reinterpret_cast<const uint4*>(v + t * 128 + (((ch & 7u) ^ (t & 7u)) << 4));
                            const uint32_t pair[4] = {q.x, q.y, q.z, q.w};
                            const float p = __uint_as_float(tc_ld1(s_at + t));
                            const bool seen = sees >> t & 1ull;
#pragma unroll
                            for (int y = 0; y < 8; y++) {
                                const T* e = reinterpret_cast<const T*>(&pair[y >> 1]);
                                if (seen) o[y] = __float_as_uint(__uint_as_float(o[y]) + p * to_float<T>(e[y & 1]));
                            }
                            __syncwarp();
                        }
                        tc_st8(tmem + lane_base + O_COL + ch * 8, o);
                    }
                } else if (rescale) {
#pragma unroll 1
                    for (uint32_t c0 = 0; c0 < (uint32_t)D; c0 += 32) {
                        uint32_t o[32];
                        tc_ld32(o, tmem + lane_base + O_COL + c0);
                        tc_wait_ld();
                        tc_pin32(o);
#pragma unroll
                        for (int c = 0; c < 32; c++) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
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
            tc_after();
            // The four warps agree on how the piece ended: it is complete when each of them saw its last
            // product, whatever the other roles come to.  The verdict of the piece before, which all have read
            // by now, makes room.
            alive = !any_softmax(!alive);
            const uint32_t bits = alive ? *(volatile uint32_t*)&sh.bits[piece % TC_BITS_RING] : (uint32_t)GIFT_ST_STALLED;
            if (!alive && row == 0) w.note_stall(a);
            if (row == 0) *(volatile uint32_t*)&sh.bits[(piece + TC_BITS_RING - 1) % TC_BITS_RING] = 0u;
            const bool whole = w.whole();
            const uint32_t slot = w.slot();
            const bool none = bits != 0u || l == 0.f;
            const float inv = none ? 0.f : 1.f / l;
            if (warp_there) {
                // Rows leave by way of shared memory, 64 bytes of 32 rows at a time, so that four lanes write
                // a row's 64 bytes (a lane writing its own row: 5 000 clocks, most of an item's end).
                char* mine = whole ? a.out + (uint64_t)(w.row0 + i) * a.out_row + (uint64_t)hq * a.out_head
                                   : reinterpret_cast<char*>(a.part_o + ((uint64_t)slot * TC_ROWS + row) * D);
                const uint32_t last = w.all_q - w.qt * a.tile_rows < a.tile_rows ? w.all_q - w.qt * a.tile_rows : a.tile_rows;
                const uint32_t rows = last - warp * 32;                         // rows of this warp that exist, if below 32
#pragma unroll 1
                for (uint32_t c0 = 0; c0 < (uint32_t)D; c0 += 32) {
                    uint32_t o[32];
                    tc_ld32(o, tmem + lane_base + O_COL + c0);
                    tc_wait_ld();
                    tc_pin32(o);
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 16; x++)
                            o[x] = none ? 0u : pack2<T>(__uint_as_float(o[2 * x]) * inv, __uint_as_float(o[2 * x + 1]) * inv);
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
                    if (!whole) a.part_ml[(uint64_t)slot * TC_ROWS + row] = make_float2(m, l);
                    else if (a.lse) a.lse[(uint64_t)(w.row0 + i) * a.heads + hq] = none ? NEG_INF : (m + log2f(l)) * 0.6931471805599453f;
                }
            }
            if (whole) {
                if (w.h == 0 && w.qt == 0) write_request<128>(a, w.r, w.row0, w.it.rows_m, bits);
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
