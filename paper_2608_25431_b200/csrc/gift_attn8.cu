// Attention of a step's rows over labelled pages of 8 bits.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "gift_attn8.cuh"
#include "gift_attn8_tc.cuh"
#include "gift_attn_join.cuh"
#include "gift_internal.cuh"

using namespace gift;

namespace {

// ---------------------------------------------------------------------------
// few query rows per K/V head: warp-level products
// ---------------------------------------------------------------------------
//
// The split is that of the 16-bit kernel: every warp works on its own tokens of a tile, with a ring of stages that only it
// fills and reads, 4 KiB of codes a step.  Codes become fp16 numbers (exact) between shared
// memory and the matrix instructions, and those conversions are most of the work: half the bytes of a 16-bit cache in
// the time of HBM leave a warp 180 clocks of its SM for a step.  So the products are turned: K and V are the operands of 16
// rows, the query rows the operand of 8, S^T = K Q^T and O^T = V^T P^T.  With up to 8 query rows that is half the
// products, and half the registers: 16 warps per SM instead of 8.
//   K   A product's order of the 128 dimensions is free, so a lane takes 16 neighbouring codes of a token with one load, and
//       Q's fragments are laid out to match.
//   V   Loading 8 x 8 pairs of codes transposed gives a lane two neighbouring dimensions of two neighbouring
//       tokens; a byte permutation makes of it the fragments of an even and an odd dimension.
// K's scale multiplies the score, V's the weight, both in 32 bits: nothing but q and the weights is
// rounded.  Both go to fp16 by a power of two of the row's own (see top_exponent), for scales and queries of
// any size.  The maximum that weights are relative to, and the weights' power of two, change only when a score passes
// the maximum by 2^6 or a weight leaves fp16: one vote a step in place of reductions over the warp.
// Measured: a decode step of 64 requests, 32 heads, 122 us, 5.1 TB/s, 78 % of a copy; 16 requests of up to 32 768 tokens, 4 query heads to
// one, 126 us; capped, biased, under a window of 1 024, 52 us; trees of 16 rows 594 us, 3.9 TB/s (with heads of 128 such items want more than
// the 168 registers that 3 CTAs leave: 116 to 156 bytes a thread lie in local memory).  With up to 8 rows the
// chain of a step bounds it (52 % of the issue slots, 16 warps on an SM), with 16 the same with twice the products.

constexpr int FEW8_STAGES = 3;
// Items of a call before heads share a CTA.  1, 8, 16, 32, 64, 128: 16 requests with long contexts 131, 131, 131, 126, 146, 171 us; one
// request of 514 tokens 33, 19, 14.2, 13.8, 13.8, 13.8 us.
constexpr uint32_t FEW8_ITEMS = 32;
constexpr float FEW8_SLACK = 6.f;        // how far, in powers of two, a score may pass the maximum in use

template <int D, int NR> struct Few8 {
    static constexpr int warps = NR == 1 ? 8 : 4;                        // 2 CTAs per SM with 128 registers a thread, or
    static constexpr int ctas = NR == 1 ? 2 : 3;                         // 3 with 168
    static constexpr int threads = warps * 32;
    static constexpr int rows = 8 * NR;
    static constexpr int half = 2048;                                    // bytes of K's (or V's) codes of a step
    static constexpr int tok = half / D;                                 // tokens of a warp's step
    static constexpr int ring = warps * FEW8_STAGES * 2 * half;          // codes of K, of V; behind them the scales, those
    static constexpr int scales = tok * 16;                              // of a pair of heads for each token
    static constexpr int join = warps * rows * D * 4;
    static constexpr int smem = ring + warps * FEW8_STAGES * scales;
    static_assert(join <= smem, "the warps' parts lie in the ring");
    // Where 16-byte chunk `chunk` of a token lies: permuted by the copies' 128- or 64-byte swizzle, so that lanes that
    // load together (K: every other chunk of 2 tokens; V: a chunk of 8 tokens) meet different banks.
    static __device__ __forceinline__ uint32_t at(uint32_t token, uint32_t chunk)
    {
        return token * D + ((chunk ^ (D == 128 ? token & 7u : (token >> 1) & 3u)) << 4);
    }
};

// An 8 x 8 matrix of 16-bit elements, two of a row in each lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Eight of a finished row's columns, from 8 ch; and with the first of them its lse.
__device__ __forceinline__ void put_row(const Attn8Args& a, uint32_t row0, uint32_t h, uint32_t rho, uint32_t ch, const float (&acc)[8],
                                        float top, float sum, uint32_t bits)
{
    const uint32_t i = a.by_group.quot(rho), hq = h * a.group + (rho - i * a.group);
    const bool none = bits != 0u || sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (!none) {
        v.x = pack_out(a, acc[0] * inv, acc[1] * inv); v.y = pack_out(a, acc[2] * inv, acc[3] * inv);
        v.z = pack_out(a, acc[4] * inv, acc[5] * inv); v.w = pack_out(a, acc[6] * inv, acc[7] * inv);
    }
    *reinterpret_cast<uint4*>(a.out + (uint64_t)(row0 + i) * a.out_row + (uint64_t)hq * a.out_head + ch * 16) = v;
    if (a.lse && ch == 0) a.lse[(uint64_t)(row0 + i) * a.heads + hq] = none ? NEG_INF : (top + log2f(sum)) * 0.6931471805599453f;
}

// The pieces of a cut item, for all heads of its group, joined in their order: pieces w, w + 1, ... (the first is its slice's last
// piece, the others their slices' first ones), written while this kernel runs and read past L1.  bits: 0 when called.
template <int D, int ROWS, int THREADS>
__device__ __noinline__ void join8(const Attn8Args& a, const PartHead& head, uint32_t w, float2* tops, uint32_t* bits)
{
    constexpr uint32_t CH = D / 8;
    const uint32_t pieces = head.pieces;
    auto part_of = [&](uint32_t p, uint32_t hr) -> uint64_t { return (uint64_t)(2u * (w + p) + (p == 0 ? 1u : 0u)) * a.head_ways * ROWS + hr; };
    for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
        const uint32_t b = __ldcg(&a.part_head[2u * (w + p) + (p == 0 ? 1u : 0u)].bits);
        if (b) atomicOr(bits, b);
    }
    // maxima and sums: 8 threads per row, pieces dealt among them
    for (uint32_t hr0 = 0; hr0 < a.head_ways * ROWS; hr0 += THREADS / 8) {
        const uint32_t hr = hr0 + (threadIdx.x >> 3);
        const bool there = hr < a.head_ways * ROWS && hr % ROWS < head.nr;
        float top = NOTHING, sum = 0.f;
        if (there)
            for (uint32_t p = threadIdx.x & 7u; p < pieces; p += 8) {
                const float2 ml = __ldcg(&a.part_ml[part_of(p, hr)]);
                const float now = fmaxf(top, ml.x);
                sum = sum * fast_exp2(top - now) + ml.y * fast_exp2(ml.x - now);
                top = now;
            }
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) {
            const float other_top = __shfl_xor_sync(0xFFFFFFFFu, top, d), other_sum = __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            const float now = fmaxf(top, other_top);
            sum = sum * fast_exp2(top - now) + other_sum * fast_exp2(other_top - now);
            top = now;
        }
        if (there && (threadIdx.x & 7u) == 0) tops[hr] = make_float2(top, sum);
    }
    __syncthreads();
    for (uint32_t x = threadIdx.x; x < a.head_ways * ROWS * CH; x += THREADS) {
        const uint32_t ch = x % CH, hr = x / CH, row = hr % ROWS;
        if (row >= head.nr) continue;
        const float top = tops[hr].x;
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; e++) acc[e] = 0.f;
#pragma unroll 4
        for (uint32_t p = 0; p < pieces; p++) {
            const uint64_t part = part_of(p, hr);
            const float f = fast_exp2(__ldcg(&a.part_ml[part]).x - top);
            const float4* from = reinterpret_cast<const float4*>(a.part_o + part * D + ch * 8);
            const float4 u = __ldcg(from), v = __ldcg(from + 1);
            acc[0] += f * u.x; acc[1] += f * u.y; acc[2] += f * u.z; acc[3] += f * u.w;
            acc[4] += f * v.x; acc[5] += f * v.y; acc[6] += f * v.z; acc[7] += f * v.w;
        }
        put_row(a, head.row0, head.h * a.head_ways + hr / ROWS, head.q0 + row, ch, acc, top, tops[hr].y, *bits);
    }
    if (head.h == 0 && head.q0 == 0) write_request<THREADS>(a, head.r, head.row0, head.rows_m, *bits);
}

// A warp's part of a piece, as it lies in shared memory: its rows' NaN, from its tokens of the piece.
template <int D, int NR>
__device__ __noinline__ void put_nan_part(const Attn8Args& a, uint32_t r, uint32_t row0, uint32_t group_of_heads, uint32_t qt, uint32_t tb, uint32_t n_tiles,
                                          float* parts)
{
    using L = Few8<D, NR>;
    __syncwarp();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const ReqShape s = load_shape(a.b, r);
    const uint32_t rho = qt * L::rows + lane, i = a.by_group.quot(rho);                // each lane has a row
    tb += first_seen(a, s.have) / a.tile_tokens;
#pragma unroll 1
    for (uint32_t k = 0; k < n_tiles; k++)
        put_nan<D>(a, r, group_of_heads * a.head_ways + (warp & (a.head_ways - 1u)), s.have, s.want, row0 + i, i,
                   (tb + k) * a.tile_tokens + warp / a.head_ways * L::tok, L::tok, lane < (uint32_t)L::rows && rho < s.rows * a.group,
                   parts + (warp * L::rows + lane) * D);
}

// NEAR: capped scores, a bias by distance or a window.  NR: query rows of an item by 8.
template <int D, int NR, bool NEAR>
__global__ void __launch_bounds__(Few8<D, NR>::threads, Few8<D, NR>::ctas) attn8_few_kernel(const __grid_constant__ Attn8Args a)
{
    using L = Few8<D, NR>;
    constexpr int ROWS = L::rows, TOK = L::tok, MT = TOK / 16, THREADS = L::threads;
    constexpr int CH = D / 8;                      // 16-byte chunks of a result's row
    constexpr int KCH = D / 16;                    // 16-byte chunks of a token's codes
    extern __shared__ __align__(1024) char smem[];
    __shared__ PlaceShared place;
    __shared__ float2 s_ml[L::warps][ROWS];
    __shared__ uint32_t s_bits, s_last, s_first;
    __shared__ float2 s_top[L::warps * ROWS];
    __shared__ PartHead s_head;

    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t total, slice;
    if (!place_unit<THREADS, NEAR>(a, blockIdx.x, a.tile_tokens, blockIdx.x == 0, &place, &total, &slice)) {
        leave_tickets(a);
        return;
    }
    const uint32_t ring = smem_u32(smem) + warp * (FEW8_STAGES * 2 * L::half);
    const uint32_t scale_ring = smem_u32(smem) + L::ring + warp * (FEW8_STAGES * L::scales);
    uint32_t put = 0, get = 0;                     // stage to fill, to read

    // this warp's head of a group, its tokens of a tile
    const uint32_t head_way = warp & (a.head_ways - 1u), first_token = warp / a.head_ways * TOK;
    Walk<0, NEAR> w;
    const uint64_t begin = slice * blockIdx.x, units = slice < total - begin ? slice : total - begin;
    w.start(a, place.at, 0, units);
    while (w.next(a)) {
        const ReqShape& s = w.s;
        const ItemShape& it = w.it;
        const uint32_t r = w.r, row0 = w.row0, tb = w.tb + (NEAR ? it.first : 0u), n_tiles = w.n_tiles, h = w.h * a.head_ways + head_way;
        const uint32_t all_q = it.rows_m * a.group;                // query rows of the K/V head
        const uint32_t q0 = w.qt * ROWS;
        const int32_t owner = a.b.owner[r];
        const int32_t* table = a.b.table + (uint64_t)r * a.b.max_blocks;
        const bool masked_short = w.masked_short(a);
        const uint32_t low = NEAR ? first_seen(a, s.have) : 0u;    // tokens before it are nobody's to see
        uint32_t bits = masked_short ? GIFT_ST_BAD_DESC : 0u;

        // Fragments of query rows g (+ 8); this lane's dimensions are 16 from 16 (c D / 64 + i).  Scores, weights and results
        // are those of query rows 2 c, 2 c + 1 (+ 8).
        const uint32_t g = lane >> 2, c = lane & 3u;
        uint32_t qf[NR][D / 16][2];
        float qs[NR][2], slope[NR][2];
        uint32_t row_i[NR][2];
#pragma unroll
        for (int n = 0; n < NR; n++) {
            const uint32_t rho = q0 + n * 8 + g;
            const bool there = rho < all_q;
            const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = h * a.group + (there ? rho - i * a.group : 0u);
            const uint4* q = reinterpret_cast<const uint4*>(a.q + (uint64_t)(row0 + i) * a.q_row + (uint64_t)hq * a.q_head);
            uint32_t x[D / 8];
#pragma unroll
            for (int y = 0; y < D / 32; y++) {
                const uint4 v = there ? q[c * (D / 32) + y] : make_uint4(0u, 0u, 0u, 0u);
                x[4 * y] = v.x; x[4 * y + 1] = v.y; x[4 * y + 2] = v.z; x[4 * y + 3] = v.w;
            }
            float scale = NEAR && a.cap_out != 0.f ? a.cap_in : a.scale_log2;
            if (!a.half) {
                uint32_t top = 0u;
#pragma unroll
                for (int y = 0; y < D / 8; y++) top = max(top, max(x[y] << 16 & 0x7FFFFFFFu, x[y] & 0x7FFF0000u));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const uint32_t e = top_exponent(top);
                const float f = to_half_range(e);
                scale *= from_half_range(e);
#pragma unroll
                for (int y = 0; y < D / 8; y++)
                    x[y] = pack2<__half>(__uint_as_float(x[y] << 16) * f, __uint_as_float(x[y] & 0xFFFF0000u) * f);
            }
#pragma unroll
            for (int ks = 0; ks < D / 16; ks++) {
                qf[n][ks][0] = x[2 * ks];
                qf[n][ks][1] = x[2 * ks + 1];
            }
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const uint32_t rho_j = q0 + n * 8 + 2 * c + j;
                const bool there_j = rho_j < all_q;
                row_i[n][j] = there_j ? a.by_group.quot(rho_j) : 0u;
                qs[n][j] = __shfl_sync(0xFFFFFFFFu, scale, (2 * c + j) * 4);
                slope[n][j] = NEAR && a.slopes && there_j ? a.slopes[h * a.group + rho_j - row_i[n][j] * a.group] * LOG2_E : 0.f;
            }
        }
        float o[D / 16][NR][4];
        float m[NR][2], l[NR][2];                                  // the maximum in use, the sum relative to it
        float most[NR][2];                                         // the weight that their power of two goes by:
        float to_half[NR][2], room[NR][2];                         // the factor, and the weight that it serves at most
#pragma unroll
        for (int n = 0; n < NR; n++) {
#pragma unroll
            for (int j = 0; j < 2; j++) { m[n][j] = NOTHING; l[n][j] = most[n][j] = 0.f; to_half[n][j] = to_half_range(9u); room[n][j] = half_range_end(9u); }
#pragma unroll
            for (int x = 0; x < D / 16; x++)
#pragma unroll
                for (int e = 0; e < 4; e++) o[x][n][e] = 0.f;
        }

        // Lane x looks after token x % TOK of the warp's: its table entry is fetched one step ahead of
        // the copies that need it, its label judged one step after it was asked for.
        const uint32_t my = lane % TOK, chunk = lane % KCH;
        const char* head = a.pages + (uint64_t)h * D + chunk * 16;
        const uint32_t row_bytes = (lane / KCH) * (uint32_t)a.token_bytes, rows_bytes = (32 / KCH) * (uint32_t)a.token_bytes;
        // a token's entry, if any row may see it
        auto entry = [&](uint32_t step) -> int32_t {
            const uint32_t t = (tb + step) * a.tile_tokens + first_token + my;
            return step < n_tiles && t < s.want && (!NEAR || t >= low) ? table[a.b.page.quot(t)] : -1;
        };
        int32_t next = entry(0), label = GIFT_OWNER_PARAM;
        auto issue = [&](uint32_t step) {
            if (step < n_tiles) {
                const uint32_t base = ring + put * (2 * L::half), scales = scale_ring + put * L::scales + (h & 1u) * 8u;
                const uint32_t t0 = (tb + step) * a.tile_tokens + first_token, t = t0 + my;
                const int32_t page = next;
                next = entry(step + 1);
                bits |= label_read_status(label, owner);
                label = GIFT_OWNER_PARAM;
                // the token's slot; tokens that nobody sees are filled with zeros: what memory holds there does not matter
                uint32_t slot = 0xFFFFFFFFu;
                if (t < s.want && (!NEAR || t >= low)) {
                    if ((uint32_t)page < a.b.n_pages) {
                        slot = (uint32_t)page * a.b.page_tokens + (t - a.b.page.quot(t) * a.b.page_tokens);
                        if (a.owner_map) label = a.owner_map[page];
                    } else {
                        bits |= GIFT_ST_BAD_DESC;
                    }
                }
                if (a.whole_steps && __all_sync(0xFFFFFFFFu, slot != 0xFFFFFFFFu)) {
                    // the step lies in one page: its tokens follow one another
                    const char* p = a.pages + (uint64_t)slot * a.token_bytes;
                    if (TOK == 32 || lane < TOK) cp_async8(scales + my * 16u, p + 2u * a.codes + h * 8u, 8u);
                    p = head + (uint64_t)(slot - my) * a.token_bytes + row_bytes;
#pragma unroll
                    for (int i = 0; i < KCH * TOK / 32; i++) {
                        cp_async16(base + L::at(i * (32 / KCH) + lane / KCH, chunk), p, 16u);
                        cp_async16(base + L::half + L::at(i * (32 / KCH) + lane / KCH, chunk), p + a.codes, 16u);
                        p += rows_bytes;
                    }
                } else {
                    if (TOK == 32 || lane < TOK) {
                        const bool there = slot != 0xFFFFFFFFu;
                        cp_async8(scales + my * 16u, a.pages + (there ? slot * a.token_bytes + 2ull * a.codes + h * 8u : 0ull), there ? 8u : 0u);
                    }
#pragma unroll
                    for (int i = 0; i < KCH * TOK / 32; i++) {
                        const uint32_t row = i * (32 / KCH) + lane / KCH;
                        const uint32_t from = __shfl_sync(0xFFFFFFFFu, slot, row);
                        const bool there = from != 0xFFFFFFFFu;
                        const char* p = there ? head + from * a.token_bytes : head;
                        cp_async16(base + L::at(row, chunk), p, there ? 16u : 0u);
                        cp_async16(base + L::half + L::at(row, chunk), p + a.codes, there ? 16u : 0u);
                    }
                }
                put = put == FEW8_STAGES - 1 ? 0u : put + 1u;
            }
            cp_commit();
        };
        // the first rounds only fill the ring (one copy of the code: it is large, and short items meet it cold)
#pragma unroll 1
        for (uint32_t round = 0; round < n_tiles + FEW8_STAGES - 1; round++) {
            issue(round);
            if (round < (uint32_t)FEW8_STAGES - 1) continue;
            const uint32_t step = round - (FEW8_STAGES - 1);
            cp_wait<FEW8_STAGES - 1>();
            __syncwarp();
            const uint32_t base = ring + get * (2 * L::half), scales = scale_ring + get * L::scales + (h & 1u) * 8u;
            const uint32_t t0 = (tb + step) * a.tile_tokens + first_token;
            // some rows may not see some of these tokens
            const bool mixed = t0 + TOK > s.have || (NEAR && a.window && t0 + a.window < s.want);
            if (mixed) {
                // 0 * NaN is NaN: codes of NaN in V, hidden from some row perhaps, become 0, and the rows that see them get
                // their NaN at the piece's end
                bool odd = false;
#pragma unroll
                for (int i = 0; i < L::half / 512; i++) {
                    const uint4 x = lds128(base + L::half + (i * 32 + lane) * 16);
                    odd |= codes_nan(x.x) || codes_nan(x.y) || codes_nan(x.z) || codes_nan(x.w);
                }
                if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll 1
                    for (int i = 0; i < L::half / 128; i++) {
                        const uint32_t at = (i * 32 + lane) * 4;
                        uint32_t x;
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(base + L::half + at) : "memory");
                        if (codes_nan(x)) {
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + L::half + at), "r"(codes_without_nan(x)) : "memory");
                            bits |= FOUND_NAN;
                        }
                    }
                    __syncwarp();
                }
            }
            float sc[MT][NR][4], vs[MT][2], away[NR][2];
            if (NEAR)
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int j = 0; j < 2; j++) away[n][j] = (float)((int32_t)(t0 + g) - (int32_t)(s.have + row_i[n][j]));
#pragma unroll
            for (int x = 0; x < MT; x++) {
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) sc[x][n][e] = 0.f;
#pragma unroll
                for (int i = 0; i < D / 64; i++) {
                    const uint4 k0 = lds128(base + L::at(x * 16 + g, c * (D / 64) + i)), k1 = lds128(base + L::at(x * 16 + 8 + g, c * (D / 64) + i));
                    const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
                    for (int y = 0; y < 4; y++) {
                        uint32_t f[4];
                        four_codes(w0[y], f[0], f[2]);
                        four_codes(w1[y], f[1], f[3]);
#pragma unroll
                        for (int n = 0; n < NR; n++) mma16816<__half>(sc[x][n], f, qf[n][i * 4 + y][0], qf[n][i * 4 + y][1]);
                    }
                }
#pragma unroll
                for (int e2 = 0; e2 < 2; e2++) {
                    const float2 ks_vs = lds_pair(scales + (x * 16 + e2 * 8 + g) * 16u);
                    vs[x][e2] = ks_vs.y;
#pragma unroll
                    for (int n = 0; n < NR; n++)
#pragma unroll
                        for (int j = 0; j < 2; j++) {
                            float& y = sc[x][n][2 * e2 + j];
                            y *= ks_vs.x * qs[n][j];
                        }
                }
            }
            if constexpr (NEAR) {
                if (a.cap_out != 0.f) {
                    float far = 0.f;
#pragma unroll
                    for (int x = 0; x < MT; x++)
#pragma unroll
                        for (int n = 0; n < NR; n++)
#pragma unroll
                            for (int e = 0; e < 4; e += 2) far = max3(far, fabsf(sc[x][n][e]), fabsf(sc[x][n][e + 1]));
                    if (__any_sync(0xFFFFFFFFu, !(far <= TANH_NEAR))) {
#pragma unroll
                        for (int x = 0; x < MT; x++)
#pragma unroll
                            for (int n = 0; n < NR; n++)
#pragma unroll
                                for (int e = 0; e < 4; e++) sc[x][n][e] = capped(sc[x][n][e], a.cap_out);
                    } else {
                        const uint64_t cap2 = pair2(a.cap_out, a.cap_out);
#pragma unroll
                        for (int x = 0; x < MT; x++)
#pragma unroll
                            for (int n = 0; n < NR; n++)
#pragma unroll
                                for (int e = 0; e < 4; e += 2) split2(capped_near(pair2(sc[x][n][e], sc[x][n][e + 1]), cap2), sc[x][n][e], sc[x][n][e + 1]);
                    }
                }
                if (a.slopes)
#pragma unroll
                    for (int x = 0; x < MT; x++)
#pragma unroll
                        for (int n = 0; n < NR; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) sc[x][n][e] += slope[n][e & 1] * (away[n][e & 1] + (float)(x * 16 + (e >> 1) * 8));
            }
            uint32_t sees[NR][2];                      // of the step's tokens, by row: bit x is token x * 8 + g
            if (mixed) {
                const bool none = masked_short || t0 >= s.want;
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        uint32_t all = none ? 0u : (uint32_t)row_sees64(a, s.have, s.want, row0 + row_i[n][j], row_i[n][j], t0);
                        if (NEAR && a.window) all &= (uint32_t)in_window64(a.window, s.have + row_i[n][j], t0);
                        sees[n][j] = all >> g;
#pragma unroll
                        for (int x = 0; x < 2 * MT; x++)
                            if (!(sees[n][j] >> (x * 8) & 1u)) sc[x >> 1][n][2 * (x & 1) + j] = NEG_INF;
                    }
            }
            float alpha[NR][2];
            bool grow = false;
            float top[NR][2];
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    top[n][j] = fmaxf(sc[0][n][j], sc[0][n][2 + j]);
#pragma unroll
                    for (int x = 1; x < MT; x++) top[n][j] = fmaxf(top[n][j], fmaxf(sc[x][n][j], sc[x][n][2 + j]));
                    grow |= top[n][j] > m[n][j] + FEW8_SLACK;          // also when nothing has been seen yet
                    alpha[n][j] = 1.f;
                }
            grow = __any_sync(0xFFFFFFFFu, grow);
            if (grow) {
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top[n][j] = fmaxf(top[n][j], __shfl_xor_sync(0xFFFFFFFFu, top[n][j], d));
                        const float now = top[n][j] > m[n][j] + FEW8_SLACK ? top[n][j] : m[n][j];      // each row by its own
                        alpha[n][j] = fast_exp2(m[n][j] - now);
                        m[n][j] = now;
                        l[n][j] *= alpha[n][j];
                    }
            }
            bool out = grow;
            float big[NR][2];
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    big[n][j] = 0.f;
#pragma unroll
                    for (int x = 0; x < 2 * MT; x++) {
                        float& y = sc[x >> 1][n][2 * (x & 1) + j];
                        const float p = fast_exp2(y - m[n][j]);
                        l[n][j] += p;
                        y = p * vs[x >> 1][x & 1];
                        if (mixed && !(sees[n][j] >> (x * 8) & 1u)) y = 0.f;
                        big[n][j] = fmaxf(big[n][j], y);
                    }
                    out |= big[n][j] > room[n][j];
                }
            if (__any_sync(0xFFFFFFFFu, out)) {
                float ratio[NR][2];
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) big[n][j] = fmaxf(big[n][j], __shfl_xor_sync(0xFFFFFFFFu, big[n][j], d));
                        ratio[n][j] = 1.f;
                        if (alpha[n][j] == 1.f && !(big[n][j] > room[n][j])) continue;
                        most[n][j] = fmaxf(most[n][j] * alpha[n][j], big[n][j]);
                        const uint32_t e = top_exponent(__float_as_uint(most[n][j]));
                        const float f = to_half_range(e);
                        ratio[n][j] = alpha[n][j] * inverse_power(to_half[n][j]) * f;              // powers of two but for alpha
                        to_half[n][j] = f;
                        room[n][j] = half_range_end(e);
                    }
#pragma unroll
                for (int x = 0; x < D / 16; x++)
#pragma unroll
                    for (int n = 0; n < NR; n++)
#pragma unroll
                        for (int e = 0; e < 4; e++) o[x][n][e] *= ratio[n][e & 1];
            }
            // Weights in fp16, 2^-11 relative at most; the sum of the weights takes them unrounded.
            uint32_t pf[MT][NR][2];
#pragma unroll
            for (int n = 0; n < NR; n++) {
                const float f0 = to_half[n][0], f1 = to_half[n][1];
#pragma unroll
                for (int x = 0; x < 2 * MT; x++)
                    pf[x >> 1][n][x & 1] = transposed(pack2<__half>(sc[x >> 1][n][2 * (x & 1)] * f0, sc[x >> 1][n][2 * (x & 1) + 1] * f1));
            }
            if constexpr (MT == 1) {
#pragma unroll
                for (int np = 0; np < D / 16; np += 2) {
                    uint32_t v[4];                     // 16 tokens of chunk np, of chunk np + 1
                    ldsm4t(v, base + L::half + L::at(lane & 15u, np + (lane >> 4)));
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        uint32_t f[4];
                        four_codes(__byte_perm(v[2 * y], 0u, 0x3120), f[0], f[1]);
                        four_codes(__byte_perm(v[2 * y + 1], 0u, 0x3120), f[2], f[3]);
#pragma unroll
                        for (int n = 0; n < NR; n++) mma16816<__half>(o[np + y][n], f, pf[0][n][0], pf[0][n][1]);
                    }
                }
            } else {
#pragma unroll
                for (int np = 0; np < D / 16; np++) {
                    uint32_t v[4];                     // 32 tokens of chunk np
                    ldsm4t(v, base + L::half + L::at(lane, np));
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        uint32_t f[4];
                        four_codes(__byte_perm(v[2 * y], 0u, 0x3120), f[0], f[1]);
                        four_codes(__byte_perm(v[2 * y + 1], 0u, 0x3120), f[2], f[3]);
#pragma unroll
                        for (int n = 0; n < NR; n++) mma16816<__half>(o[np][n], f, pf[y][n][0], pf[y][n][1]);
                    }
                }
            }
            __syncwarp();                              // the stage may be filled again
            get = get == FEW8_STAGES - 1 ? 0u : get + 1u;
        }
        bits |= label_read_status(label, owner);
        cp_wait<0>();

        // Join the warps' parts.
#pragma unroll
        for (int n = 0; n < NR; n++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xFFFFFFFFu, l[n][j], d);
                if (g == 0) s_ml[warp][n * 8 + 2 * c + j] = make_float2(m[n][j], l[n][j]);
            }
        bits = __reduce_or_sync(0xFFFFFFFFu, bits);
        if (threadIdx.x == 0) s_bits = 0u;
        __syncthreads();                               // the ring is idle; s_ml is complete
        if (lane == 0 && (bits & ~FOUND_NAN)) atomicOr(&s_bits, bits & ~FOUND_NAN);
        const uint32_t nr = all_q - q0 < (uint32_t)ROWS ? all_q - q0 : (uint32_t)ROWS;
        float* join = reinterpret_cast<float*>(smem) + (uint32_t)warp * (ROWS * D);
#pragma unroll
        for (int n = 0; n < NR; n++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const uint32_t row = n * 8 + 2 * c + j;
                const float unit = inverse_power(to_half[n][j]);
                if (row < nr)
#pragma unroll
                    for (int np = 0; np < D / 16; np++)
                        *reinterpret_cast<float2*>(join + row * D + np * 16 + 2 * g) = make_float2(o[np][n][j] * unit, o[np][n][2 + j] * unit);
            }
        if (bits & FOUND_NAN) put_nan_part<D, NR>(a, w.r, w.row0, w.h, w.qt, w.tb, w.n_tiles, reinterpret_cast<float*>(smem));
        __syncthreads();
        bits = s_bits;
        const bool whole = w.whole();
        const uint32_t at = w.slot() * a.head_ways;    // the first of the heads' parts
        const uint32_t heads_rows = a.head_ways * ROWS;
        for (uint32_t x = threadIdx.x; x < heads_rows * CH; x += THREADS) {
            const uint32_t ch = x % CH, row = x / CH % ROWS, hw = x / (CH * ROWS);
            if (row >= nr) continue;
            float top = NOTHING;
            for (uint32_t y = hw; y < (uint32_t)L::warps; y += a.head_ways) top = fmaxf(top, s_ml[y][row].x);
            float sum = 0.f, acc[8];
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] = 0.f;
            for (uint32_t y = hw; y < (uint32_t)L::warps; y += a.head_ways) {
                const float f = fast_exp2(s_ml[y][row].x - top);
                sum += s_ml[y][row].y * f;
                const float4* from = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (y * ROWS + row) * D + ch * 8);
                const float4 u = from[0], v = from[1];
                // a warp that saw nothing holds zeros
                acc[0] += f * u.x; acc[1] += f * u.y; acc[2] += f * u.z; acc[3] += f * u.w;
                acc[4] += f * v.x; acc[5] += f * v.y; acc[6] += f * v.z; acc[7] += f * v.w;
            }
            if (whole) {
                put_row(a, row0, w.h * a.head_ways + hw, q0 + row, ch, acc, top, sum, bits);
            } else {
                const uint64_t part = (uint64_t)(at + hw) * ROWS + row;
                float4* to = reinterpret_cast<float4*>(a.part_o + part * D + ch * 8);
                to[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                to[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (ch == 0) a.part_ml[part] = make_float2(top, sum);
            }
        }
        if (whole) {
            if (w.h == 0 && w.qt == 0) write_request<THREADS>(a, r, row0, it.rows_m, bits);
            __syncthreads();                           // smem is free for the next piece
            continue;
        }
        // The last of an item's pieces to be ready joins them: every piece is in memory before its CTA takes a
        // ticket.
        if (threadIdx.x == 0) a.part_head[w.slot()].bits = bits;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint64_t item = begin + (units - w.left) - w.u;      // the item's first unit
            const uint32_t w0 = (uint32_t)((item + a.extra) / slice);  // the slice with its first tile
            s_head.pieces = (uint32_t)((item + it.cost - 1) / slice) - w0 + 1u;
            s_head.r = r; s_head.row0 = row0; s_head.rows_m = it.rows_m;
            s_head.h = w.h; s_head.q0 = q0; s_head.nr = nr;
            s_first = w0;
            s_last = atomicAdd(&a.tickets[w0], 1u) + 1u == s_head.pieces;
            s_bits = 0u;
        }
        __syncthreads();
        if (s_last) {
            __threadfence();
            join8<D, ROWS, THREADS>(a, s_head, s_first, s_top, &s_bits);
        }
        __syncthreads();                               // smem is free for the next piece
    }
    leave_tickets(a);
}

template <int D, int NR, bool NEAR>
int launch_few8(gift_ctx* c, Attn8Args& a, cudaStream_t st)
{
    using L = Few8<D, NR>;
    CU_TRY((allow_smem<attn8_few_kernel<D, NR, NEAR>>(c->device, L::smem)));
    a.n_slices = (uint32_t)L::ctas * c->num_sms;
    a.ways = 1;
    a.tile_rows = L::rows;
    a.by_tile_rows = fixed_div(a.tile_rows);
    a.least = 1;
    a.extra = 4;                             // a decode step with 0, 2, 4, 8, 16: 129, 124, 120, 122, 130 us, at the time
    // Heads lie next to one another in a token, so warps that take the heads of the same tokens read longer runs of memory
    // at a time; but with few items in a call, fewer heads in each mean fewer pieces for one CTA to join.
    a.head_ways = L::warps;
    while (a.head_ways > 1 && (a.kv_heads % a.head_ways || (uint64_t)a.b.n_req * (a.kv_heads / a.head_ways) < FEW8_ITEMS)) a.head_ways /= 2;
    a.kv_heads /= a.head_ways;
    a.tile_tokens = L::warps / a.head_ways * L::tok;
    a.whole_steps = a.b.page_tokens % L::tok == 0;
    attn8_few_kernel<D, NR, NEAR><<<a.n_slices, L::threads, L::smem, st>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

// The pool as rows of one token, taken a head's codes of a run of tokens at a time.
int map_of_codes(const Attn8Args& a, uint32_t head_dim, CUtensorMap* map)
{
    EncodeTiled encode;
    const int rc = encode_tiled(&encode);
    if (rc != GIFT_OK) return rc;
    const cuuint64_t dims[2] = {a.token_bytes, a.b.n_pages ? (cuuint64_t)a.b.n_pages * a.b.page_tokens : 1};
    const cuuint64_t strides[1] = {a.token_bytes};
    const cuuint32_t box[2] = {head_dim, a.copy_run}, steps[2] = {1, 1};
    if (encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<char*>(a.pages), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return GIFT_E_CUDA;
    return GIFT_OK;
}

template <int D, bool NEAR>
int launch_many8(gift_ctx* c, Attn8Args& a, uint64_t rows, cudaStream_t st)
{
    CUtensorMap q_map, code_map;
    a.copy_run = a.b.page_tokens & (0u - a.b.page_tokens);
    if (a.copy_run > (uint32_t)TC8_TILE) a.copy_run = TC8_TILE;
    int rc = map_of_q(a, a.half != 0u, D, &q_map);
    if (rc == GIFT_OK) rc = map_of_codes(a, D, &code_map);
    if (rc != GIFT_OK) return rc;
    constexpr int smem = Tc8Smem<D>::bytes;
    CU_TRY((allow_smem<attn8_tc_kernel<D, NEAR>>(c->device, smem)));
    // two CTAs to a slice when an average request's rows fill more than one tile: neighbouring items read the same tokens
    // (prompt chunks 361 us, with a slice to each CTA 417, at the time)
    a.ways = rows > (uint64_t)TC8_ROWS ? 2u : 1u;
    a.n_slices = 2u * c->num_sms / a.ways;
    a.tile_rows = TC8_ROWS / a.group * a.group;            // whole tokens
    a.by_tile_rows = fixed_div(a.tile_rows);
    a.tile_tokens = (uint32_t)TC8_ROWS / a.group;
    a.least = 4;
    a.extra = 8;                             // 4, 6, 12: 0.1, 0.6, 1.6 % more for trees with grouped heads
    // the kernel takes the maximum before it scales: the scale must be positive
    a.negate = a.scale_log2 < 0.f ? 1u : 0u;
    a.wait_tries = c->attn_wait_ns ? (uint32_t)(c->attn_wait_ns / TC_SUSPEND_NS) : TC_WAIT_TRIES;
    a.wait_ns = c->attn_wait_ns && c->attn_wait_ns < TC_SUSPEND_NS ? (uint32_t)c->attn_wait_ns : TC_SUSPEND_NS;
    a.scale_log2 = fabsf(a.scale_log2);
    a.cap_in = fabsf(a.cap_in);
    attn8_tc_kernel<D, NEAR><<<a.n_slices * a.ways, TC8_THREADS, smem, st>>>(a, q_map, code_map);
    c->launches++;
    CU_TRY(cudaGetLastError());
    if (a.half) CU_TRY((launch_join<__half, D, TC8_ROWS>(a, st)));
    else CU_TRY((launch_join<__nv_bfloat16, D, TC8_ROWS>(a, st)));
    c->launches++;
    return GIFT_OK;
}

template <int D>
int launch_attn8(gift_ctx* c, Attn8Args& a, cudaStream_t st)
{
    const bool near = a.cap_out != 0.f || a.slopes || a.window;
    // what the tensor map of q does not describe: groups of more heads than a tile has rows, a q whose rows or heads
    // share memory
    const bool plain_q = a.group <= (uint32_t)TC8_ROWS && (a.n_rows == 1 || a.q_row > 0) && (a.heads == 1 || a.q_head > 0);
    // Rows of an average request's K/V head decide for the whole call; 17 to 24 of them: 633 us with tcgen05 products, 690 with two items of 16,
    // at the time.  A call that mixes prompts and decode rows pays for it (64 decode rows and a prompt of 2 048: 625 us, apart 121 and 150).
    const uint64_t rows = ((uint64_t)a.n_rows + a.b.n_req - 1) / a.b.n_req * a.group;
    if (rows <= 8) return near ? launch_few8<D, 1, true>(c, a, st) : launch_few8<D, 1, false>(c, a, st);
    if (rows <= 16 || !plain_q) return near ? launch_few8<D, 2, true>(c, a, st) : launch_few8<D, 2, false>(c, a, st);
    return near ? launch_many8<D, true>(c, a, rows, st) : launch_many8<D, false>(c, a, rows, st);
}

}  // namespace

extern "C" int gift_kv_attention_codes(gift_ctx* c, const gift_batch* batch, const gift_kv_pool* pool, const gift_attn_codes* t8,
                                  uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    int rc = batch_args_ok(batch);
    if (rc != GIFT_OK) return rc;
    if (pool && pool->dtype != GIFT_E4M3) return GIFT_E_INVAL;
    if ((rc = any_pool_args_ok(pool)) != GIFT_OK) return rc;
    if (!t8) return GIFT_E_INVAL;
    const gift_attn* t = &t8->attn;
    if (batch->n_req == 0) return GIFT_OK;
    if (!status || pool->n_pages != batch->n_pages || pool->page_tokens != batch->page_tokens) return GIFT_E_INVAL;
    if (t8->dtype != GIFT_BF16 && t8->dtype != GIFT_FP16) return GIFT_E_INVAL;
    if (pool->head_dim != 64 && pool->head_dim != 128) return GIFT_E_RANGE;
    if (t->n_heads == 0 || t->n_heads % pool->n_heads != 0) return GIFT_E_INVAL;
    if (t->n_heads > GIFT_MAX_HEADS || t->mask_words > 0x00FFFFFFu || (uint64_t)t->n_rows * t->n_heads > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (t->tree_mask && t->mask_words == 0) return GIFT_E_INVAL;
    if (t->tree_mask && (t8->slopes || t8->window)) return GIFT_E_INVAL;
    if (t8->window > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (!isfinite(t->scale) || !isfinite(t8->softcap) || t8->softcap < 0.f) return GIFT_E_INVAL;
    if (!isfinite(t->scale * LOG2_E) || !isfinite(t8->softcap * LOG2_E)) return GIFT_E_RANGE;
    if (t8->softcap != 0.f && !isfinite(t->scale / t8->softcap)) return GIFT_E_RANGE;
    if (t->n_rows) {
        if ((rc = rows_args_ok(t->q, t->q_row_stride, t->q_head_stride)) != GIFT_OK) return rc;
        if ((rc = rows_args_ok(t->out, t->out_row_stride, t->out_head_stride)) != GIFT_OK) return rc;
        // rows that share memory cannot all be written
        if ((t->n_rows > 1 && t->out_row_stride == 0) || (t->n_heads > 1 && t->out_head_stride == 0)) return GIFT_E_INVAL;
    }
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = scratch_ensure(c, st)) != GIFT_OK) return rc;
    Attn8Args a;
    memset(&a, 0, sizeof(a));
    a.b = batch_args(batch);
    a.pages = static_cast<const char*>(pool->pages);
    const Kv8 layout = kv8_layout(pool);
    a.token_bytes = layout.token;
    a.codes = layout.codes;
    a.kv_heads = pool->n_heads; a.heads = t->n_heads; a.group = t->n_heads / pool->n_heads;
    a.by_group = fixed_div(a.group);
    a.q = static_cast<const char*>(t->q); a.q_row = t->q_row_stride * 2; a.q_head = t->q_head_stride * 2;
    a.out = static_cast<char*>(t->out); a.out_row = t->out_row_stride * 2; a.out_head = t->out_head_stride * 2;
    a.n_rows = t->n_rows;
    a.scale_log2 = t->scale * LOG2_E;
    a.mask = t->tree_mask; a.mask_words = t->mask_words;
    a.lse = t->lse; a.row_owner = t->row_owner; a.owner_map = pool->owner_map; a.status = status;
    a.window = t8->window;
    a.slopes = t8->slopes;
    if (t8->softcap != 0.f) {
        a.cap_in = t->scale / t8->softcap;
        a.cap_out = t8->softcap * LOG2_E;
    }
    use_scratch(c, a);
    a.half = t8->dtype == GIFT_FP16;
    return pool->head_dim == 128 ? launch_attn8<128>(c, a, st) : launch_attn8<64>(c, a, st);
}
