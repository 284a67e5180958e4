// Attention of a step's rows over the labelled paged cache (the subject of the SEGREDUCE rule,
// with the rule checked on the very block table that is read).
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "gift_attn.cuh"
#include "gift_attn_join.cuh"
#include "gift_attn_tc.cuh"
#include "gift_internal.cuh"
#include "gift_kv.cuh"

using namespace gift;

namespace {

// ---------------------------------------------------------------------------
// few query rows per K/V head: warp-level products
// ---------------------------------------------------------------------------
//
// With R query rows per K/V head the kernel does R operations per K/V byte, so up to 16 rows HBM
// bandwidth bounds it and the matrix instructions need only keep out of the way.  Every warp
// works on its own tokens of a tile (16 of 64, or 32 of 128 when a head is 64 wide, so that a
// step moves 8 KiB either way), with a ring of 3 stages of K and V rows in shared memory that
// only it fills and reads: no barrier inside a piece.  2 CTAs of 4 warps per SM keep up to 192 KiB
// in flight.  The warps' maxima, sums and rows are joined at a piece's end, the pieces of a cut item by
// the CTA whose piece is ready last (a second kernel for that: 29.6 us a call of one token from Python,
// this way 27.0; the device's time is the same).  64 requests of 256 to 8192
// tokens, 32 heads: 16 rows 688 us (6.5 TB/s), 8 rows 678 us; one row over 256 to 2048 tokens 198 us
// (6.1 TB/s); one request of 514 tokens and one row 14.4 us.

constexpr int FEW_WARPS = 4;
constexpr int FEW_THREADS = FEW_WARPS * 32;
static_assert(FEW_THREADS == JOIN_THREADS, "the last CTA of a cut item joins it");
constexpr int FEW_ROWS = 16;
constexpr int FEW_STAGES = 3;
template <int D> constexpr int FEW_BLOCKS = 128 / D;                     // 16-token blocks of a warp's step
template <int D> constexpr int FEW_TILE = FEW_WARPS * 16 * FEW_BLOCKS<D>;

// Address of 16-byte chunk `chunk` of row `row` in a tile of rows of D elements: chunks are
// permuted within a row by the row number, so that 8 rows' equal chunks lie in different banks.
template <int D> __device__ __forceinline__ uint32_t tile_at(uint32_t base, uint32_t row, uint32_t chunk)
{
    return base + row * (D * 2) + ((chunk ^ (row & 7u)) << 4);
}

template <int D> struct FewSmem {
    static constexpr int half = 16 * FEW_BLOCKS<D> * D * 2;              // bytes of a step's K (or V) rows
    static constexpr int ring = FEW_WARPS * FEW_STAGES * 2 * half;
    static constexpr int join = FEW_WARPS * FEW_ROWS * D * 4;
    static constexpr int bytes = ring > join ? ring : join;
};

template <class T, int D>
__global__ void __launch_bounds__(FEW_THREADS, 2) attn_few_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr int ROWS = FEW_ROWS, NB = FEW_BLOCKS<D>, TOK = 16 * NB, TILE = FEW_TILE<D>;
    constexpr int CH = D / 8;                      // 16-byte chunks of a K or V row
    constexpr int KS = D / 16;                     // k steps of the score product
    constexpr uint32_t HALF = FewSmem<D>::half;
    extern __shared__ __align__(128) char smem[];
    __shared__ PlaceShared place;
    __shared__ float2 s_ml[FEW_WARPS][ROWS];
    __shared__ uint32_t s_bits, s_last, s_first;
    __shared__ JoinShared s_join;
    __shared__ PartHead s_head;

    uint64_t total, slice;
    if (!place_unit<FEW_THREADS>(a, blockIdx.x, TILE, blockIdx.x == 0, &place, &total, &slice)) {
        leave_tickets(a);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (FEW_STAGES * 2 * HALF);

    Walk<TILE> w;
    const uint64_t begin = slice * blockIdx.x, units = slice < total - begin ? slice : total - begin;
    w.start(a, place.at, 0, units);
    while (w.next(a)) {
        const ReqShape& s = w.s;
        const ItemShape& it = w.it;
        const uint32_t r = w.r, row0 = w.row0, tb = w.tb, n_tiles = w.n_tiles, h = w.h, qt = w.qt;
        const uint32_t all_q = it.rows_m * a.group;                // query rows of the K/V head
        const uint32_t q0 = qt * ROWS;
        const int32_t owner = a.b.owner[r];
        const int32_t* table = a.b.table + (uint64_t)r * a.b.max_blocks;
        const bool masked_short = w.masked_short(a);
        uint32_t bits = masked_short ? GIFT_ST_BAD_DESC : 0u;

        // this lane's query rows g and g + 8
        const uint32_t g = lane >> 2, c2 = (lane & 3) * 2;
        uint32_t qf[KS][4];
        uint32_t row_i[2];
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const uint32_t rho = q0 + half * 8 + g;
            const bool there = rho < all_q;
            const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = h * a.group + (there ? rho - i * a.group : 0u);
            row_i[half] = i;
            const char* q = a.q + (uint64_t)(row0 + i) * a.q_row + (uint64_t)hq * a.q_head;
#pragma unroll
            for (int ks = 0; ks < KS; ks++)
#pragma unroll
                for (int hi = 0; hi < 2; hi++)
                    qf[ks][hi * 2 + half] = there ? *reinterpret_cast<const uint32_t*>(q + (ks * 16 + hi * 8 + c2) * 2) : 0u;
        }
        float o[D / 8][4];
        float m[2] = {NEG_INF, NEG_INF}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < D / 8; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) o[n][e] = 0.f;

        // Lane x looks after token x % TOK of the warp's: its table entry is fetched one step ahead of
        // the copies that need it, its label is judged one step after it was asked for.
        const uint32_t my = lane % TOK;
        auto entry = [&](uint32_t step) -> int32_t {
            const uint32_t t = (tb + step) * TILE + warp * TOK + my;
            return step < n_tiles && t < s.want ? table[a.b.page.quot(t)] : -1;
        };
        int32_t next = entry(0), label = GIFT_OWNER_PARAM;
        auto issue = [&](uint32_t step) {
            if (step < n_tiles) {
                const uint32_t t = (tb + step) * TILE + warp * TOK + my;
                const int32_t page = next;
                next = entry(step + 1);
                bits |= label_read_status(label, owner);
                label = GIFT_OWNER_PARAM;
                // the token's slot; rows past the context are filled with zeros: what memory holds there does not matter
                uint32_t slot = 0xFFFFFFFFu;
                if (t < s.want) {
                    if ((uint32_t)page < a.b.n_pages) {
                        slot = (uint32_t)page * a.b.page_tokens + (t - a.b.page.quot(t) * a.b.page_tokens);
                        if (a.owner_map) label = a.owner_map[page];
                    } else {
                        bits |= GIFT_ST_BAD_DESC;
                    }
                }
                const uint32_t base = ring + (step % FEW_STAGES) * (2 * HALF), chunk = lane % CH;
                const char* head = a.pages + (uint64_t)h * (D * 2) + chunk * 16;
                const uint64_t to_v = (uint64_t)a.kv_heads * (D * 2);
#pragma unroll
                for (int i = 0; i < CH * TOK / 32; i++) {
                    const uint32_t row = i * (32 / CH) + lane / CH;
                    const uint32_t from = __shfl_sync(0xFFFFFFFFu, slot, row);
                    const bool there = from != 0xFFFFFFFFu;
                    const char* p = there ? head + (uint64_t)from * a.token_bytes : head;
                    cp_async16(tile_at<D>(base, row, chunk), p, there ? 16u : 0u);
                    cp_async16(tile_at<D>(base + HALF, row, chunk), p + to_v, there ? 16u : 0u);
                }
            }
            cp_commit();
        };
        // the first rounds only fill the ring (one copy of the code: it is large, and short items meet it cold)
#pragma unroll 1
        for (uint32_t round = 0; round < n_tiles + FEW_STAGES - 1; round++) {
            issue(round);
            if (round < (uint32_t)FEW_STAGES - 1) continue;
            const uint32_t step = round - (FEW_STAGES - 1);
            cp_wait<FEW_STAGES - 1>();
            __syncwarp();
            const uint32_t kb = ring + (step % FEW_STAGES) * (2 * HALF), vb = kb + HALF;
            const uint32_t t0 = (tb + step) * TILE + warp * TOK;
            float sc[2 * NB][4];
#pragma unroll
            for (int n = 0; n < 2 * NB; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) sc[n][e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ks++)
#pragma unroll
                for (int k = 0; k < NB; k++) {
                    uint32_t kf[4];
                    ldsm4(kf, tile_at<D>(kb, k * 16 + (lane >> 4) * 8 + (lane & 7), ks * 2 + ((lane >> 3) & 1)));
                    mma16816<T>(sc[2 * k], qf[ks], kf[0], kf[1]);
                    mma16816<T>(sc[2 * k + 1], qf[ks], kf[2], kf[3]);
                }
#pragma unroll
            for (int n = 0; n < 2 * NB; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) sc[n][e] *= a.scale_log2;
            const bool mixed = t0 + TOK > s.have;      // some rows may not see some of these tokens
            uint32_t sees[2];                          // of the step's tokens, by row
            if (mixed) {
                const bool none = masked_short || t0 >= s.want;
#pragma unroll
                for (int half = 0; half < 2; half++)
                    sees[half] = none ? 0u : (uint32_t)row_sees64(a, s.have, s.want, row0 + row_i[half], row_i[half], t0);
#pragma unroll
                for (int n = 0; n < 2 * NB; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (!(sees[e >> 1] >> (n * 8 + c2 + (e & 1)) & 1u)) sc[n][e] = NEG_INF;
            }
            float alpha[2];
#pragma unroll
            for (int half = 0; half < 2; half++) {
                float top = fmaxf(sc[0][half * 2], sc[0][half * 2 + 1]);
#pragma unroll
                for (int n = 1; n < 2 * NB; n++) top = fmaxf(top, fmaxf(sc[n][half * 2], sc[n][half * 2 + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const float now = fmaxf(m[half], top);
                const float use = now == NEG_INF ? 0.f : now;          // nothing seen yet: exp2(-inf - 0) = 0
                alpha[half] = fast_exp2(m[half] - use);
                m[half] = now;
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < 2 * NB; n++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const float p = fast_exp2(sc[n][half * 2 + e] - use);
                        sc[n][half * 2 + e] = p;
                        sum += p;
                    }
                l[half] = l[half] * alpha[half] + sum;
            }
            if (__any_sync(0xFFFFFFFFu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int n = 0; n < D / 8; n++) {
                    o[n][0] *= alpha[0]; o[n][1] *= alpha[0];
                    o[n][2] *= alpha[1]; o[n][3] *= alpha[1];
                }
            }
            // 0 * inf is NaN: where a row may not see a token whose v is not finite, the product is
            // taken token by token, over what the row sees
            bool plain = true;
            if (mixed) {
                bool odd = false;
#pragma unroll
                for (int i = 0; i < CH * TOK / 32; i++) {
                    uint4 x;
                    const uint32_t at = vb + (i * 32 + lane) * 16;
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
                    odd |= pair_not_finite<T>(x.x) || pair_not_finite<T>(x.y) || pair_not_finite<T>(x.z) || pair_not_finite<T>(x.w);
                }
                plain = !__any_sync(0xFFFFFFFFu, odd);
            }
            if (plain) {
                // p is rounded to the pool's type: the operands of one product have one type, and the
                // rounding (half a step: 2^-8 relative at most for bf16, 2^-11 for fp16) is of the size of v's own;
                // the sum of the weights takes them unrounded
                uint32_t pf[NB][4];
#pragma unroll
                for (int k = 0; k < NB; k++) {
                    pf[k][0] = pack2<T>(sc[2 * k][0], sc[2 * k][1]);
                    pf[k][1] = pack2<T>(sc[2 * k][2], sc[2 * k][3]);
                    pf[k][2] = pack2<T>(sc[2 * k + 1][0], sc[2 * k + 1][1]);
                    pf[k][3] = pack2<T>(sc[2 * k + 1][2], sc[2 * k + 1][3]);
                }
#pragma unroll
                for (int np = 0; np < D / 16; np++)
#pragma unroll
                    for (int k = 0; k < NB; k++) {
                        uint32_t vf[4];
                        ldsm4t(vf, tile_at<D>(vb, k * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), np * 2 + (lane >> 4)));
                        mma16816<T>(o[np * 2], pf[k], vf[0], vf[1]);
                        mma16816<T>(o[np * 2 + 1], pf[k], vf[2], vf[3]);
                    }
            } else {
#pragma unroll
                for (int n0 = 0; n0 < 2 * NB; n0++)
#pragma unroll 1
                    for (int t = n0 * 8; t < n0 * 8 + 8; t++) {
#pragma unroll
                        for (int half = 0; half < 2; half++) {
                            // token t's p of this lane's row: held by lane (t % 8) / 2 of the row's four
                            const int from = (lane & ~3) | ((t & 7) >> 1);
                            const float p0 = __shfl_sync(0xFFFFFFFFu, sc[n0][half * 2], from);
                            const float p1 = __shfl_sync(0xFFFFFFFFu, sc[n0][half * 2 + 1], from);
                            const float p = t & 1 ? p1 : p0;
                            if (sees[half] >> t & 1u) {
#pragma unroll
                                for (int n = 0; n < D / 8; n++) {
                                    uint32_t x;
                                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(tile_at<D>(vb, t, n) + c2 * 2) : "memory");
                                    const T* v = reinterpret_cast<const T*>(&x);
                                    o[n][half * 2] += p * to_float<T>(v[0]);
                                    o[n][half * 2 + 1] += p * to_float<T>(v[1]);
                                }
                            }
                            __syncwarp();
                        }
                    }
            }
            __syncwarp();                              // the stage may be filled again
        }
        bits |= label_read_status(label, owner);
        cp_wait<0>();

        // Join the four warps' parts.
#pragma unroll
        for (int half = 0; half < 2; half++) {
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 1);
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 2);
            if ((lane & 3) == 0) s_ml[warp][half * 8 + g] = make_float2(m[half], l[half]);
        }
        bits = __reduce_or_sync(0xFFFFFFFFu, bits);
        if (threadIdx.x == 0) s_bits = 0u;
        __syncthreads();                               // the ring is idle; s_ml is complete
        if (lane == 0 && bits) atomicOr(&s_bits, bits);
        float* join = reinterpret_cast<float*>(smem) + (uint32_t)warp * (ROWS * D);
#pragma unroll
        for (int n = 0; n < D / 8; n++)
#pragma unroll
            for (int half = 0; half < 2; half++)
                *reinterpret_cast<float2*>(join + (half * 8 + g) * D + n * 8 + c2) = make_float2(o[n][half * 2], o[n][half * 2 + 1]);
        __syncthreads();
        bits = s_bits;
        const bool whole = w.whole();
        const uint32_t slot = w.slot();
        const uint32_t nr = all_q - q0 < (uint32_t)ROWS ? all_q - q0 : (uint32_t)ROWS;
        for (uint32_t c = threadIdx.x; c < nr * (uint32_t)CH; c += FEW_THREADS) {
            const uint32_t row = c / CH, ch = c % CH;
            float top = NEG_INF;
#pragma unroll
            for (int w = 0; w < FEW_WARPS; w++) top = fmaxf(top, s_ml[w][row].x);
            const float use = top == NEG_INF ? 0.f : top;
            float sum = 0.f, acc[8];
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < FEW_WARPS; w++) {
                const float f = fast_exp2(s_ml[w][row].x - use);
                sum += s_ml[w][row].y * f;
                const float4* from = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * ROWS + row) * D + ch * 8);
                const float4 x = from[0], y = from[1];
                // a warp that saw nothing holds zeros, and f is 0
                acc[0] += f * x.x; acc[1] += f * x.y; acc[2] += f * x.z; acc[3] += f * x.w;
                acc[4] += f * y.x; acc[5] += f * y.y; acc[6] += f * y.z; acc[7] += f * y.w;
            }
            if (whole) {
                const uint32_t rho = q0 + row, i = a.by_group.quot(rho), hq = h * a.group + (rho - i * a.group);
                const bool none = bits != 0u || sum == 0.f;
                const float inv = none ? 0.f : 1.f / sum;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (!none) {
                    v.x = pack2<T>(acc[0] * inv, acc[1] * inv); v.y = pack2<T>(acc[2] * inv, acc[3] * inv);
                    v.z = pack2<T>(acc[4] * inv, acc[5] * inv); v.w = pack2<T>(acc[6] * inv, acc[7] * inv);
                }
                *reinterpret_cast<uint4*>(a.out + (uint64_t)(row0 + i) * a.out_row + (uint64_t)hq * a.out_head + ch * 16) = v;
                if (a.lse && ch == 0)
                    a.lse[(uint64_t)(row0 + i) * a.heads + hq] = none ? NEG_INF : (top + log2f(sum)) * 0.6931471805599453f;
            } else {
                float4* to = reinterpret_cast<float4*>(a.part_o + ((uint64_t)slot * ROWS + row) * D + ch * 8);
                to[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                to[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (ch == 0) a.part_ml[(uint64_t)slot * ROWS + row] = make_float2(top, sum);
            }
        }
        if (whole) {
            if (h == 0 && qt == 0) write_request<FEW_THREADS>(a, r, row0, it.rows_m, bits);
            __syncthreads();                           // smem is free for the next piece
            continue;
        }
        // The last of an item's pieces to be ready joins them: every piece is in memory before its CTA takes a
        // ticket.
        if (threadIdx.x == 0) a.part_head[slot].bits = bits;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint64_t item = begin + (units - w.left) - w.u;      // the item's first unit
            const uint32_t w0 = (uint32_t)((item + a.extra) / slice);  // the slice with its first tile
            s_head.pieces = (uint32_t)((item + it.cost - 1) / slice) - w0 + 1u;
            s_head.r = r; s_head.row0 = row0; s_head.rows_m = it.rows_m;
            s_head.h = h; s_head.q0 = q0; s_head.nr = nr;
            s_first = w0;
            s_last = atomicAdd(&a.tickets[w0], 1u) + 1u == s_head.pieces;
        }
        __syncthreads();
        if (s_last) {
            __threadfence();
            join_here<T, D, ROWS>(a, s_head, s_first, &s_join);
        }
        __syncthreads();                               // smem is free for the next piece
    }
    leave_tickets(a);
}

template <class T, int D>
int launch_few(gift_ctx* c, AttnArgs& a, cudaStream_t st)
{
    constexpr int smem = FewSmem<D>::bytes;
    CU_TRY((allow_smem<attn_few_kernel<T, D>>(c->device, smem)));
    a.n_slices = 2u * c->num_sms;
    a.ways = 1;
    a.tile_rows = FEW_ROWS;
    a.by_tile_rows = fixed_div(a.tile_rows);
    a.least = 1;
    a.extra = 4;                                           // 195 us for a decode step, with 0 235 us
    attn_few_kernel<T, D><<<a.n_slices, FEW_THREADS, smem, st>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

// The pool as rows of one token (row = slot), taken a run of rows by 64 columns at a time.
int slot_map_of_pool(const AttnArgs& a, bool half, uint32_t head_dim, CUtensorMap* map)
{
    EncodeTiled encode;
    const int rc = encode_tiled(&encode);
    if (rc != GIFT_OK) return rc;
    const cuuint64_t dims[2] = {(cuuint64_t)2 * a.kv_heads * head_dim, a.b.n_pages ? (cuuint64_t)a.b.n_pages * a.b.page_tokens : 1};
    const cuuint64_t strides[1] = {a.token_bytes};
    const cuuint32_t box[2] = {64, a.run < 8 ? 1 : a.run}, steps[2] = {1, 1};     // gathers take boxes of one row
    if (encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<char*>(a.pages), dims,
               strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return GIFT_E_CUDA;
    return GIFT_OK;
}

template <class T, int D>
int launch_many(gift_ctx* c, AttnArgs& a, uint64_t rows, cudaStream_t st)
{
    a.run = a.b.page_tokens & (0u - a.b.page_tokens);
    if (a.run > (uint32_t)TC_TILE) a.run = TC_TILE;
    CUtensorMap map, q_map;
    int rc = slot_map_of_pool(a, std::is_same<T, __half>::value, D, &map);
    if (rc == GIFT_OK) rc = map_of_q(a, std::is_same<T, __half>::value, D, &q_map);
    if (rc != GIFT_OK) return rc;
    constexpr int smem = TcSmem<D>::bytes;
    CU_TRY((allow_smem<attn_tc_kernel<T, D>>(c->device, smem)));
    // two CTAs to a slice when an average request's rows fill more than one tile (48 requests of 4 to 256
    // rows, up to 16384 tokens: 390 us, with a slice each 431 us: the second reading comes from HBM)
    a.ways = rows > (uint64_t)TC_ROWS ? 2u : 1u;
    a.n_slices = 2u * c->num_sms / a.ways;
    a.tile_rows = TC_ROWS / a.group * a.group;             // whole tokens
    a.by_tile_rows = fixed_div(a.tile_rows);
    a.least = 4;
    a.extra = 8;                                           // 202 us for 16 requests of 256 to 8192 tokens, with 0 273 us
    // the kernel takes the maximum before it scales: the scale must be positive (0 becomes a factor that
    // makes every finite score 0 in effect, and keeps a hidden token's minus infinity what it is)
    a.negate = a.scale_log2 < 0.f ? 1u : 0u;
    a.wait_tries = c->attn_wait_ns ? (uint32_t)(c->attn_wait_ns / TC_SUSPEND_NS) : TC_WAIT_TRIES;
    a.wait_ns = c->attn_wait_ns && c->attn_wait_ns < TC_SUSPEND_NS ? (uint32_t)c->attn_wait_ns : TC_SUSPEND_NS;
    a.scale_log2 = fmaxf(fabsf(a.scale_log2), 1e-44f);
    attn_tc_kernel<T, D><<<a.n_slices * a.ways, TC_THREADS, smem, st>>>(a, map, q_map);
    c->launches++;
    CU_TRY(cudaGetLastError());
    CU_TRY((launch_join<T, D, TC_ROWS>(a, st)));
    c->launches++;
    return GIFT_OK;
}

template <class T, int D>
int launch_attn(gift_ctx* c, AttnArgs& a, cudaStream_t st)
{
    // what the tensor maps of the tcgen05 kernel do not describe: groups of more heads than a tile has
    // rows, a q whose rows or heads share memory
    const bool plain_q = a.group <= (uint32_t)TC_ROWS && (a.n_rows == 1 || a.q_row > 0) && (a.heads == 1 || a.q_head > 0);
    // Rows of an average request's K/V head.  64 requests of 256 to 8192 tokens, 32 heads, warp-level against
    // tcgen05 products: 8 rows 678 and 744 us, 16 rows 687 and 706 us, 24 rows (two tiles of 16) 1389 and 714 us.
    const uint64_t rows = ((uint64_t)a.n_rows + a.b.n_req - 1) / a.b.n_req * a.group;
    return rows <= (uint64_t)FEW_ROWS || !plain_q ? launch_few<T, D>(c, a, st) : launch_many<T, D>(c, a, rows, st);
}

}  // namespace

extern "C" int gift_ctx_wait_limit(gift_ctx* c, uint64_t ns)
{
    if (!c) return GIFT_E_INVAL;
    if (ns > GIFT_MAX_WAIT_NS) return GIFT_E_RANGE;
    c->attn_wait_ns = ns;
    return GIFT_OK;
}

extern "C" int gift_kv_attention(gift_ctx* c, const gift_batch* batch, const gift_kv_pool* pool, const gift_attn* t,
                                 uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    int rc = batch_args_ok(batch);
    if (rc != GIFT_OK) return rc;
    if ((rc = pool_args_ok(pool)) != GIFT_OK) return rc;
    if (!t) return GIFT_E_INVAL;
    if (batch->n_req == 0) return GIFT_OK;
    if (!status || pool->n_pages != batch->n_pages || pool->page_tokens != batch->page_tokens) return GIFT_E_INVAL;
    if (pool->head_dim != 64 && pool->head_dim != 128) return GIFT_E_RANGE;
    if (t->n_heads == 0 || t->n_heads % pool->n_heads != 0) return GIFT_E_INVAL;
    if (t->n_heads > GIFT_MAX_HEADS || t->mask_words > 0x00FFFFFFu || (uint64_t)t->n_rows * t->n_heads > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (t->tree_mask && t->mask_words == 0) return GIFT_E_INVAL;
    if (!isfinite(t->scale)) return GIFT_E_INVAL;
    if (!isfinite(t->scale * 1.4426950408889634f)) return GIFT_E_RANGE;
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
    AttnArgs a;
    memset(&a, 0, sizeof(a));
    a.b = batch_args(batch);
    a.pages = static_cast<const char*>(pool->pages);
    a.token_bytes = (uint64_t)pool->n_heads * pool->head_dim * 4;
    a.kv_heads = pool->n_heads; a.heads = t->n_heads; a.group = t->n_heads / pool->n_heads;
    a.by_group = fixed_div(a.group);
    a.q = static_cast<const char*>(t->q); a.q_row = t->q_row_stride * 2; a.q_head = t->q_head_stride * 2;
    a.out = static_cast<char*>(t->out); a.out_row = t->out_row_stride * 2; a.out_head = t->out_head_stride * 2;
    a.n_rows = t->n_rows;
    a.scale_log2 = t->scale * 1.4426950408889634f;
    a.mask = t->tree_mask; a.mask_words = t->mask_words;
    a.lse = t->lse; a.row_owner = t->row_owner; a.owner_map = pool->owner_map; a.status = status;
    use_scratch(c, a);
    if (pool->dtype == GIFT_BF16)
        return pool->head_dim == 128 ? launch_attn<__nv_bfloat16, 128>(c, a, st) : launch_attn<__nv_bfloat16, 64>(c, a, st);
    return pool->head_dim == 128 ? launch_attn<__half, 128>(c, a, st) : launch_attn<__half, 64>(c, a, st);
}
