// Attention of a step's rows over labelled pages of 8 bits.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "gift_attn8.cuh"
#include "gift_attn_join.cuh"
#include "gift_internal.cuh"

using namespace gift;

namespace {

// ---------------------------------------------------------------------------
// few query rows per K/V head: warp-level products
// ---------------------------------------------------------------------------
//
// The split is that of the 16-bit kernel: every warp works on its own tokens of a tile, with a ring of 3 stages that
// only it fills and reads, 8 KiB of codes a step.  Codes become fp16 numbers (exact) on their way
// from shared memory to the matrix instructions:
//   K   A product's order of the 128 dimensions is free, so a lane takes 16 neighbouring codes of a token with one load, and
//       Q's fragments are laid out to match.
//   V   Loading 8 x 8 pairs of codes transposed gives a lane two neighbouring dimensions of two neighbouring
//       tokens; a byte permutation makes of it the fragments of an even and an odd dimension.
// K's scale multiplies the score, V's the weight, both in 32 bits: nothing but q and the weights is
// rounded.  Both go to fp16 by a power of two of the row's own (see top_exponent), for scales and queries of
// any size: the weights' follows the largest p * scale so far, as the maximum follows the scores.

constexpr int FEW8_WARPS = 4;
constexpr int FEW8_THREADS = FEW8_WARPS * 32;
constexpr int FEW8_ROWS = 16;
constexpr int FEW8_STAGES = 3;

template <int D> struct Few8 {
    static constexpr int tok = 4096 / D;                                 // tokens of a warp's step
    static constexpr int tile = FEW8_WARPS * tok;
    static constexpr int stage = 2 * 4096 + tok * 8;                     // codes of K, of V, scales
    static constexpr int ring = FEW8_WARPS * FEW8_STAGES * stage;
    static constexpr int join = FEW8_WARPS * FEW8_ROWS * D * 4;
    static constexpr int smem = ring > join ? ring : join;
    // Where 16-byte chunk `chunk` of a token lies in K's and in V's part: permuted so that the lanes that
    // load together (K: 4 chunks of 2 tokens; V: a chunk of 8 tokens) meet different banks.
    static __device__ __forceinline__ uint32_t k_at(uint32_t token, uint32_t chunk)
    {
        return token * D + ((D == 128 ? chunk ^ ((token & 1u) << 2) : chunk) << 4);
    }
    static __device__ __forceinline__ uint32_t v_at(uint32_t token, uint32_t chunk)
    {
        return 4096u + token * D + ((chunk ^ (D == 128 ? token & 7u : (token >> 1) & 3u)) << 4);
    }
};

__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}

// NEAR: capped scores, a bias by distance or a window.
template <class T, int D, bool NEAR>
__global__ void __launch_bounds__(FEW8_THREADS, 2) attn8_few_kernel(const __grid_constant__ Attn8Args a)
{
    using L = Few8<D>;
    constexpr int ROWS = FEW8_ROWS, TOK = L::tok, TILE = L::tile, NT = TOK / 8;
    constexpr int CH = D / 8;                      // 16-byte chunks of a result's row
    constexpr int KCH = D / 16;                    // 16-byte chunks of a token's codes
    extern __shared__ __align__(128) char smem[];
    __shared__ PlaceShared place;
    __shared__ float2 s_ml[FEW8_WARPS][ROWS];
    __shared__ uint32_t s_bits, s_last, s_first;
    __shared__ JoinShared s_join;
    __shared__ PartHead s_head;

    uint64_t total, slice;
    if (!place_unit<FEW8_THREADS, NEAR>(a, blockIdx.x, TILE, blockIdx.x == 0, &place, &total, &slice)) {
        leave_tickets(a);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (FEW8_STAGES * L::stage);

    Walk<TILE, NEAR> w;
    const uint64_t begin = slice * blockIdx.x, units = slice < total - begin ? slice : total - begin;
    w.start(a, place.at, 0, units);
    while (w.next(a)) {
        const ReqShape& s = w.s;
        const ItemShape& it = w.it;
        const uint32_t r = w.r, row0 = w.row0, tb = w.tb + (NEAR ? it.first : 0u), n_tiles = w.n_tiles, h = w.h;
        const uint32_t all_q = it.rows_m * a.group;                // query rows of the K/V head
        const uint32_t q0 = w.qt * ROWS;
        const int32_t owner = a.b.owner[r];
        const int32_t* table = a.b.table + (uint64_t)r * a.b.max_blocks;
        const bool masked_short = w.masked_short(a);
        const uint32_t low = NEAR ? first_seen(a, s.have) : 0u;    // tokens before it are nobody's to see
        uint32_t bits = masked_short ? GIFT_ST_BAD_DESC : 0u;

        // this lane's query rows g and g + 8; its dimensions are 16 from 16 (c + 4 i)
        const uint32_t g = lane >> 2, c = lane & 3u;
        uint32_t qf[D / 16][4];
        uint32_t row_i[2];
        float qs[2], slope[2];
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const uint32_t rho = q0 + half * 8 + g;
            const bool there = rho < all_q;
            const uint32_t i = there ? a.by_group.quot(rho) : 0u, hq = h * a.group + (there ? rho - i * a.group : 0u);
            row_i[half] = i;
            const uint4* q = reinterpret_cast<const uint4*>(a.q + (uint64_t)(row0 + i) * a.q_row + (uint64_t)hq * a.q_head);
            uint32_t x[D / 8];
#pragma unroll
            for (int y = 0; y < D / 32; y++) {
                const uint4 v = there ? q[(c + 4 * (y >> 1)) * 2 + (y & 1)] : make_uint4(0u, 0u, 0u, 0u);
                x[4 * y] = v.x; x[4 * y + 1] = v.y; x[4 * y + 2] = v.z; x[4 * y + 3] = v.w;
            }
            qs[half] = NEAR && a.cap_out != 0.f ? a.cap_in : a.scale_log2;
            if constexpr (!std::is_same<T, __half>::value) {
                uint32_t top = 0u;
#pragma unroll
                for (int y = 0; y < D / 8; y++) top = max(top, max(x[y] << 16 & 0x7FFFFFFFu, x[y] & 0x7FFF0000u));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const uint32_t e = top_exponent(top);
                const float f = to_half_range(e);
                qs[half] *= from_half_range(e);
#pragma unroll
                for (int y = 0; y < D / 8; y++)
                    x[y] = pack2<__half>(__uint_as_float(x[y] << 16) * f, __uint_as_float(x[y] & 0xFFFF0000u) * f);
            }
#pragma unroll
            for (int ks = 0; ks < D / 16; ks++) {
                qf[ks][half] = x[2 * ks];
                qf[ks][2 + half] = x[2 * ks + 1];
            }
            slope[half] = NEAR && a.slopes && there ? a.slopes[hq] * LOG2_E : 0.f;
        }
        float o[D / 8][4];
        float m[2] = {NEG_INF, NEG_INF}, l[2] = {0.f, 0.f};
        float most[2] = {0.f, 0.f};                                // largest p * scale, relative to the maximum
        uint32_t ew[2] = {13u, 13u};                               // its exponent: o is in units of from_half_range
#pragma unroll
        for (int n = 0; n < D / 8; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) o[n][e] = 0.f;

        // Lane x looks after tokens x (and x + 32) of the warp's: table entries are fetched one step ahead of
        // the copies that need them, labels judged one step after they were asked for.
        int32_t next[TOK / 32], label[TOK / 32];
        auto entry = [&](uint32_t step, int e) -> int32_t {
            const uint32_t t = (tb + step) * TILE + warp * TOK + e * 32 + lane;
            return step < n_tiles && t < s.want && (!NEAR || t >= low) ? table[a.b.page.quot(t)] : -1;
        };
#pragma unroll
        for (int e = 0; e < TOK / 32; e++) {
            next[e] = entry(0, e);
            label[e] = GIFT_OWNER_PARAM;
        }
        auto issue = [&](uint32_t step) {
            if (step < n_tiles) {
                const uint32_t base = ring + (step % FEW8_STAGES) * L::stage;
                uint32_t slot[TOK / 32];
#pragma unroll
                for (int e = 0; e < TOK / 32; e++) {
                    const uint32_t t = (tb + step) * TILE + warp * TOK + e * 32 + lane;
                    const int32_t page = next[e];
                    next[e] = entry(step + 1, e);
                    bits |= label_read_status(label[e], owner);
                    label[e] = GIFT_OWNER_PARAM;
                    // the token's slot; rows that nobody sees are filled with zeros: what memory holds there does not matter
                    slot[e] = 0xFFFFFFFFu;
                    if (t < s.want && (!NEAR || t >= low)) {
                        if ((uint32_t)page < a.b.n_pages) {
                            slot[e] = (uint32_t)page * a.b.page_tokens + (t - a.b.page.quot(t) * a.b.page_tokens);
                            if (a.owner_map) label[e] = a.owner_map[page];
                        } else {
                            bits |= GIFT_ST_BAD_DESC;
                        }
                    }
                    const bool there = slot[e] != 0xFFFFFFFFu;
                    cp_async8(base + 8192u + (e * 32 + lane) * 8u, a.pages + (there ? slot[e] * a.token_bytes + 2ull * a.codes + h * 8u : 0ull), there ? 8u : 0u);
                }
                const uint32_t chunk = lane % KCH;
                const char* head = a.pages + (uint64_t)h * D + chunk * 16;
#pragma unroll
                for (int i = 0; i < KCH * TOK / 32; i++) {
                    const uint32_t row = i * (32 / KCH) + lane / KCH;
                    const uint32_t from = __shfl_sync(0xFFFFFFFFu, slot[i * (32 / KCH) / 32], row & 31u);
                    const bool there = from != 0xFFFFFFFFu;
                    const char* p = there ? head + from * a.token_bytes : head;
                    cp_async16(base + L::k_at(row, chunk), p, there ? 16u : 0u);
                    cp_async16(base + L::v_at(row, chunk), p + a.codes, there ? 16u : 0u);
                }
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
            const uint32_t base = ring + (step % FEW8_STAGES) * L::stage;
            const uint32_t t0 = (tb + step) * TILE + warp * TOK;
            // some rows may not see some of these tokens
            const bool mixed = t0 + TOK > s.have || (NEAR && a.window && t0 + a.window < s.want);
            if (mixed) {
                // 0 * NaN is NaN: a token whose V holds the code of NaN, hidden from some row perhaps, gets it into its
                // scale, which is only used where the token is seen
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint4 x = lds128(base + 4096u + (i * 32 + lane) * 16);
                    odd |= codes_nan(x.x) || codes_nan(x.y) || codes_nan(x.z) || codes_nan(x.w);
                }
                if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll 1
                    for (int i = 0; i < 32; i++) {
                        const uint32_t at = (i * 32 + lane) * 4;
                        uint32_t x;
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(base + 4096u + at) : "memory");
                        if (codes_nan(x)) {
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + 4096u + at), "r"(codes_without_nan(x)) : "memory");
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + 8192u + (at / D) * 8u + 4u), "r"(0x7FC00000u) : "memory");
                        }
                    }
                    __syncwarp();
                }
            }
            float sc[NT][4], vs[NT][2];
#pragma unroll
            for (int n = 0; n < NT; n++) {
#pragma unroll
                for (int e = 0; e < 4; e++) sc[n][e] = 0.f;
#pragma unroll
                for (int i = 0; i < D / 64; i++) {
                    const uint4 k = lds128(base + L::k_at(n * 8 + g, c + 4 * i));
                    mma16816<__half>(sc[n], qf[i * 4], codes_to_half2(k.x & 0xFFFFu), codes_to_half2(k.x >> 16));
                    mma16816<__half>(sc[n], qf[i * 4 + 1], codes_to_half2(k.y & 0xFFFFu), codes_to_half2(k.y >> 16));
                    mma16816<__half>(sc[n], qf[i * 4 + 2], codes_to_half2(k.z & 0xFFFFu), codes_to_half2(k.z >> 16));
                    mma16816<__half>(sc[n], qf[i * 4 + 3], codes_to_half2(k.w & 0xFFFFu), codes_to_half2(k.w >> 16));
                }
                const uint4 x = lds128(base + 8192u + (n * 8 + c * 2) * 8u);
                const float ks[2] = {__uint_as_float(x.x), __uint_as_float(x.z)};
                vs[n][0] = __uint_as_float(x.y);
                vs[n][1] = __uint_as_float(x.w);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    sc[n][e] *= ks[e & 1] * qs[e >> 1];
                    if constexpr (NEAR) {
                        if (a.cap_out != 0.f) sc[n][e] = a.cap_out * tanh_of(sc[n][e]);
                        const int32_t away = (int32_t)(t0 + n * 8 + c * 2 + (e & 1)) - (int32_t)(s.have + row_i[e >> 1]);
                        if (a.slopes) sc[n][e] += slope[e >> 1] * (float)away;
                    }
                }
            }
            uint64_t sees[2] = {~0ull, ~0ull};
            if (mixed) {
                const bool none = masked_short || t0 >= s.want;
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    sees[half] = none ? 0ull : row_sees64(a, s.have, s.want, row0 + row_i[half], row_i[half], t0);
                    if (NEAR && a.window) sees[half] &= in_window64(a.window, s.have + row_i[half], t0);
                }
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (!(sees[e >> 1] >> (n * 8 + c * 2 + (e & 1)) & 1ull)) sc[n][e] = NEG_INF;
            }
            float ratio[2];
#pragma unroll
            for (int half = 0; half < 2; half++) {
                float top = fmaxf(sc[0][half * 2], sc[0][half * 2 + 1]);
#pragma unroll
                for (int n = 1; n < NT; n++) top = fmaxf(top, fmaxf(sc[n][half * 2], sc[n][half * 2 + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const float now = fmaxf(m[half], top);
                const float use = now == NEG_INF ? 0.f : now;          // nothing seen yet: exp2(-inf - 0) = 0
                const float alpha = fast_exp2(m[half] - use);
                m[half] = now;
                float sum = 0.f, big = 0.f;
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const float p = fast_exp2(sc[n][half * 2 + e] - use);
                        sum += p;
                        float x = p * vs[n][e];
                        if (mixed && !(sees[half] >> (n * 8 + c * 2 + e) & 1ull)) x = 0.f;
                        sc[n][half * 2 + e] = x;
                        big = fmaxf(big, x);
                    }
                l[half] = l[half] * alpha + sum;
                big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
                most[half] = fmaxf(most[half] * alpha, big);
                const uint32_t e = top_exponent(__float_as_uint(most[half]));
                ratio[half] = alpha * from_half_range(ew[half]) * to_half_range(e);
                ew[half] = e;
            }
            if (__any_sync(0xFFFFFFFFu, ratio[0] != 1.f || ratio[1] != 1.f)) {
#pragma unroll
                for (int n = 0; n < D / 8; n++) {
                    o[n][0] *= ratio[0]; o[n][1] *= ratio[0];
                    o[n][2] *= ratio[1]; o[n][3] *= ratio[1];
                }
            }
            // Weights in fp16, 2^-11 relative at most; the sum of the weights takes them unrounded.
            const float f0 = to_half_range(ew[0]), f1 = to_half_range(ew[1]);
            uint32_t pf[TOK / 16][4];
#pragma unroll
            for (int k = 0; k < TOK / 16; k++)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    pf[k][2 * x] = pack2<__half>(sc[2 * k + x][0] * f0, sc[2 * k + x][1] * f0);
                    pf[k][2 * x + 1] = pack2<__half>(sc[2 * k + x][2] * f1, sc[2 * k + x][3] * f1);
                }
#pragma unroll
            for (int np = 0; np < D / 16; np++)
#pragma unroll
                for (int k = 0; k < TOK / 32; k++) {
                    uint32_t v[4];
                    ldsm4t(v, base + L::v_at(k * 32 + lane, np));
#pragma unroll
                    for (int x = 0; x < 4; x++) v[x] = __byte_perm(v[x], 0u, 0x3120);
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        mma16816<__half>(o[np * 2], pf[2 * k + x], codes_to_half2(v[2 * x] & 0xFFFFu), codes_to_half2(v[2 * x + 1] & 0xFFFFu));
                        mma16816<__half>(o[np * 2 + 1], pf[2 * k + x], codes_to_half2(v[2 * x] >> 16), codes_to_half2(v[2 * x + 1] >> 16));
                    }
                }
            __syncwarp();                              // the stage may be filled again
        }
#pragma unroll
        for (int e = 0; e < TOK / 32; e++) bits |= label_read_status(label[e], owner);
        cp_wait<0>();

        // Join the four warps' parts.
#pragma unroll
        for (int half = 0; half < 2; half++) {
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 1);
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 2);
            if (c == 0) s_ml[warp][half * 8 + g] = make_float2(m[half], l[half]);
        }
        bits = __reduce_or_sync(0xFFFFFFFFu, bits);
        if (threadIdx.x == 0) s_bits = 0u;
        __syncthreads();                               // the ring is idle; s_ml is complete
        if (lane == 0 && bits) atomicOr(&s_bits, bits);
        float* join = reinterpret_cast<float*>(smem) + (uint32_t)warp * (ROWS * D);
        const float unit[2] = {from_half_range(ew[0]), from_half_range(ew[1])};
#pragma unroll
        for (int np = 0; np < D / 16; np++)
#pragma unroll
            for (int half = 0; half < 2; half++)
                // a lane's columns 2 c, 2 c + 1 are dimensions 4 c, 4 c + 2 of the even product, 4 c + 1, 4 c + 3 of the odd one
                *reinterpret_cast<float4*>(join + (half * 8 + g) * D + np * 16 + 4 * c) =
                    make_float4(o[np * 2][half * 2] * unit[half], o[np * 2 + 1][half * 2] * unit[half],
                                o[np * 2][half * 2 + 1] * unit[half], o[np * 2 + 1][half * 2 + 1] * unit[half]);
        __syncthreads();
        bits = s_bits;
        const bool whole = w.whole();
        const uint32_t at = w.slot();
        const uint32_t nr = all_q - q0 < (uint32_t)ROWS ? all_q - q0 : (uint32_t)ROWS;
        for (uint32_t x = threadIdx.x; x < nr * (uint32_t)CH; x += FEW8_THREADS) {
            const uint32_t row = x / CH, ch = x % CH;
            float top = NEG_INF;
#pragma unroll
            for (int y = 0; y < FEW8_WARPS; y++) top = fmaxf(top, s_ml[y][row].x);
            const float use = top == NEG_INF ? 0.f : top;
            float sum = 0.f, acc[8];
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] = 0.f;
#pragma unroll
            for (int y = 0; y < FEW8_WARPS; y++) {
                const float f = fast_exp2(s_ml[y][row].x - use);
                sum += s_ml[y][row].y * f;
                const float4* from = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (y * ROWS + row) * D + ch * 8);
                const float4 u = from[0], v = from[1];
                // a warp that saw nothing holds zeros, and f is 0
                acc[0] += f * u.x; acc[1] += f * u.y; acc[2] += f * u.z; acc[3] += f * u.w;
                acc[4] += f * v.x; acc[5] += f * v.y; acc[6] += f * v.z; acc[7] += f * v.w;
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
                float4* to = reinterpret_cast<float4*>(a.part_o + ((uint64_t)at * ROWS + row) * D + ch * 8);
                to[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                to[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (ch == 0) a.part_ml[(uint64_t)at * ROWS + row] = make_float2(top, sum);
            }
        }
        if (whole) {
            if (h == 0 && w.qt == 0) write_request<FEW8_THREADS>(a, r, row0, it.rows_m, bits);
            __syncthreads();                           // smem is free for the next piece
            continue;
        }
        // The last of an item's pieces to be ready joins them: every piece is in memory before its CTA takes a
        // ticket.
        if (threadIdx.x == 0) a.part_head[at].bits = bits;
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

template <class T, int D, bool NEAR>
int launch_few8(gift_ctx* c, Attn8Args& a, cudaStream_t st)
{
    constexpr int smem = Few8<D>::smem;
    CU_TRY((allow_smem<attn8_few_kernel<T, D, NEAR>>(c->device, smem)));
    a.n_slices = 2u * c->num_sms;
    a.ways = 1;
    a.tile_rows = FEW8_ROWS;
    a.by_tile_rows = fixed_div(a.tile_rows);
    a.least = 1;
    a.extra = 2;
    attn8_few_kernel<T, D, NEAR><<<a.n_slices, FEW8_THREADS, smem, st>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

template <class T, int D>
int launch_attn8(gift_ctx* c, Attn8Args& a, cudaStream_t st)
{
    const bool near = a.cap_out != 0.f || a.slopes || a.window;
    return near ? launch_few8<T, D, true>(c, a, st) : launch_few8<T, D, false>(c, a, st);
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
    if (t8->dtype == GIFT_BF16)
        return pool->head_dim == 128 ? launch_attn8<__nv_bfloat16, 128>(c, a, st) : launch_attn8<__nv_bfloat16, 64>(c, a, st);
    return pool->head_dim == 128 ? launch_attn8<__half, 128>(c, a, st) : launch_attn8<__half, 64>(c, a, st);
}
