// Rows on their way into the labelled pages and out of them: norms of the heads, rotary positions and 8-bit
// codes in the pass that writes, values in the pass that reads.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "gift_internal.cuh"
#include "gift_kv8.cuh"

using namespace gift;

namespace {

constexpr int ROW_THREADS = 256;
constexpr float CODE_MAX = 448.f;                // largest e4m3 number
constexpr float LEAST_SCALE = 0x1p-126f;         // a scale and its reciprocal are normal numbers
constexpr float SUM_MAX = 0x1p120f, SUM_MIN = 0x1p-90f;  // between which a sum of squares is as good as its 32 bits
constexpr int WRITE_UNROLL = 2;                  // heads that a group of lanes has under way

template <class T> __device__ __forceinline__ float2 unpack2(uint32_t x);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t x)
{
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
template <class T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// ---------------------------------------------------------------------------
// writing
// ---------------------------------------------------------------------------
//
// A pass over the rows: every byte is read once and written once, and HBM bandwidth should bound it; what has to be
// kept small is the instructions between (norm, turn and code are some 10 per element when done plainly).  A head is a
// group of L lanes with 16 elements each, in runs of 4: two quads of pairs where halves of a head turn
// against one another, so that a pair never leaves its lane.  The 8 angles of a lane are the same for all heads of a
// row: the warp's groups work out a share each and hand them round.  A warp takes the heads of a row kind by kind, so
// that its weights stay in registers, all of them where rows abound, a share where they do not.
// 32 700 rows of 32 + 2 x 32 heads of 128 to 8 bits: 316 us, 4.3 TB/s, 65 % of a copy; 256 rows 6.5 us.  What bounds it is the chain of
// a head's instructions with 16 warps on an SM (with 4 heads under way 347 us, with more warps of fewer registers 390 to 583), and accesses of
// 8 and 4 bytes, also to neighbours: L1 is asked for a sector more than once.

struct WriteArgs {
    const char *q, *k, *v;
    uint64_t q_row, q_head, k_row, k_head, v_row, v_head;    // strides in bytes
    char* q_out;
    uint64_t qo_row, qo_head;
    char* pages;
    uint64_t token_bytes;
    uint32_t codes;                          // K's (or V's) elements of one token
    const int64_t* slots;
    const int32_t* row_owner;
    const int32_t* owner_map;
    uint32_t* status;
    uint32_t n_rows, n_slots, dim;
    uint32_t q_heads, kv_heads;
    uint32_t q_rounds, kv_rounds;            // rounds of a warp over the heads of q, of k (and of v)
    uint32_t parts, iters;                   // warps that share a row, rounds of each
    uint64_t tasks;
    FixedDiv page;
    const void *q_norm, *k_norm;
    float eps, inv_dim;
    uint32_t n_freq;
    uint32_t ends[GIFT_MAX_AXES];            // first pair of the next axis
    const float* freq;
    const int32_t* pos;
    uint64_t pos_stride;
};

// cos and sin of pos * freq: the product in 64 bits (a position of 2^20 times a 32-bit frequency has no 32-bit
// place for its fraction of a turn), reduced to half a turn either way, the rest in 32 bits.
__device__ __forceinline__ float2 turn(int32_t pos, float freq)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189535;
    float2 r;
    sincospif(2.f * (float)(turns - rint(turns)), &r.y, &r.x);
    return r;
}

// A lane's place in a head.
struct Lane {
    uint32_t at[4];                          // first elements of its runs of 4
    bool holds[2], turns[2];                 // per quad
};

// Two 32-bit elements at a time.
struct Two { uint64_t v; };
__device__ __forceinline__ Two two(float lo, float hi)
{
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 apart(Two a)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Two mul(Two a, Two b)
{
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c)
{
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// The larger magnitude; NaN if either is.
__device__ __forceinline__ float top_of(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
template <class T> __device__ __forceinline__ Two unpack_two(uint32_t x)
{
    const float2 f = unpack2<T>(x);
    return two(f.x, f.y);
}

// The rounds [first, last) of one kind of head: KIND 0 q, 1 k, 2 v.  PAIRED: neighbours turn against one another.
// A head's norm is a factor of all its elements, so it waits: for q until the end, while K's codes do not change by it, only
// their scale does.
template <class T, bool POOL8, int L, bool PAIRED, int KIND>
__device__ __forceinline__ void write_heads(const WriteArgs& a, const Lane& own, uint32_t t, char* token, uint32_t first, uint32_t last,
                                            const Two (&cosines)[4], const Two (&sines)[4])
{
    constexpr uint32_t GROUPS = 32 / L;
    constexpr bool CODES = POOL8 && KIND != 0;
    if (first >= last) return;
    const uint32_t lane = threadIdx.x & 31, j = lane % L, group = lane / L;
    const uint32_t heads = KIND == 0 ? a.q_heads : a.kv_heads;
    const void* norm = KIND == 0 ? a.q_norm : KIND == 1 ? a.k_norm : nullptr;
    uint32_t at[4];
#pragma unroll
    for (int x = 0; x < 4; x++) at[x] = KIND == 2 ? 16 * j + 4 * x : own.at[x];
    const bool holds[2] = {KIND == 2 ? 16 * j < a.dim : own.holds[0], KIND == 2 ? 16 * j + 8 < a.dim : own.holds[1]};
    Two weight[4][2];
    if (KIND != 2 && norm)
#pragma unroll
        for (int x = 0; x < 4; x++) {
            const uint2 w = holds[x >> 1] ? *reinterpret_cast<const uint2*>(static_cast<const char*>(norm) + at[x] * 2) : make_uint2(0u, 0u);
            weight[x][0] = unpack_two<T>(w.x);
            weight[x][1] = unpack_two<T>(w.y);
        }
    const char* from = KIND == 0 ? a.q + t * a.q_row : KIND == 1 ? a.k + t * a.k_row : a.v + t * a.v_row;
    const uint64_t head_bytes = KIND == 0 ? a.q_head : KIND == 1 ? a.k_head : a.v_head;
#pragma unroll 1
    for (uint32_t it = first; it < last; it += WRITE_UNROLL) {
        uint2 raw[WRITE_UNROLL][4];
#pragma unroll
        for (int u = 0; u < WRITE_UNROLL; u++) {
            const uint32_t h = (it + u) * GROUPS + group;
            const char* p = from + h * head_bytes;
            const bool there = it + u < last && h < heads;
#pragma unroll
            for (int x = 0; x < 4; x++)
                raw[u][x] = there && holds[x >> 1] ? __ldcs(reinterpret_cast<const uint2*>(p + at[x] * 2)) : make_uint2(0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < WRITE_UNROLL; u++) {
            if (it + u >= last) break;
            const uint32_t h = (it + u) * GROUPS + group;
            const bool there = h < heads;
            char* to = KIND == 0 ? a.q_out + t * a.qo_row + h * a.qo_head
                                 : POOL8 ? token + (KIND == 2 ? a.codes : 0u) + h * a.dim : token + ((KIND == 2 ? a.codes : 0u) + h * a.dim) * 2ull;
            if constexpr (KIND == 2 && !POOL8) {
                // values on their way unchanged keep their bits
#pragma unroll
                for (int x = 0; x < 4; x++)
                    if (there && holds[x >> 1]) *reinterpret_cast<uint2*>(to + at[x] * 2) = raw[u][x];
            } else {
                Two e[4][2];
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    e[x][0] = unpack_two<T>(raw[u][x].x);
                    e[x][1] = unpack_two<T>(raw[u][x].y);
                }
                float r = 1.f;
                if (KIND != 2 && norm) {
                    Two sums[2] = {two(0.f, 0.f), two(0.f, 0.f)};
#pragma unroll
                    for (int x = 0; x < 4; x++)
#pragma unroll
                        for (int y = 0; y < 2; y++) sums[y] = fma(e[x][y], e[x][y], sums[y]);
                    const float2 s0 = apart(sums[0]), s1 = apart(sums[1]);
                    float sum = (s0.x + s0.y) + (s1.x + s1.y);
#pragma unroll
                    for (int d = 1; d < L; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
                    float eps = a.eps;
                    // squares that leave 32 bits, or are too small for all of their bits: both are rare, and the head of a power
                    // of two has the same norm
                    const bool large = sum > SUM_MAX, small = sum < SUM_MIN && eps < SUM_MIN;
                    if (__any_sync(0xFFFFFFFFu, large || small)) {
                        const float f = large ? 0x1p-70f : small ? 0x1p70f : 1.f;
                        const Two f2 = two(f, f);
                        float again = 0.f;
#pragma unroll
                        for (int x = 0; x < 4; x++)
#pragma unroll
                            for (int y = 0; y < 2; y++) {
                                e[x][y] = mul(e[x][y], f2);
                                const float2 m = apart(e[x][y]);
                                again = fmaf(m.x, m.x, fmaf(m.y, m.y, again));
                            }
#pragma unroll
                        for (int d = 1; d < L; d <<= 1) again += __shfl_xor_sync(0xFFFFFFFFu, again, d);
                        if (large || small) {
                            sum = again;
                            eps = eps * f * f;
                        }
                    }
                    r = rsqrtf(sum * a.inv_dim + eps);
#pragma unroll
                    for (int x = 0; x < 4; x++)
#pragma unroll
                        for (int y = 0; y < 2; y++) e[x][y] = mul(e[x][y], weight[x][y]);
                }
                if (KIND != 2) {
#pragma unroll
                    for (int x = 0; x < 2; x++)
                        if (own.turns[x]) {
                            // p: the first elements of 4 pairs, q: the second ones
                            Two p[2], q[2];
                            if constexpr (PAIRED) {
#pragma unroll
                                for (int y = 0; y < 2; y++) {
                                    const float2 m = apart(e[2 * x + y][0]), n = apart(e[2 * x + y][1]);
                                    p[y] = two(m.x, n.x);
                                    q[y] = two(m.y, n.y);
                                }
                            } else {
#pragma unroll
                                for (int y = 0; y < 2; y++) { p[y] = e[2 * x][y]; q[y] = e[2 * x + 1][y]; }
                            }
#pragma unroll
                            for (int y = 0; y < 2; y++) {
                                const Two c = cosines[2 * x + y], s = sines[2 * x + y];
                                Two minus;
                                minus.v = s.v ^ 0x8000000080000000ull;
                                const Two u0 = fma(q[y], minus, mul(p[y], c)), v0 = fma(p[y], s, mul(q[y], c));
                                p[y] = u0;
                                q[y] = v0;
                            }
                            if constexpr (PAIRED) {
#pragma unroll
                                for (int y = 0; y < 2; y++) {
                                    const float2 m = apart(p[y]), n = apart(q[y]);
                                    e[2 * x + y][0] = two(m.x, n.x);
                                    e[2 * x + y][1] = two(m.y, n.y);
                                }
                            } else {
#pragma unroll
                                for (int y = 0; y < 2; y++) { e[2 * x][y] = p[y]; e[2 * x + 1][y] = q[y]; }
                            }
                        }
                }
                if (!CODES) {
                    const Two r2 = two(r, r);
#pragma unroll
                    for (int x = 0; x < 4; x++)
                        if (there && holds[x >> 1]) {
                            const float2 m = apart(norm ? mul(e[x][0], r2) : e[x][0]), n = apart(norm ? mul(e[x][1], r2) : e[x][1]);
                            const bool same = !norm && !own.turns[x >> 1];
                            *reinterpret_cast<uint2*>(to + at[x] * 2) = same ? raw[u][x] : make_uint2(pack_pair<T>(m.x, m.y), pack_pair<T>(n.x, n.y));
                        }
                } else {
                    float top = 0.f;
#pragma unroll
                    for (int x = 0; x < 4; x++)
#pragma unroll
                        for (int y = 0; y < 2; y++) {
                            const float2 m = apart(e[x][y]);
                            top = top_of(top, top_of(m.x, m.y));
                        }
#pragma unroll
                    for (int d = 1; d < L; d <<= 1) top = top_of(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                    top *= r;
                    const bool fine = top <= FLT_MAX;                 // neither infinite nor NaN
                    // 1 / 448 and the reciprocal are off by 2^-24 and 2^-23: as much for a value that lies so near the middle of two codes
                    const float scale = fmaxf(top * (1.f / CODE_MAX), LEAST_SCALE);
                    float inv = __frcp_rn(scale);
                    if (KIND == 1) {
                        // a head of zeros, or nearly: the two factors in one leave 32 bits
                        const float both = inv * r;
                        const bool far = both > FLT_MAX;
                        if (__any_sync(0xFFFFFFFFu, far)) {
                            const Two f2 = far ? two(r, r) : two(1.f, 1.f);
#pragma unroll
                            for (int x = 0; x < 4; x++)
#pragma unroll
                                for (int y = 0; y < 2; y++) e[x][y] = mul(e[x][y], f2);
                        }
                        if (!far) inv = both;
                    }
                    const Two inv2 = two(inv, inv);
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const float2 m = apart(mul(e[x][0], inv2)), n = apart(mul(e[x][1], inv2));
                        const uint32_t w = floats_to_codes(m.x, m.y) | floats_to_codes(n.x, n.y) << 16;
                        if (there && holds[x >> 1]) *reinterpret_cast<uint32_t*>(to + at[x]) = fine ? w : 0u;      // 0 * inf is no code
                    }
                    if (there && j == 0) {
                        float* scales = reinterpret_cast<float*>(token + 2ull * a.codes);
                        scales[2 * h + (KIND == 2 ? 1 : 0)] = fine ? scale : __uint_as_float(0x7FC00000u);
                        // what lies behind the scales of an odd number of heads
                        if (KIND == 2 && h + 1 == a.kv_heads && (a.kv_heads & 1u)) scales[2 * h + 2] = scales[2 * h + 3] = 0.f;
                    }
                }
            }
        }
    }
}

template <class T, bool POOL8, int L, bool PAIRED>
__global__ void __launch_bounds__(ROW_THREADS, 2) kv_write_kernel(const __grid_constant__ WriteArgs a)
{
    const uint32_t lane = threadIdx.x & 31, j = lane % L, group = lane / L;
    const uint32_t n_warps = gridDim.x * (ROW_THREADS / 32);
    Lane own;
#pragma unroll
    for (int x = 0; x < 2; x++) {
        const uint32_t quad = 2 * j + x;
        own.turns[x] = 4 * quad < a.n_freq;
        own.holds[x] = 8 * quad < a.dim;
        const bool halves = own.turns[x] && !PAIRED;
        own.at[2 * x] = halves ? 4 * quad : 8 * quad;
        own.at[2 * x + 1] = halves ? a.n_freq + 4 * quad : 8 * quad + 4;
    }
    for (uint64_t task = blockIdx.x * (ROW_THREADS / 32) + (threadIdx.x >> 5); task < a.tasks; task += n_warps) {
        const uint32_t t = a.parts == 1 ? (uint32_t)task : (uint32_t)(task / a.parts), part = (uint32_t)(task - (uint64_t)t * a.parts);
        const int64_t slot = a.slots[t];
        uint32_t st = 0u;
        if (slot != -1) {
            if (slot < 0 || slot >= (int64_t)a.n_slots) st = GIFT_ST_BAD_DESC;
            else if (a.owner_map) st = label_write_status(a.owner_map[a.page.quot((uint32_t)slot)], a.row_owner[t]);
        }
        if (part == 0 && lane == 0) a.status[t] = st;
        if (st != 0u || slot == -1) continue;
        char* token = a.pages + (uint64_t)slot * a.token_bytes;
        const uint32_t r0 = part * a.iters, r1 = r0 + a.iters;

        Two cosines[4], sines[4];
        if (a.n_freq && r0 < a.q_rounds + a.kv_rounds) {
            constexpr int OWN = L / 4;                 // angles that a group works out
            float2 mine[OWN];
#pragma unroll
            for (int y = 0; y < OWN; y++) {
                const uint32_t f = 8 * j + group * OWN + y;
                uint32_t axis = 0;
#pragma unroll
                for (int x = 0; x < (int)GIFT_MAX_AXES - 1; x++) axis += f >= a.ends[x];
                mine[y] = f < a.n_freq ? turn(a.pos[axis * a.pos_stride + t], a.freq[f]) : make_float2(1.f, 0.f);
            }
            float c[8], s[8];
#pragma unroll
            for (int y = 0; y < 8; y++) {
                c[y] = __shfl_sync(0xFFFFFFFFu, mine[y % OWN].x, y / OWN * L + j);
                s[y] = __shfl_sync(0xFFFFFFFFu, mine[y % OWN].y, y / OWN * L + j);
            }
#pragma unroll
            for (int y = 0; y < 4; y++) {
                cosines[y] = two(c[2 * y], c[2 * y + 1]);
                sines[y] = two(s[2 * y], s[2 * y + 1]);
            }
        }
        const uint32_t k0 = a.q_rounds, v0 = k0 + a.kv_rounds, end = v0 + a.kv_rounds;
        write_heads<T, POOL8, L, PAIRED, 0>(a, own, t, token, r0, min(r1, k0), cosines, sines);
        write_heads<T, POOL8, L, PAIRED, 1>(a, own, t, token, max(r0, k0) - k0, max(min(r1, v0), k0) - k0, cosines, sines);
        write_heads<T, POOL8, L, PAIRED, 2>(a, own, t, token, max(r0, v0) - v0, max(min(r1, end), v0) - v0, cosines, sines);
    }
}

template <class T, bool POOL8, bool PAIRED>
void launch_write(const WriteArgs& a, uint32_t lanes, uint32_t grid, cudaStream_t st)
{
    if (lanes == 4) kv_write_kernel<T, POOL8, 4, PAIRED><<<grid, ROW_THREADS, 0, st>>>(a);
    else if (lanes == 8) kv_write_kernel<T, POOL8, 8, PAIRED><<<grid, ROW_THREADS, 0, st>>>(a);
    else kv_write_kernel<T, POOL8, 16, PAIRED><<<grid, ROW_THREADS, 0, st>>>(a);
}
template <class T>
void launch_write(const WriteArgs& a, bool pool8, bool paired, uint32_t lanes, uint32_t grid, cudaStream_t st)
{
    if (pool8) paired ? launch_write<T, true, true>(a, lanes, grid, st) : launch_write<T, true, false>(a, lanes, grid, st);
    else paired ? launch_write<T, false, true>(a, lanes, grid, st) : launch_write<T, false, false>(a, lanes, grid, st);
}

// ---------------------------------------------------------------------------
// reading
// ---------------------------------------------------------------------------
//
// The same copy the other way: a thread takes 8 elements of K and of V of a head, 2 such places at a time (one at a time: 237 us).
// 41 000 tokens of 32 heads of 128 from 8 bits: 182 us, 5.6 TB/s, 85 % of a copy.

struct ReadArgs {
    const char* pages;
    uint64_t token_bytes;
    uint32_t codes;
    char *k, *v;
    uint64_t k_row, k_head, v_row, v_head;   // strides in bytes
    const int64_t* slots;
    const int32_t* row_owner;
    const int32_t* owner_map;
    uint32_t* status;
    uint32_t n_rows, n_slots;
    FixedDiv page, head;                     // by page_tokens, by chunks of one head
    uint32_t head_chunks, chunks;            // of one head, of K (or V) of one token
    uint32_t lanes, rows_per_cta;            // threads that share a row, rows a CTA has in flight at once
};

template <class T> __device__ __forceinline__ uint4 values8(uint32_t lo, uint32_t hi, float scale)
{
    uint4 r;
    uint32_t* out = &r.x;
#pragma unroll
    for (int x = 0; x < 4; x++) {
        const uint32_t two = codes_to_half2((x < 2 ? lo : hi) >> (16 * (x & 1)) & 0xFFFFu);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&two));
        out[x] = pack_pair<T>(f.x * scale, f.y * scale);
    }
    return r;
}

template <class T, bool POOL8>
__global__ void __launch_bounds__(ROW_THREADS) kv_read_kernel(const __grid_constant__ ReadArgs a)
{
    const uint32_t sub = threadIdx.x / a.lanes, lane = threadIdx.x - sub * a.lanes;
    if (sub >= a.rows_per_cta) return;
    for (uint64_t t = (uint64_t)blockIdx.x * a.rows_per_cta + sub; t < a.n_rows; t += (uint64_t)gridDim.x * a.rows_per_cta) {
        const int64_t slot = a.slots[t];
        uint32_t st = 0u;
        if (slot != -1) {
            if (slot < 0 || slot >= (int64_t)a.n_slots) st = GIFT_ST_BAD_DESC;
            else if (a.owner_map) st = label_read_status(a.owner_map[a.page.quot((uint32_t)slot)], a.row_owner[t]);
        }
        if (lane == 0) a.status[t] = st;
        if (slot == -1) continue;
        const char* token = a.pages + (st ? 0ull : (uint64_t)slot * a.token_bytes);
        for (uint32_t x0 = lane; x0 < a.chunks; x0 += 2 * a.lanes) {
            uint4 kv[2][2];
#pragma unroll
            for (int y = 0; y < 2; y++) {
                const uint32_t x = x0 + y * a.lanes;
                kv[y][0] = kv[y][1] = make_uint4(0u, 0u, 0u, 0u);
                if (x >= a.chunks || st != 0u) continue;
                if constexpr (POOL8) {
                    const uint2 k = __ldcs(reinterpret_cast<const uint2*>(token) + x), v = __ldcs(reinterpret_cast<const uint2*>(token + a.codes) + x);
                    const uint2 scales = *reinterpret_cast<const uint2*>(token + 2ull * a.codes + a.head.quot(x) * 8u);
                    kv[y][0] = make_uint4(k.x, k.y, scales.x, 0u);
                    kv[y][1] = make_uint4(v.x, v.y, scales.y, 0u);
                } else {
                    kv[y][0] = __ldcs(reinterpret_cast<const uint4*>(token) + x);
                    kv[y][1] = __ldcs(reinterpret_cast<const uint4*>(token + 2ull * a.codes) + x);
                }
            }
#pragma unroll
            for (int y = 0; y < 2; y++) {
                const uint32_t x = x0 + y * a.lanes;
                if (x >= a.chunks) break;
                const uint32_t h = a.head.quot(x), o = x - h * a.head_chunks;
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    char* to = z ? a.v + t * a.v_row + (uint64_t)h * a.v_head + o * 16 : a.k + t * a.k_row + (uint64_t)h * a.k_head + o * 16;
                    const uint4 w = kv[y][z];
                    __stcs(reinterpret_cast<uint4*>(to), POOL8 ? values8<T>(w.x, w.y, __uint_as_float(w.z)) : w);
                }
            }
        }
    }
}

int rows_dtype_ok(const gift_kv_pool* pool, uint32_t dtype)
{
    if (dtype != GIFT_BF16 && dtype != GIFT_FP16) return GIFT_E_INVAL;
    return pool->dtype == GIFT_E4M3 || pool->dtype == dtype ? GIFT_OK : GIFT_E_INVAL;
}

// Rows that share memory cannot all be written.
bool writable(uint64_t row, uint64_t head, uint32_t n_rows, uint32_t n_heads)
{
    return (n_rows <= 1 || row != 0) && (n_heads <= 1 || head != 0);
}

}  // namespace

extern "C" int gift_kv_write(gift_ctx* c, const gift_kv_pool* pool, const gift_kv_rows* rows, const int64_t* slots,
                             const int32_t* row_owner, uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    int rc = any_pool_args_ok(pool);
    if (rc != GIFT_OK) return rc;
    if (!rows) return GIFT_E_INVAL;
    if (pool->head_dim > 256u) return GIFT_E_RANGE;
    if ((rc = rows_dtype_ok(pool, rows->dtype)) != GIFT_OK) return rc;
    if (rows->flags & ~GIFT_ROTATE_PAIRS) return GIFT_E_INVAL;
    if (!(rows->eps >= 0.f) || isinf(rows->eps)) return GIFT_E_INVAL;
    if (rows->n_freq) {
        if (!rows->freq || !rows->pos || rows->n_axes == 0) return GIFT_E_INVAL;
        if (rows->n_axes > GIFT_MAX_AXES || rows->n_freq > pool->head_dim / 2) return GIFT_E_RANGE;
        if (rows->n_freq % 4) return GIFT_E_ALIGN;
        uint64_t sum = 0;
        for (uint32_t x = 0; x < rows->n_axes; x++) sum += rows->sections[x];
        if (sum != rows->n_freq) return GIFT_E_INVAL;
    }
    if (((uintptr_t)rows->q_norm & 15) || ((uintptr_t)rows->k_norm & 15)) return GIFT_E_ALIGN;
    if (!rows->q && (rows->q_out || rows->q_norm)) return GIFT_E_INVAL;
    if (rows->q && (rows->n_heads == 0 || !rows->q_out)) return GIFT_E_INVAL;
    if (rows->q && rows->n_heads > GIFT_MAX_HEADS) return GIFT_E_RANGE;
    if (rows->n_rows > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (rows->n_rows == 0) return GIFT_OK;
    if (!slots || !status || (pool->owner_map && !row_owner)) return GIFT_E_INVAL;
    if ((rc = rows_args_ok(rows->k, rows->k_row_stride, rows->k_head_stride)) != GIFT_OK) return rc;
    if ((rc = rows_args_ok(rows->v, rows->v_row_stride, rows->v_head_stride)) != GIFT_OK) return rc;
    if (rows->q) {
        if ((rc = rows_args_ok(rows->q, rows->q_row_stride, rows->q_head_stride)) != GIFT_OK) return rc;
        if ((rc = rows_args_ok(rows->q_out, rows->q_out_row_stride, rows->q_out_head_stride)) != GIFT_OK) return rc;
        if (!writable(rows->q_out_row_stride, rows->q_out_head_stride, rows->n_rows, rows->n_heads)) return GIFT_E_INVAL;
    }
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    const bool pool8 = pool->dtype == GIFT_E4M3;
    WriteArgs a;
    memset(&a, 0, sizeof(a));
    a.q = static_cast<const char*>(rows->q); a.q_row = rows->q_row_stride * 2; a.q_head = rows->q_head_stride * 2;
    a.k = static_cast<const char*>(rows->k); a.k_row = rows->k_row_stride * 2; a.k_head = rows->k_head_stride * 2;
    a.v = static_cast<const char*>(rows->v); a.v_row = rows->v_row_stride * 2; a.v_head = rows->v_head_stride * 2;
    a.q_out = static_cast<char*>(rows->q_out); a.qo_row = rows->q_out_row_stride * 2; a.qo_head = rows->q_out_head_stride * 2;
    a.pages = static_cast<char*>(pool->pages);
    a.codes = pool->n_heads * pool->head_dim;
    a.token_bytes = pool8 ? kv8_layout(pool).token : (uint64_t)a.codes * 4;
    a.slots = slots; a.row_owner = row_owner; a.owner_map = pool->owner_map; a.status = status;
    a.n_rows = rows->n_rows; a.n_slots = pool->n_pages * pool->page_tokens; a.dim = pool->head_dim;
    a.q_heads = rows->q ? rows->n_heads : 0u; a.kv_heads = pool->n_heads;
    a.page = fixed_div(pool->page_tokens);
    a.q_norm = rows->q_norm; a.k_norm = rows->k_norm; a.eps = rows->eps; a.inv_dim = 1.f / pool->head_dim;
    a.n_freq = rows->n_freq;
    uint32_t end = 0;
    for (uint32_t x = 0; x < GIFT_MAX_AXES; x++) {
        end += x < rows->n_axes && rows->n_freq ? rows->sections[x] : 0u;
        a.ends[x] = x + 1 < rows->n_axes ? end : 0xFFFFFFFFu;
    }
    a.freq = rows->freq; a.pos = rows->pos; a.pos_stride = rows->pos_stride;
    const uint32_t lanes = a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16, groups = 32 / lanes;
    a.q_rounds = (a.q_heads + groups - 1) / groups;
    a.kv_rounds = (a.kv_heads + groups - 1) / groups;
    const uint32_t rounds = a.q_rounds + 2 * a.kv_rounds;
    // a warp takes a whole row where the rows fill the GPU, a share of one where they do not, so many rounds
    // at least as it has under way at once
    const uint64_t warps = 16ull * c->num_sms;
    uint64_t parts = (warps + a.n_rows - 1) / a.n_rows;
    const uint32_t most = (rounds + WRITE_UNROLL - 1) / WRITE_UNROLL;
    if (parts > most) parts = most;
    a.iters = (uint32_t)((rounds + parts - 1) / parts);
    a.parts = (rounds + a.iters - 1) / a.iters;
    a.tasks = (uint64_t)a.n_rows * a.parts;
    const uint64_t ctas = (a.tasks + ROW_THREADS / 32 - 1) / (ROW_THREADS / 32), fit = 2ull * c->num_sms;
    const uint32_t grid = (uint32_t)(ctas < fit ? ctas : fit);
    cudaStream_t st = (cudaStream_t)stream;
    const bool paired = rows->flags & GIFT_ROTATE_PAIRS;
    if (rows->dtype == GIFT_BF16) launch_write<__nv_bfloat16>(a, pool8, paired, lanes, grid, st);
    else launch_write<__half>(a, pool8, paired, lanes, grid, st);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

extern "C" int gift_kv_read(gift_ctx* c, const gift_kv_pool* pool, uint32_t dtype, uint32_t n_rows, const int64_t* slots,
                            const int32_t* row_owner, void* k, uint64_t k_row_stride, uint64_t k_head_stride, void* v,
                            uint64_t v_row_stride, uint64_t v_head_stride, uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    int rc = any_pool_args_ok(pool);
    if (rc != GIFT_OK) return rc;
    if ((rc = rows_dtype_ok(pool, dtype)) != GIFT_OK) return rc;
    if (n_rows > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (n_rows == 0) return GIFT_OK;
    if (!slots || !status || (pool->owner_map && !row_owner)) return GIFT_E_INVAL;
    if ((rc = rows_args_ok(k, k_row_stride, k_head_stride)) != GIFT_OK) return rc;
    if ((rc = rows_args_ok(v, v_row_stride, v_head_stride)) != GIFT_OK) return rc;
    if (!writable(k_row_stride, k_head_stride, n_rows, pool->n_heads) || !writable(v_row_stride, v_head_stride, n_rows, pool->n_heads))
        return GIFT_E_INVAL;
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    const bool pool8 = pool->dtype == GIFT_E4M3;
    ReadArgs a;
    memset(&a, 0, sizeof(a));
    a.pages = static_cast<const char*>(pool->pages);
    a.codes = pool->n_heads * pool->head_dim;
    a.token_bytes = pool8 ? kv8_layout(pool).token : (uint64_t)a.codes * 4;
    a.k = static_cast<char*>(k); a.k_row = k_row_stride * 2; a.k_head = k_head_stride * 2;
    a.v = static_cast<char*>(v); a.v_row = v_row_stride * 2; a.v_head = v_head_stride * 2;
    a.slots = slots; a.row_owner = row_owner; a.owner_map = pool->owner_map; a.status = status;
    a.n_rows = n_rows; a.n_slots = pool->n_pages * pool->page_tokens;
    a.page = fixed_div(pool->page_tokens);
    a.head_chunks = pool->head_dim / 8;
    a.head = fixed_div(a.head_chunks);
    a.chunks = pool->n_heads * a.head_chunks;
    // two places a thread and row
    a.lanes = (a.chunks + 1) / 2 < (uint32_t)ROW_THREADS ? (a.chunks + 1) / 2 : (uint32_t)ROW_THREADS;
    a.rows_per_cta = ROW_THREADS / a.lanes;
    const uint64_t tiles = ((uint64_t)n_rows + a.rows_per_cta - 1) / a.rows_per_cta, fit = 8ull * c->num_sms;
    const uint32_t grid = (uint32_t)(tiles < fit ? tiles : fit);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == GIFT_BF16) {
        if (pool8) kv_read_kernel<__nv_bfloat16, true><<<grid, ROW_THREADS, 0, st>>>(a);
        else kv_read_kernel<__nv_bfloat16, false><<<grid, ROW_THREADS, 0, st>>>(a);
    } else {
        if (pool8) kv_read_kernel<__half, true><<<grid, ROW_THREADS, 0, st>>>(a);
        else kv_read_kernel<__half, false><<<grid, ROW_THREADS, 0, st>>>(a);
    }
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}
