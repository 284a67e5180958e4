// Rows on their way into the labelled pages and out of them: norms of the heads, rotary positions and 8-bit
// codes in the pass that writes, values in the pass that reads.
#include <cuda_runtime.h>
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
constexpr float LEAST_SCALE = 1.17549435e-38f;   // 2^-126: a scale and its reciprocal are normal numbers
constexpr int WRITE_UNROLL = 4;                  // heads that a group of lanes has under way

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
// A pass over the rows: every byte is read once and written once, and HBM bandwidth bounds it.  A head is a
// group of L lanes with 8 elements each (L = 8, 16 or 32); where halves of a head turn against one
// another a lane holds 4 elements of each half, so that a pair never leaves its lane, and the 4 angles of
// a lane are the same for all heads of a row: they are worked out once per row and warp and stay in
// registers.  A warp takes a share of a row's heads, the whole row where rows abound.

struct WriteArgs {
    const char *q, *k, *v;
    uint64_t q_row, q_head, k_row, k_head, v_row, v_head;    // strides in bytes
    char* q_out;
    uint64_t qo_row, qo_head;
    char* pages;
    uint64_t token_bytes;
    uint32_t codes;                          // bytes of K's (or V's) elements of one token
    const int64_t* slots;
    const int32_t* row_owner;
    const int32_t* owner_map;
    uint32_t* status;
    uint32_t n_rows, n_slots, dim;
    uint32_t q_heads, kv_heads, units;       // units: heads of q, of k, of v
    uint32_t parts, iters;                   // warps that share a row, rounds of each
    uint64_t tasks;
    FixedDiv page;
    const void *q_norm, *k_norm;
    float eps, inv_dim;
    uint32_t n_freq, pairs;
    uint32_t ends[GIFT_MAX_AXES];            // first pair of the next axis
    const float* freq;
    const int32_t* pos;
    uint64_t pos_stride;
};

// cos and sin of pos * freq: the product in 64 bits (a position of 2^20 times a 32-bit frequency has no 32-bit
// place for its fraction of a turn), reduced to half a turn either way, the rest in 32 bits.
__device__ __forceinline__ void turn(int32_t pos, float freq, float& c, float& s)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189535;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
}

template <class T, bool POOL8, int L>
__global__ void __launch_bounds__(ROW_THREADS) kv_write_kernel(const __grid_constant__ WriteArgs a)
{
    constexpr uint32_t GROUPS = 32 / L;
    const uint32_t lane = threadIdx.x & 31, j = lane % L, group = lane / L;
    const uint32_t n_warps = gridDim.x * (ROW_THREADS / 32);
    const bool holds = j * 8 < a.dim, turns = j * 8 < 2 * a.n_freq;
    // a lane's two runs of 4 elements: next to one another, or in the two halves that turn
    const bool apart = turns && !a.pairs;
    const uint32_t lo_turned = apart ? 4 * j : 8 * j, hi_turned = apart ? a.n_freq + 4 * j : 8 * j + 4;

    for (uint64_t task = blockIdx.x * (ROW_THREADS / 32) + (threadIdx.x >> 5); task < a.tasks; task += n_warps) {
        const uint32_t t = (uint32_t)(task / a.parts), part = (uint32_t)(task - (uint64_t)t * a.parts);
        const int64_t slot = a.slots[t];
        uint32_t st = 0u;
        if (slot != -1) {
            if (slot < 0 || slot >= (int64_t)a.n_slots) st = GIFT_ST_BAD_DESC;
            else if (a.owner_map) st = label_write_status(a.owner_map[a.page.quot((uint32_t)slot)], a.row_owner[t]);
        }
        if (part == 0 && lane == 0) a.status[t] = st;
        if (st != 0u || slot == -1) continue;
        char* token = a.pages + (uint64_t)slot * a.token_bytes;

        float c[4], s[4];
        if (turns) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t f = 4 * j + i;
                uint32_t axis = 0;
#pragma unroll
                for (int x = 0; x < (int)GIFT_MAX_AXES - 1; x++) axis += f >= a.ends[x];
                turn(a.pos[axis * a.pos_stride + t], a.freq[f], c[i], s[i]);
            }
        }
#pragma unroll 1
        for (uint32_t it = part * a.iters; it < (part + 1) * a.iters; it += WRITE_UNROLL) {
            uint2 raw[WRITE_UNROLL][2];
#pragma unroll
            for (int x = 0; x < WRITE_UNROLL; x++) {
                const uint32_t u = (it + x) * GROUPS + group;
                raw[x][0] = raw[x][1] = make_uint2(0u, 0u);
                if (it + x >= (part + 1) * a.iters || u >= a.units || !holds) continue;
                const bool is_q = u < a.q_heads, is_v = u >= a.q_heads + a.kv_heads;
                const char* p = is_q ? a.q + t * a.q_row + u * a.q_head
                                     : is_v ? a.v + t * a.v_row + (u - a.q_heads - a.kv_heads) * a.v_head
                                            : a.k + t * a.k_row + (u - a.q_heads) * a.k_head;
                raw[x][0] = __ldcs(reinterpret_cast<const uint2*>(p + (is_v ? 8 * j : lo_turned) * 2));
                raw[x][1] = __ldcs(reinterpret_cast<const uint2*>(p + (is_v ? 8 * j + 4 : hi_turned) * 2));
            }
#pragma unroll
            for (int x = 0; x < WRITE_UNROLL; x++) {
                const uint32_t u = (it + x) * GROUPS + group;
                const bool there = it + x < (part + 1) * a.iters && u < a.units;
                if (!__any_sync(0xFFFFFFFFu, there)) break;
                const bool is_q = u < a.q_heads, is_v = u >= a.q_heads + a.kv_heads;
                const uint32_t h = is_q ? u : is_v ? u - a.q_heads - a.kv_heads : u - a.q_heads;
                const uint32_t lo = is_v ? 8 * j : lo_turned, hi = is_v ? 8 * j + 4 : hi_turned;
                float e[8], z[8];
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const float2 m = unpack2<T>(raw[x][y].x), n = unpack2<T>(raw[x][y].y);
                    e[4 * y] = m.x; e[4 * y + 1] = m.y; e[4 * y + 2] = n.x; e[4 * y + 3] = n.y;
                }
                const void* norm = is_v ? nullptr : is_q ? a.q_norm : a.k_norm;
                if (a.q_norm || a.k_norm) {
                    float sum = 0.f;
#pragma unroll
                    for (int y = 0; y < 8; y++) sum += e[y] * e[y];
#pragma unroll
                    for (int d = 1; d < L; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
                    if (norm && holds) {
                        const float r = rsqrtf(sum * a.inv_dim + a.eps);
#pragma unroll
                        for (int y = 0; y < 2; y++) {
                            const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const char*>(norm) + (y ? hi : lo) * 2);
                            const float2 m = unpack2<T>(w.x), n = unpack2<T>(w.y);
                            e[4 * y] *= r * m.x; e[4 * y + 1] *= r * m.y; e[4 * y + 2] *= r * n.x; e[4 * y + 3] *= r * n.y;
                        }
                    }
                }
                if (turns && !is_v) {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        // elements (i, 4 + i), or neighbours
                        const float p = a.pairs ? e[2 * i] : e[i], r = a.pairs ? e[2 * i + 1] : e[4 + i];
                        z[i] = p * c[i] - r * s[i];
                        z[4 + i] = r * c[i] + p * s[i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++) e[i] = a.pairs ? z[(i & 1) * 4 + i / 2] : z[i];
                }
                if (!POOL8 || is_q) {
                    if (there && holds) {
                        char* to = is_q ? a.q_out + t * a.qo_row + h * a.qo_head : token + (is_v ? (uint64_t)a.codes * 2 : 0u) + (uint64_t)h * a.dim * 2;
                        // values on their way unchanged keep their bits
                        const bool same = is_v || (!norm && !turns);
                        *reinterpret_cast<uint2*>(to + lo * 2) = same ? raw[x][0] : make_uint2(pack_pair<T>(e[0], e[1]), pack_pair<T>(e[2], e[3]));
                        *reinterpret_cast<uint2*>(to + hi * 2) = same ? raw[x][1] : make_uint2(pack_pair<T>(e[4], e[5]), pack_pair<T>(e[6], e[7]));
                    }
                }
                if (POOL8 && __any_sync(0xFFFFFFFFu, there && !is_q)) {
                    // as whole numbers the magnitudes of infinities and NaN are above all others
                    uint32_t top = 0u;
#pragma unroll
                    for (int y = 0; y < 8; y++) {
                        const uint32_t m = __float_as_uint(e[y]) & 0x7FFFFFFFu;
                        top = m > top ? m : top;
                    }
#pragma unroll
                    for (int d = 1; d < L; d <<= 1) {
                        const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, top, d);
                        top = o > top ? o : top;
                    }
                    const bool fine = top < 0x7F800000u;
                    const float scale = fmaxf(__fdiv_rn(__uint_as_float(top), CODE_MAX), LEAST_SCALE);
                    const float inv = fine ? __frcp_rn(scale) : 0.f;
                    uint32_t w[2];
#pragma unroll
                    for (int y = 0; y < 2; y++)
                        w[y] = floats_to_codes(e[4 * y] * inv, e[4 * y + 1] * inv) | floats_to_codes(e[4 * y + 2] * inv, e[4 * y + 3] * inv) << 16;
                    if (!fine) w[0] = w[1] = 0u;                       // 0 * inf is no code
                    if (there && !is_q && holds) {
                        char* to = token + (is_v ? a.codes : 0u) + h * a.dim;
                        *reinterpret_cast<uint32_t*>(to + lo) = w[0];
                        *reinterpret_cast<uint32_t*>(to + hi) = w[1];
                        if (j == 0) {
                            float* scales = reinterpret_cast<float*>(token + 2ull * a.codes);
                            scales[2 * h + (is_v ? 1 : 0)] = fine ? scale : __uint_as_float(0x7FC00000u);
                            // what lies behind the scales of an odd number of heads
                            if (is_v && h + 1 == a.kv_heads && (a.kv_heads & 1u)) scales[2 * h + 2] = scales[2 * h + 3] = 0.f;
                        }
                    }
                }
            }
        }
    }
}

template <class T, bool POOL8>
void launch_write(const WriteArgs& a, uint32_t lanes, uint32_t grid, cudaStream_t st)
{
    if (lanes == 8) kv_write_kernel<T, POOL8, 8><<<grid, ROW_THREADS, 0, st>>>(a);
    else if (lanes == 16) kv_write_kernel<T, POOL8, 16><<<grid, ROW_THREADS, 0, st>>>(a);
    else kv_write_kernel<T, POOL8, 32><<<grid, ROW_THREADS, 0, st>>>(a);
}

// ---------------------------------------------------------------------------
// reading
// ---------------------------------------------------------------------------
//
// The same copy the other way: a thread takes 16 elements of K and of V of a head (8 of a 16-bit pool).

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
        for (uint32_t x = lane; x < a.chunks; x += a.lanes) {
            const uint32_t h = a.head.quot(x), o = x - h * a.head_chunks;
            char* k = a.k + t * a.k_row + (uint64_t)h * a.k_head + o * (POOL8 ? 32 : 16);
            char* v = a.v + t * a.v_row + (uint64_t)h * a.v_head + o * (POOL8 ? 32 : 16);
            if constexpr (POOL8) {
                uint4 kk = make_uint4(0u, 0u, 0u, 0u), vv = kk;
                float2 scale = make_float2(0.f, 0.f);
                if (st == 0u) {
                    kk = __ldcs(reinterpret_cast<const uint4*>(token) + x);
                    vv = __ldcs(reinterpret_cast<const uint4*>(token + a.codes) + x);
                    scale = *reinterpret_cast<const float2*>(token + 2ull * a.codes + h * 8u);
                }
                reinterpret_cast<uint4*>(k)[0] = values8<T>(kk.x, kk.y, scale.x);
                reinterpret_cast<uint4*>(k)[1] = values8<T>(kk.z, kk.w, scale.x);
                reinterpret_cast<uint4*>(v)[0] = values8<T>(vv.x, vv.y, scale.y);
                reinterpret_cast<uint4*>(v)[1] = values8<T>(vv.z, vv.w, scale.y);
            } else {
                uint4 kk = make_uint4(0u, 0u, 0u, 0u), vv = kk;
                if (st == 0u) {
                    kk = __ldcs(reinterpret_cast<const uint4*>(token) + x);
                    vv = __ldcs(reinterpret_cast<const uint4*>(token + 2ull * a.codes) + x);
                }
                *reinterpret_cast<uint4*>(k) = kk;
                *reinterpret_cast<uint4*>(v) = vv;
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
    a.q_heads = rows->q ? rows->n_heads : 0u; a.kv_heads = pool->n_heads; a.units = a.q_heads + 2 * a.kv_heads;
    a.page = fixed_div(pool->page_tokens);
    a.q_norm = rows->q_norm; a.k_norm = rows->k_norm; a.eps = rows->eps; a.inv_dim = 1.f / pool->head_dim;
    a.n_freq = rows->n_freq; a.pairs = rows->flags & GIFT_ROTATE_PAIRS;
    uint32_t end = 0;
    for (uint32_t x = 0; x < GIFT_MAX_AXES; x++) {
        end += x < rows->n_axes && rows->n_freq ? rows->sections[x] : 0u;
        a.ends[x] = x + 1 < rows->n_axes ? end : 0xFFFFFFFFu;
    }
    a.freq = rows->freq; a.pos = rows->pos; a.pos_stride = rows->pos_stride;
    const uint32_t lanes = a.dim <= 64 ? 8 : a.dim <= 128 ? 16 : 32, groups = 32 / lanes;
    const uint32_t rounds = (a.units + groups - 1) / groups;
    // a warp takes a whole row where the rows fill the GPU, a share of one where they do not, so many rounds
    // at least as it has under way at once
    const uint64_t warps = 32ull * c->num_sms;
    uint64_t parts = (warps + a.n_rows - 1) / a.n_rows;
    const uint32_t most = (rounds + WRITE_UNROLL - 1) / WRITE_UNROLL;
    if (parts > most) parts = most;
    a.iters = (uint32_t)((rounds + parts - 1) / parts);
    a.parts = (rounds + a.iters - 1) / a.iters;
    a.tasks = (uint64_t)a.n_rows * a.parts;
    const uint64_t ctas = (a.tasks + ROW_THREADS / 32 - 1) / (ROW_THREADS / 32), fit = 8ull * c->num_sms;
    const uint32_t grid = (uint32_t)(ctas < fit ? ctas : fit);
    cudaStream_t st = (cudaStream_t)stream;
    if (rows->dtype == GIFT_BF16) pool8 ? launch_write<__nv_bfloat16, true>(a, lanes, grid, st) : launch_write<__nv_bfloat16, false>(a, lanes, grid, st);
    else pool8 ? launch_write<__half, true>(a, lanes, grid, st) : launch_write<__half, false>(a, lanes, grid, st);
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
    a.head_chunks = pool->head_dim / (pool8 ? 16 : 8);
    a.head = fixed_div(a.head_chunks);
    a.chunks = pool->n_heads * a.head_chunks;
    a.lanes = a.chunks < (uint32_t)ROW_THREADS ? a.chunks : (uint32_t)ROW_THREADS;
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
