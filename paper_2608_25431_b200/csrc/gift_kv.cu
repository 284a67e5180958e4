// K and V rows of a step into the labelled pages (the write side of the paged cache).  A copy:
// every byte of the rows is read once and written once, and HBM bandwidth bounds it.  The page's
// label decides, in the same pass, whether a row may be written (paper sec. 3 step 4: every
// byte has one owner), so no byte of another user's page is ever touched.  32 700 rows of 16 KiB:
// 178 us, 6.0 TB/s of 6.45 measured for a copy; 256 rows: 5 us.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "gift_internal.cuh"
#include "gift_kv.cuh"

using namespace gift;

namespace {

constexpr int APPEND_THREADS = 256;

struct AppendArgs {
    const uint4* k;
    const uint4* v;
    uint64_t k_row, k_head, v_row, v_head;   // strides in 16-byte chunks
    uint4* pages;
    const int64_t* slots;
    const int32_t* row_owner;
    const int32_t* owner_map;
    uint32_t* status;
    uint32_t n_rows, n_slots;
    FixedDiv page, head;                     // by page_tokens, by head_chunks
    uint32_t head_chunks;                    // 16-byte chunks of one head
    uint32_t half_chunks;                    // chunks of K (or of V) of one token
    uint32_t lanes;                          // threads that share a row
    uint32_t rows_per_cta;                   // rows a CTA has in flight at once
};

__device__ __forceinline__ uint32_t row_status(const AppendArgs& a, int64_t slot, uint32_t t)
{
    if (slot < 0 || slot >= (int64_t)a.n_slots) return GIFT_ST_BAD_DESC;
    if (!a.owner_map) return 0u;
    return label_write_status(a.owner_map[a.page.quot((uint32_t)slot)], a.row_owner[t]);
}

__global__ void __launch_bounds__(APPEND_THREADS) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    const uint32_t sub = threadIdx.x / a.lanes, lane = threadIdx.x - sub * a.lanes;
    if (sub >= a.rows_per_cta) return;
    for (uint32_t t = blockIdx.x * a.rows_per_cta + sub; t < a.n_rows; t += gridDim.x * a.rows_per_cta) {
        const int64_t slot = a.slots[t];
        if (slot == -1) {                    // a padded row, or a rejected draft
            if (lane == 0) a.status[t] = 0u;
            continue;
        }
        const uint32_t st = row_status(a, slot, t);
        if (lane == 0) a.status[t] = st;
        if (st != 0u) continue;
        // a token is K then V, each heads x head_dim: 2 * half_chunks contiguous chunks
        uint4* dst = a.pages + (uint64_t)slot * (2u * a.half_chunks);
        for (uint32_t c = lane; c < a.half_chunks; c += a.lanes) {
            const uint32_t h = a.head.quot(c), o = c - h * a.head_chunks;
            const uint4 kk = __ldcs(a.k + (uint64_t)t * a.k_row + (uint64_t)h * a.k_head + o);
            const uint4 vv = __ldcs(a.v + (uint64_t)t * a.v_row + (uint64_t)h * a.v_head + o);
            dst[c] = kk;
            dst[a.half_chunks + c] = vv;
        }
    }
}

}  // namespace

extern "C" int gift_kv_append(gift_ctx* c, const gift_kv_pool* pool, const void* k, uint64_t k_row_stride,
                              uint64_t k_head_stride, const void* v, uint64_t v_row_stride, uint64_t v_head_stride,
                              uint32_t n_rows, const int64_t* slots, const int32_t* row_owner, uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    int rc = pool_args_ok(pool);
    if (rc != GIFT_OK) return rc;
    if (n_rows == 0) return GIFT_OK;
    if (n_rows > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (!slots || !status || (pool->owner_map && !row_owner)) return GIFT_E_INVAL;
    if ((rc = rows_args_ok(k, k_row_stride, k_head_stride)) != GIFT_OK) return rc;
    if ((rc = rows_args_ok(v, v_row_stride, v_head_stride)) != GIFT_OK) return rc;
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    AppendArgs a;
    memset(&a, 0, sizeof(a));
    a.k = static_cast<const uint4*>(k); a.v = static_cast<const uint4*>(v);
    a.k_row = k_row_stride / 8; a.k_head = k_head_stride / 8; a.v_row = v_row_stride / 8; a.v_head = v_head_stride / 8;
    a.pages = static_cast<uint4*>(pool->pages);
    a.slots = slots; a.row_owner = row_owner; a.owner_map = pool->owner_map; a.status = status;
    a.n_rows = n_rows; a.n_slots = pool->n_pages * pool->page_tokens; a.page = fixed_div(pool->page_tokens);
    a.head_chunks = pool->head_dim / 8;
    a.head = fixed_div(a.head_chunks);
    a.half_chunks = pool->n_heads * a.head_chunks;
    a.lanes = a.half_chunks < (uint32_t)APPEND_THREADS ? a.half_chunks : (uint32_t)APPEND_THREADS;
    a.rows_per_cta = APPEND_THREADS / a.lanes;
    const uint64_t tiles = ((uint64_t)n_rows + a.rows_per_cta - 1) / a.rows_per_cta;
    const uint64_t most = 8ull * c->num_sms;
    kv_append_kernel<<<(uint32_t)(tiles < most ? tiles : most), APPEND_THREADS, 0, (cudaStream_t)stream>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}
