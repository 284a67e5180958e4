// Pieces that the attention kernels over 16-bit and over 8-bit pages share: the joining of cut items, the
// scratch, warp-level matrix primitives.  In an unnamed namespace: each file that includes this has its own
// kernels.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "gift_attn.cuh"
#include "gift_internal.cuh"

using namespace gift;

namespace {

constexpr int MOST_TILE_ROWS = 128;      // of an item, in any of the kernels

// ---------------------------------------------------------------------------
// joining the pieces of cut items
// ---------------------------------------------------------------------------

constexpr int JOIN_THREADS = 128;
constexpr int JOIN_ROWS = 16;

struct JoinShared {
    float2 top[JOIN_ROWS];
    uint32_t bits;
};

// 16 rows from row_lo of the item that begins in slice w: the item is that slice's last piece and goes on
// as the first piece of w + 1, w + 2, ...  Called by JOIN_THREADS threads.  LIVE: the pieces may have been written
// while this kernel runs, and are read past L1.
template <bool LIVE, class V> __device__ __forceinline__ V load_part(const V* p) { return LIVE ? __ldcg(p) : *p; }

template <class T, int D, int ROWS, bool LIVE>
__device__ __forceinline__ void join_rows(const AttnArgs& a, const PartHead& head, uint32_t w, uint32_t way, uint32_t row_lo, JoinShared* sh)
{
    constexpr int CH = D / 8;
    const uint32_t pieces = head.pieces, r = head.r, row0 = head.row0, h = head.h, q0 = head.q0 + row_lo;
    const uint32_t nr = head.nr - row_lo < (uint32_t)JOIN_ROWS ? head.nr - row_lo : (uint32_t)JOIN_ROWS;
    auto slot_of = [&](uint32_t p) -> uint64_t { return 2ull * ((w + p) * a.ways + way) + (p == 0 ? 1 : 0); };
    if (threadIdx.x == 0) sh->bits = 0u;
    __syncthreads();
    for (uint32_t p = threadIdx.x; p < pieces; p += JOIN_THREADS) {
        const uint32_t bits = load_part<LIVE>(&a.part_head[slot_of(p)].bits);
        if (bits) atomicOr(&sh->bits, bits);
    }
    // maxima and sums: 8 threads per row, pieces dealt among them
    {
        const uint32_t row = threadIdx.x >> 3, sub = threadIdx.x & 7u;
        float top = NEG_INF, sum = 0.f;
        if (row < nr)
            for (uint32_t p = sub; p < pieces; p += 8) {
                const float2 ml = load_part<LIVE>(&a.part_ml[slot_of(p) * ROWS + row_lo + row]);
                const float now = fmaxf(top, ml.x), use = now == NEG_INF ? 0.f : now;
                sum = sum * fast_exp2(top - use) + ml.y * fast_exp2(ml.x - use);
                top = now;
            }
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) {
            const float other_top = __shfl_xor_sync(0xFFFFFFFFu, top, d), other_sum = __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            const float now = fmaxf(top, other_top), use = now == NEG_INF ? 0.f : now;
            sum = sum * fast_exp2(top - use) + other_sum * fast_exp2(other_top - use);
            top = now;
        }
        if (row < nr && sub == 0) sh->top[row] = make_float2(top, sum);
    }
    __syncthreads();
    const uint32_t bits = sh->bits;
    for (uint32_t c = threadIdx.x; c < nr * (uint32_t)CH; c += JOIN_THREADS) {
        const uint32_t row = c / CH, ch = c % CH;
        const float top = sh->top[row].x, sum = sh->top[row].y, use = top == NEG_INF ? 0.f : top;
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; e++) acc[e] = 0.f;
#pragma unroll 4
        for (uint32_t p = 0; p < pieces; p++) {
            const uint64_t at = slot_of(p) * ROWS + row_lo + row;
            const float f = fast_exp2(load_part<LIVE>(&a.part_ml[at]).x - use);
            const float4* from = reinterpret_cast<const float4*>(a.part_o + at * D + ch * 8);
            const float4 x = load_part<LIVE>(from), y = load_part<LIVE>(from + 1);
            acc[0] += f * x.x; acc[1] += f * x.y; acc[2] += f * x.z; acc[3] += f * x.w;
            acc[4] += f * y.x; acc[5] += f * y.y; acc[6] += f * y.z; acc[7] += f * y.w;
        }
        const uint32_t rho = q0 + row, i = a.by_group.quot(rho), hq = h * a.group + (rho - i * a.group);
        const bool none = bits != 0u || sum == 0.f;
        const float inv = none ? 0.f : 1.f / sum;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (!none) {
            v.x = pack2<T>(acc[0] * inv, acc[1] * inv); v.y = pack2<T>(acc[2] * inv, acc[3] * inv);
            v.z = pack2<T>(acc[4] * inv, acc[5] * inv); v.w = pack2<T>(acc[6] * inv, acc[7] * inv);
        }
        *reinterpret_cast<uint4*>(a.out + (uint64_t)(row0 + i) * a.out_row + (uint64_t)hq * a.out_head + ch * 16) = v;
        if (a.lse && ch == 0) a.lse[(uint64_t)(row0 + i) * a.heads + hq] = none ? NEG_INF : (top + log2f(sum)) * 0.6931471805599453f;
    }
    if (h == 0 && q0 == 0) write_request<JOIN_THREADS>(a, r, row0, head.rows_m, bits);
}

// The same from within the attention kernel, kept out of its loops' code.
template <class T, int D, int ROWS>
__device__ __noinline__ void join_here(const AttnArgs& a, const PartHead& head, uint32_t w, JoinShared* sh)
{
    join_rows<T, D, ROWS, true>(a, head, w, 0, 0, sh);
}

// At the end of every CTA of the few-row kernel, when it takes no more tickets: the call's last CTA makes all
// tickets 0 for the next call.  The CTAs are counted, a number that only the launch fixes, so nothing that a
// call meets (lengths that change while it runs, a second call at the same time against the rule) is
// left to a later one; a counter in step with the grid returns to 0 by itself.
__device__ __forceinline__ void leave_tickets(const AttnArgs& a)
{
    if (threadIdx.x >= 32) return;
    bool last = false;
    if (threadIdx.x == 0) {
        __threadfence();                               // this CTA's tickets are taken
        last = atomicInc(a.tickets + a.n_slices, gridDim.x - 1u) == gridDim.x - 1u;
    }
    if (__shfl_sync(0xFFFFFFFFu, last, 0))
        for (uint32_t k = threadIdx.x; k < a.n_slices; k += 32) a.tickets[k] = 0u;
}

// ---------------------------------------------------------------------------
// warp-level primitives
// ---------------------------------------------------------------------------

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <class T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------
// launching
// ---------------------------------------------------------------------------

// What a wait that ran out leaves: a CTA knows of its own pieces only, so the requests that it could not
// finish become zero here, when all of the rows' writers are done, by all CTAs of the joining kernel.
template <int D>
__device__ __noinline__ void clear_stalled(const AttnArgs& a, uint32_t cta, uint32_t n_cta)
{
    constexpr uint32_t CH = D / 8;
#pragma unroll 1
    for (uint32_t k = 0; k < a.n_slices * a.ways; k++) {
        const uint4 s = __ldcg(a.part_stall + k);
        for (uint32_t r = s.x + cta * JOIN_THREADS + threadIdx.x; r < s.y; r += n_cta * JOIN_THREADS)
            if (load_shape(a.b, r).rows) a.status[r] = GIFT_ST_STALLED;
        for (uint32_t t = s.z + cta; t < s.w; t += n_cta) {
            for (uint32_t c = threadIdx.x; c < a.heads * CH; c += JOIN_THREADS) {
                const uint32_t hq = c / CH, ch = c % CH;
                *reinterpret_cast<uint4*>(a.out + (uint64_t)t * a.out_row + (uint64_t)hq * a.out_head + ch * 16) = make_uint4(0u, 0u, 0u, 0u);
                if (a.lse && ch == 0) a.lse[(uint64_t)t * a.heads + hq] = NEG_INF;
            }
            if (a.row_owner && threadIdx.x == 0) a.row_owner[t] = GIFT_OWNER_CONFLICT;
        }
    }
}

// Joins the pieces of the items that a slice boundary cuts, 16 rows per CTA.  CTAs (w, *, way) look
// after the item that slice w leaves unfinished, if it begins there.
template <class T, int D, int ROWS>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ JoinShared sh;
    const uint32_t w = blockIdx.x, row_lo = blockIdx.y * JOIN_ROWS, way = blockIdx.z;
    // until the attention kernel is complete and what it wrote can be seen
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const PartHead head = a.part_head[2u * (w * a.ways + way) + 1u];
    bool any = false, mine = false;
    for (uint32_t k = threadIdx.x; k < a.n_slices * a.ways; k += JOIN_THREADS) {
        const uint4 s = a.part_stall[k];
        any = any || s.y != 0u;
        mine = mine || (head.r >= s.x && head.r < s.y);
    }
    if (__syncthreads_or(any)) {
        clear_stalled<D>(a, blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), gridDim.x * gridDim.y * gridDim.z);
        if (__syncthreads_or(mine)) return;
    }
    if (head.pieces == 0 || row_lo >= head.nr) return;
    join_rows<T, D, ROWS, false>(a, head, w, way, row_lo, &sh);
}

// The joining kernel may start while the attention kernel runs: its launch is hidden behind it, and it
// waits for the pieces itself.
template <class T, int D, int ROWS>
cudaError_t launch_join(const AttnArgs& a, cudaStream_t st)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(a.n_slices - 1, ROWS / JOIN_ROWS, a.ways);
    cfg.blockDim = dim3(JOIN_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn_join_kernel<T, D, ROWS>, a);
}

// A kernel's shared-memory limit, raised once per device: the call costs as much as a launch's half.
template <auto KERNEL> cudaError_t allow_smem(int device, int bytes)
{
    static bool done[64];
    if (device < 0 || device >= 64) return cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (done[device]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    done[device] = e == cudaSuccess;
    return e;
}

// cuTensorMapEncodeTiled of the driver, looked up once: the library does not link against it.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int encode_tiled(EncodeTiled* out)
{
    static EncodeTiled fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        CU_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q));
        if (q != cudaDriverEntryPointSuccess || !p) return GIFT_E_CUDA;
        fn = reinterpret_cast<EncodeTiled>(p);
    }
    *out = fn;
    return GIFT_OK;
}

// Q as (columns, heads, rows): a box holds the group's heads of as many tokens as a tile of rows takes.
int map_of_q(const AttnArgs& a, bool half, uint32_t head_dim, CUtensorMap* map)
{
    EncodeTiled encode;
    const int rc = encode_tiled(&encode);
    if (rc != GIFT_OK) return rc;
    const cuuint64_t dims[3] = {head_dim, a.heads, a.n_rows};
    // the stride of a dimension of one entry is never used, but may not be 0
    const cuuint64_t strides[2] = {a.heads > 1 ? a.q_head : head_dim * 2, a.n_rows > 1 ? a.q_row : (cuuint64_t)a.heads * head_dim * 2};
    const cuuint32_t box[3] = {64, a.group, (cuuint32_t)(MOST_TILE_ROWS / a.group)}, steps[3] = {1, 1, 1};
    if (encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<char*>(a.q), dims, strides,
               box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return GIFT_E_CUDA;
    return GIFT_OK;
}

constexpr uint32_t PART_ROWS = MOST_TILE_ROWS;  // most rows of a tile of query rows
constexpr uint32_t PART_D = 128;
constexpr size_t MOST_CTAS = 3;          // per SM, in any of the kernels: slices
constexpr size_t PART_HEADS = 2 * MOST_CTAS;

// The scratch is allocated once, at a size that no call exceeds, and stays where it is until the
// ctx is destroyed: a captured graph that names it stays valid.  Not under a capture: the tickets' first
// zeros would then be the graph's to write, and calls before its first replay would find whatever was there.
int scratch_ensure(gift_ctx* c, cudaStream_t st)
{
    if (c->d_attn) return GIFT_OK;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    CU_TRY(cudaStreamIsCapturing(st, &capture));
    if (capture != cudaStreamCaptureStatusNone) return GIFT_E_INVAL;
    const size_t parts = 4ull * c->num_sms;
    const size_t before = parts * PART_ROWS * (PART_D * 4 + 8) + PART_HEADS * c->num_sms * sizeof(PartHead) + 2ull * c->num_sms * sizeof(uint4);
    const size_t tickets = (MOST_CTAS * c->num_sms + 1) * 4;
    void* p = nullptr;
    CU_TRY(cudaMalloc(&p, before + tickets));
    const cudaError_t e = cudaMemsetAsync(static_cast<char*>(p) + before, 0, tickets, st);     // tickets are 0 between calls
    if (e != cudaSuccess) {
        gift_note_cuda_error(e, __FILE__, __LINE__);
        cudaFree(p);
        return GIFT_E_CUDA;
    }
    c->d_attn = p;
    return GIFT_OK;
}

// Where the pieces go.
inline void use_scratch(gift_ctx* c, AttnArgs& a)
{
    const size_t parts = 4ull * c->num_sms;
    char* p = static_cast<char*>(c->d_attn);
    a.part_o = reinterpret_cast<float*>(p);
    a.part_ml = reinterpret_cast<float2*>(p + parts * PART_ROWS * PART_D * 4);
    a.part_head = reinterpret_cast<PartHead*>(p + parts * PART_ROWS * (PART_D * 4 + 8));
    a.part_stall = reinterpret_cast<uint4*>(a.part_head + PART_HEADS * c->num_sms);
    a.tickets = reinterpret_cast<uint32_t*>(a.part_stall + 2ull * c->num_sms);
}

}  // namespace
