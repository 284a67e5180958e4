// Block tables, slot maps and segment tables from request lengths (paper sec. 4.2 on the KV
// blocks' ownership records, sec. 4.5 on the index tables that a rule needs without a blocking
// copy).  Everything is a prefix sum over at most GIFT_MAX_REQS requests followed by independent
// work per page, row or segment.  The prefix is cheap (a few thousand additions) and every CTA
// needs it, so each CTA computes it for itself: no second launch, no flag between CTAs.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "gift_batch.cuh"
#include "gift_internal.cuh"

namespace cg = cooperative_groups;
using namespace gift;

namespace {

// ---------------------------------------------------------------------------
// block tables
// ---------------------------------------------------------------------------
//
// One cluster of 16 CTAs (8 where the device cannot co-schedule 16), so that the stages (check and
// claim, commit labels and taken entries, push what is given back) can be separated by the
// cluster's hardware barrier.  What they touch is a word per page that changes hands and layer,
// scattered over the label map: latency bound when few pages change hands, bound by the 16 SMs'
// scattered accesses when many do.  2 to 32 threads share a page when there are threads to spare;
// a thread has 8 layers' labels under way at once, and what it needs of the page's request lies in
// shared memory.
//
// Stack and tables may be the untrusted side's and may be rewritten while the call runs, so a page is
// read once, by one of the threads that share it, and what was checked is what is committed: the threads keep
// the pages of their first BT_KEEP rounds in shared memory (131 072 pages with 16 CTAs).  Behind those a page is
// read again, and committed only if it is one that this call has claimed and not yet committed.
// 256 requests that take 16 pages in 32 layers: 12 us; 512 that take 4 000 and give back 700: 25 us (one
// thread per page and layer, the lengths read again for each, 8 CTAs: 107 us).
constexpr int BT_CTAS_PORTABLE = 8;
constexpr int BT_CTAS_LARGE = 16;
constexpr int BT_THREADS = 1024;
constexpr uint32_t BT_REQ_BYTES = 16;    // shared memory per request
constexpr uint32_t BT_KEEP = 8;          // rounds whose pages are kept
constexpr uint32_t BT_KEEP_BYTES = BT_KEEP * BT_THREADS * 4;
constexpr int BT_MAX_DEVICES = 64;

struct BlockArgs {
    BatchArgs b;
    int32_t* free_pages;
    int32_t* n_free;
    uint32_t free_cap;
    int32_t* owner_map;      // [layers][n_pages]
    uint32_t layers;
    uint32_t* status;
};

// What every CTA knows of the requests after the prefix sums.
struct BlockPlan {
    uint32_t* take;          // [n_req] exclusive prefix of the pages taken
    uint32_t* give;          // [n_req] exclusive prefix of the pages given back
    uint32_t* from;          // [n_req] first block taken, or given back
    int32_t* owner;          // [n_req]
    uint32_t taken;
    int32_t height;          // of the stack before the call
};

// One page that changes hands: item k < taken comes off the stack, the others go back to it.
struct PageMove {
    uint32_t r;
    uint64_t entry;          // its entry in the block tables
};

__device__ __forceinline__ PageMove page_move(const BlockArgs& a, const BlockPlan& p, uint32_t k)
{
    PageMove m;
    const bool take = k < p.taken;
    const uint32_t* first = take ? p.take : p.give;
    const uint32_t at = take ? k : k - p.taken;
    m.r = req_of(first, a.b.n_req, at);
    m.entry = (uint64_t)m.r * a.b.max_blocks + p.from[m.r] + (at - first[m.r]);
    return m;
}

// The page as the stack or the table has it now.
__device__ __forceinline__ int32_t page_named(const BlockArgs& a, const BlockPlan& p, uint32_t k, const PageMove& m)
{
    return k < p.taken ? __ldcg(a.free_pages + (p.height - 1 - (int32_t)k)) : __ldcg(a.b.table + m.entry);
}

__global__ void __launch_bounds__(BT_THREADS, 1)
block_tables_kernel(const __grid_constant__ BlockArgs a)
{
    extern __shared__ uint32_t dyn[];
    __shared__ uint64_t warp_sums[BT_THREADS / 32];
    __shared__ uint32_t s_bad;                          // CTA 0's copy is the cluster's
    __shared__ unsigned long long s_taken;
    __shared__ int32_t s_height;
    cg::cluster_group cl = cg::this_cluster();
    uint32_t* bad = cl.map_shared_rank(&s_bad, 0);
    // neighbouring warps of work go to different CTAs: a few pages are spread over the SMs
    const uint32_t n_cta = gridDim.x, tid = (threadIdx.x >> 5) * n_cta * 32 + blockIdx.x * 32 + (threadIdx.x & 31), nthr = n_cta * BT_THREADS;
    const uint32_t n = a.b.n_req;
    BlockPlan p;
    p.take = dyn;
    p.give = dyn + n;
    p.from = dyn + 2 * n;
    p.owner = reinterpret_cast<int32_t*>(dyn + 3 * n);
    int32_t* kept = p.owner + n + threadIdx.x;          // this thread's pages, BT_THREADS apart
    if (threadIdx.x == 0) { s_bad = 0u; s_taken = 0ull; s_height = __ldcg(a.n_free); }
    __syncthreads();
    p.height = s_height;                                // one reading, and so one number of rounds, for all threads
    const bool stack_bad = p.height < 0 || (uint32_t)p.height > a.free_cap;

    // Prefix sums.  Pages are handed out in request order; a request is served when its need and
    // all needs before it (refused ones included) fit the stack, so the served ones are a prefix
    // of those that need anything.
    uint64_t take0 = 0, give0 = 0, most = 0;
    for (uint32_t r0 = 0; r0 < n; r0 += BT_THREADS) {
        const uint32_t r = r0 + threadIdx.x;
        uint64_t need = 0, give = 0;
        if (r < n) {
            const int32_t owner = a.b.owner[r];
            const ReqShape s = req_shape(owner, a.b.have[r], a.b.want[r], a.b.page, a.b.max_blocks);
            need = req_need(s);
            give = req_give(s);
            p.owner[r] = owner;
            p.from[r] = need ? s.bh : s.bw;
        }
        uint64_t tot_take, tot_give;
        const uint64_t incl_take = take0 + block_scan<BT_THREADS>(need, warp_sums, &tot_take);
        const uint64_t incl_give = give0 + block_scan<BT_THREADS>(give, warp_sums, &tot_give);
        if (r < n) {
            p.take[r] = saturate32(incl_take - need);
            p.give[r] = saturate32(incl_give - give);
            if (need && !stack_bad && incl_take <= (uint64_t)p.height) most = incl_take;
        }
        take0 += tot_take;
        give0 += tot_give;
    }
    if (most) atomicMax(&s_taken, (unsigned long long)most);
    __syncthreads();
    p.taken = (uint32_t)s_taken;                        // <= height
    // more given back than the stack has room for (or than there are pages): some page is named twice
    const bool no_room = stack_bad || (uint64_t)(p.height - (int32_t)p.taken) + give0 > a.free_cap;
    const uint32_t given = no_room ? 0u : (uint32_t)give0;
    const uint32_t moves = no_room ? 0u : p.taken + given;
    cl.sync();                                          // every CTA's s_bad is initialised

    // threads that share a page, and this one's number among them
    uint32_t share = 32;
    while (share > 1 && (uint64_t)moves * share > nthr) share >>= 1;
    const uint32_t sub = tid & (share - 1), first = tid / share, step = nthr / share;
    const uint32_t rounds = (moves + step - 1) / step;  // one, where threads share

    // Check and claim.  A page may be taken only if nobody owns it in any layer, given back only
    // by its owner, and appear once in the call: the first mention claims its label.
    bool wrong = no_room;
    for (uint32_t i = 0; i < rounds; i++) {
        const uint32_t k = first + i * step;
        int32_t page = -1, owner = 0;
        if (k < moves) {
            const PageMove m = page_move(a, p, k);
            owner = p.owner[m.r];
            if (sub == 0) page = page_named(a, p, k, m);
        }
        page = __shfl_sync(0xFFFFFFFFu, page, threadIdx.x & (32u - share));
        if (i < BT_KEEP) kept[i * BT_THREADS] = page;
        if (k >= moves) continue;
        bool ok = page >= 0 && (uint32_t)page < a.b.n_pages;
        if (ok) {
            int32_t* lab = a.owner_map + page;
            if (sub == 0) {
                const int32_t v = __ldcg(lab);
                ok = k < p.taken ? label_takable(v) : label_givable(v, owner);
                if (ok) ok = atomicCAS(lab, v, label_flip(v)) == v;
            }
            for (uint32_t l0 = sub == 0 ? share : sub; l0 < a.layers; l0 += 8 * share) {
                int32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; e++)
                    w[e] = l0 + e * share < a.layers ? __ldcg(lab + (uint64_t)(l0 + e * share) * a.b.n_pages) : GIFT_OWNER_NONE;
#pragma unroll
                for (int e = 0; e < 8; e++) ok = ok && (k < p.taken ? label_takable(w[e]) : label_givable(w[e], owner));
            }
        }
        wrong = wrong || !ok;
    }
    if (wrong) atomicOr(bad, 1u);
    cl.sync();
    const bool refused = *bad != 0u;

    for (uint32_t r = tid; r < n; r += nthr) {
        uint32_t st = GIFT_ST_BAD_TABLE;
        if (!refused) {
            const ReqShape s = load_shape(a.b, r);
            const uint32_t need = req_need(s);
            st = !s.ok ? GIFT_ST_BAD_DESC : need && (uint64_t)p.take[r] + need > (uint64_t)p.height ? GIFT_ST_NO_BLOCKS : 0u;
        }
        a.status[r] = st;
    }
    if (refused) {
        // put the claimed labels back; a page mentioned twice is put back by whoever gets there first
        for (uint32_t i = 0; i < rounds; i++) {
            const uint32_t k = first + i * step;
            if (k >= moves || sub != 0) continue;
            const int32_t page = i < BT_KEEP ? kept[i * BT_THREADS] : page_named(a, p, k, page_move(a, p, k));
            if (page < 0 || (uint32_t)page >= a.b.n_pages) continue;
            const int32_t v = __ldcg(a.owner_map + page);
            if (label_claimed(v)) atomicCAS(a.owner_map + page, v, label_flip(v));
        }
        cl.sync();                                      // CTA 0's s_bad stays until every CTA has read it
        return;
    }

    // Commit the labels, and the taken pages' entries.
    for (uint32_t i = 0; i < rounds; i++) {
        const uint32_t k = first + i * step;
        if (k >= moves) continue;
        const PageMove m = page_move(a, p, k);
        const bool take = k < p.taken;
        const int32_t label = take ? p.owner[m.r] : GIFT_OWNER_NONE;
        const int32_t page = i < BT_KEEP ? kept[i * BT_THREADS] : page_named(a, p, k, m);
        if (i >= BT_KEEP) {
            if (page < 0 || (uint32_t)page >= a.b.n_pages) continue;
            const int32_t v = __ldcg(a.owner_map + page);
            if (!label_claimed(v) || atomicCAS(a.owner_map + page, v, label) != v) continue;
        }
        int32_t* lab = a.owner_map + page;
#pragma unroll 8
        for (uint32_t l = sub; l < a.layers; l += share) lab[(uint64_t)l * a.b.n_pages] = label;
        if (take && sub == 0) a.b.table[m.entry] = page;
    }
    cl.sync();                                          // taken entries of the stack have been read

    // Push what is given back where the taken pages were, and above.
    for (uint32_t i = 0; i < rounds; i++) {
        const uint32_t k = first + i * step;
        if (k < p.taken || k >= moves || sub != 0) continue;
        const PageMove m = page_move(a, p, k);
        a.free_pages[(uint32_t)p.height - p.taken + (k - p.taken)] = i < BT_KEEP ? kept[i * BT_THREADS] : page_named(a, p, k, m);
        a.b.table[m.entry] = -1;
    }
    if (tid == 0) *a.n_free = p.height - (int32_t)p.taken + (int32_t)given;
}

// ---------------------------------------------------------------------------
// slot maps and segment tables
// ---------------------------------------------------------------------------

constexpr int MAP_THREADS = 256;

// Exclusive prefix of count(request) into shared memory; returns the sum.
template <class F>
__device__ __forceinline__ uint64_t prefix_requests(uint32_t n, uint32_t* first, uint64_t* warp_sums, F count)
{
    uint64_t base = 0;
    for (uint32_t r0 = 0; r0 < n; r0 += MAP_THREADS) {
        const uint32_t r = r0 + threadIdx.x;
        const uint64_t c = r < n ? (uint64_t)count(r) : 0ull;
        uint64_t total;
        const uint64_t incl = base + block_scan<MAP_THREADS>(c, warp_sums, &total);
        if (r < n) first[r] = saturate32(incl - c);
        base += total;
    }
    __syncthreads();
    return base;
}

struct SlotArgs {
    BatchArgs b;
    const int32_t* rel;
    uint32_t n_rows;
    int64_t* slots;
    int32_t* row_req;
    int32_t* row_pos;
    int32_t* row_owner;
    int32_t* row_ptr;
    int64_t* total;
};

__global__ void __launch_bounds__(MAP_THREADS) slot_map_kernel(const __grid_constant__ SlotArgs a)
{
    extern __shared__ uint32_t first[];
    __shared__ uint64_t warp_sums[MAP_THREADS / 32];
    const uint64_t total = prefix_requests(a.b.n_req, first, warp_sums, [&](uint32_t r) { return load_shape(a.b, r).rows; });
    const bool fits = total <= a.n_rows;
    if (blockIdx.x == 0) {
        if (a.row_ptr)
            for (uint32_t r = threadIdx.x; r <= a.b.n_req; r += MAP_THREADS)
                a.row_ptr[r] = !fits ? 0 : r < a.b.n_req ? (int32_t)first[r] : (int32_t)total;
        if (a.total && threadIdx.x == 0) *a.total = (int64_t)total;
    }
    for (uint32_t t = blockIdx.x * MAP_THREADS + threadIdx.x; t < a.n_rows; t += gridDim.x * MAP_THREADS) {
        int64_t slot = -1;
        int32_t req = -1, pos = -1, owner = GIFT_OWNER_NONE;
        if (fits && t < total) {
            const uint32_t r = req_of(first, a.b.n_req, t);
            const ReqShape s = load_shape(a.b, r);
            const int32_t i = a.rel ? a.rel[t] : (int32_t)(t - first[r]);
            req = (int32_t)r;
            owner = a.b.owner[r];
            if (i >= 0 && (uint32_t)i < s.rows) {
                const uint32_t p = s.have + (uint32_t)i, blk = a.b.page.quot(p);
                pos = (int32_t)p;
                const int32_t page = a.b.table[(uint64_t)r * a.b.max_blocks + blk];
                if (page >= 0 && (uint32_t)page < a.b.n_pages)
                    slot = (int64_t)page * a.b.page_tokens + (p - blk * a.b.page_tokens);
            }
        }
        a.slots[t] = slot;
        if (a.row_req) a.row_req[t] = req;
        if (a.row_pos) a.row_pos[t] = pos;
        if (a.row_owner) a.row_owner[t] = owner;
    }
}

struct SegTabArgs {
    BatchArgs b;
    const uint32_t* serial;
    uint32_t layers, flags, cap;
    uint64_t token_bytes;
    uint64_t* segs;          // 5 words of 8 bytes per segment
    int32_t* page_table;
    int64_t* total;
};

__device__ __forceinline__ uint32_t first_block(const SegTabArgs& a, const ReqShape& s)
{
    if (!(a.flags & GIFT_KV_NEW_BLOCKS)) return 0u;
    const uint32_t b0 = a.b.page.quot(s.have);      // a block that was part full is exported again
    return b0 < s.bw ? b0 : s.bw;
}

// A block without new tokens is not exported under GIFT_KV_NEW_BLOCKS.
__device__ __forceinline__ uint32_t n_export(const SegTabArgs& a, const ReqShape& s)
{
    if ((a.flags & GIFT_KV_NEW_BLOCKS) && s.rows == 0) return 0u;
    return s.bw - first_block(a, s);
}

__global__ void __launch_bounds__(MAP_THREADS) kv_segments_kernel(const __grid_constant__ SegTabArgs a)
{
    extern __shared__ uint32_t first[];
    __shared__ uint64_t warp_sums[MAP_THREADS / 32];
    __shared__ uint64_t words[MAP_THREADS / 32][32 * 5];
    const uint64_t blocks = prefix_requests(a.b.n_req, first, warp_sums, [&](uint32_t r) { return n_export(a, load_shape(a.b, r)); });
    const bool fits = blocks <= a.cap && blocks * a.layers <= a.cap;
    const uint32_t n = fits ? (uint32_t)(blocks * a.layers) : 0u;
    if (a.total && blockIdx.x == 0 && threadIdx.x == 0)
        *a.total = blocks > 0x7FFFFFFFFFFFFFFFull / a.layers ? 0x7FFFFFFFFFFFFFFFll : (int64_t)(blocks * a.layers);
    // A lane makes a segment's five words; the warp writes its 32 segments as one run (each lane
    // writing its own 40 bytes: 10.3 us for 262 000 segments, this way 8.3).
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t warps = gridDim.x * (MAP_THREADS / 32);
    for (uint32_t e0 = (blockIdx.x * (MAP_THREADS / 32) + warp) * 32; e0 < a.cap; e0 += warps * 32) {
        const uint32_t e = e0 + lane;
        // an entry behind the last segment has a reserved flag set: the segment calls refuse it
        uint64_t w0 = (uint32_t)GIFT_OWNER_NONE | ((uint64_t)1 << 32), len = 0, w3 = 0, w4 = (uint64_t)e << 32;
        int32_t entry = -1;
        if (e < n) {
            const uint32_t layer = e / (uint32_t)blocks, k = e - layer * (uint32_t)blocks;
            const uint32_t r = req_of(first, a.b.n_req, k);
            const ReqShape s = load_shape(a.b, r);
            const uint32_t blk = first_block(a, s) + (k - first[r]);
            uint32_t tokens = s.want - blk * a.b.page_tokens;
            if ((a.flags & GIFT_KV_WHOLE_PAGES) || tokens > a.b.page_tokens) tokens = a.b.page_tokens;
            len = tokens * a.token_bytes;
            w0 = (uint32_t)a.b.owner[r];
            w3 = (uint64_t)a.serial[r] | ((uint64_t)layer << 32);
            w4 = (uint64_t)blk | ((uint64_t)e << 32);
            const int32_t page = a.b.table[(uint64_t)r * a.b.max_blocks + blk];
            if (page >= 0 && (uint32_t)page < a.b.n_pages) entry = (int32_t)(layer * a.b.n_pages + (uint32_t)page);
        }
        uint64_t* mine = words[warp] + lane * 5;
        mine[0] = w0; mine[1] = 0; mine[2] = len; mine[3] = w3; mine[4] = w4;
        if (e < a.cap) a.page_table[e] = entry;
        __syncwarp();
        const uint32_t n_words = (a.cap - e0 < 32u ? a.cap - e0 : 32u) * 5;
        uint64_t* o = a.segs + (uint64_t)e0 * 5;
        for (uint32_t k = lane; k < n_words; k += 32) o[k] = words[warp][k];
        __syncwarp();
    }
}

uint32_t map_grid(const gift_ctx* c, uint64_t items)
{
    const uint64_t want = (items + MAP_THREADS - 1) / MAP_THREADS, most = 4ull * c->num_sms;
    return (uint32_t)(want < 1 ? 1 : want > most ? most : want);
}

}  // namespace

extern "C" {

int gift_block_tables(gift_ctx* c, const gift_batch* batch, int32_t* free_pages, uint32_t free_cap, int32_t* n_free,
                      int32_t* owner_map, uint32_t layers, uint32_t* status, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    const int rc = batch_args_ok(batch);
    if (rc != GIFT_OK || batch->n_req == 0) return rc;
    if ((free_cap && !free_pages) || !n_free || (batch->n_pages && !owner_map) || !status || layers == 0) return GIFT_E_INVAL;
    if (layers > GIFT_MAX_LAYERS || free_cap > 0x7FFFFFFFu) return GIFT_E_RANGE;
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    BlockArgs a;
    memset(&a, 0, sizeof(a));
    a.b = batch_args(batch);
    a.free_pages = free_pages; a.n_free = n_free; a.free_cap = free_cap;
    a.owner_map = owner_map; a.layers = layers; a.status = status;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.blockDim = dim3(BT_THREADS, 1, 1);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    // Once per device: shared memory for the most requests, and whether 16 such CTAs can be co-scheduled.
    static int ctas_for_device[BT_MAX_DEVICES];
    const int slot = c->device >= 0 && c->device < BT_MAX_DEVICES ? c->device : -1;
    int ctas = slot >= 0 ? ctas_for_device[slot] : 0;
    if (ctas == 0) {
        CU_TRY(cudaFuncSetAttribute(block_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GIFT_MAX_REQS * BT_REQ_BYTES + BT_KEEP_BYTES));
        ctas = BT_CTAS_PORTABLE;
        if (cudaFuncSetAttribute(block_tables_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
            int n_clusters = 0;
            cfg.gridDim = dim3(BT_CTAS_LARGE, 1, 1);
            cfg.dynamicSmemBytes = GIFT_MAX_REQS * BT_REQ_BYTES + BT_KEEP_BYTES;
            attr.val.clusterDim.x = BT_CTAS_LARGE;
            if (cudaOccupancyMaxActiveClusters(&n_clusters, block_tables_kernel, &cfg) == cudaSuccess && n_clusters >= 1)
                ctas = BT_CTAS_LARGE;
        }
        (void)cudaGetLastError();
        if (slot >= 0) ctas_for_device[slot] = ctas;
    }
    cfg.gridDim = dim3(ctas, 1, 1);
    cfg.dynamicSmemBytes = (size_t)batch->n_req * BT_REQ_BYTES + BT_KEEP_BYTES;
    attr.val.clusterDim.x = ctas;
    CU_TRY(cudaLaunchKernelEx(&cfg, block_tables_kernel, a));
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

int gift_slot_map(gift_ctx* c, const gift_batch* batch, const int32_t* rel, uint32_t n_rows, int64_t* slots,
                  int32_t* row_req, int32_t* row_pos, int32_t* row_owner, int32_t* row_ptr, int64_t* total, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    const int rc = batch_args_ok(batch);
    if (rc != GIFT_OK) return rc;
    if (n_rows && !slots) return GIFT_E_INVAL;
    if (n_rows > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (n_rows == 0 && !row_ptr && !total) return GIFT_OK;
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    SlotArgs a;
    memset(&a, 0, sizeof(a));
    a.b = batch_args(batch);
    a.rel = rel; a.n_rows = n_rows; a.slots = slots; a.row_req = row_req; a.row_pos = row_pos;
    a.row_owner = row_owner; a.row_ptr = row_ptr; a.total = total;
    slot_map_kernel<<<map_grid(c, n_rows), MAP_THREADS, (size_t)batch->n_req * 4, (cudaStream_t)stream>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

int gift_kv_segments(gift_ctx* c, const gift_batch* batch, const uint32_t* serial, uint32_t layers, uint64_t token_bytes,
                     uint32_t flags, gift_seg* segs, int32_t* page_table, uint32_t cap, int64_t* total, void* stream)
{
    if (!c) return GIFT_E_INVAL;
    const int rc = batch_args_ok(batch);
    if (rc != GIFT_OK) return rc;
    if (flags & ~(GIFT_KV_WHOLE_PAGES | GIFT_KV_NEW_BLOCKS)) return GIFT_E_INVAL;
    if (layers == 0 || token_bytes == 0 || (batch->n_req && !serial) || (cap && (!segs || !page_table))) return GIFT_E_INVAL;
    if (layers > GIFT_MAX_LAYERS || cap > 0x7FFFFFFFu || token_bytes > (1u << 30)) return GIFT_E_RANGE;
    if ((uint64_t)layers * batch->n_pages > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if ((uintptr_t)segs & 7) return GIFT_E_ALIGN;
    if (cap == 0 && !total) return GIFT_OK;
    DeviceGuard g(c->device);
    if (!g.ok) return GIFT_E_CUDA;
    SegTabArgs a;
    memset(&a, 0, sizeof(a));
    a.b = batch_args(batch);
    a.serial = serial; a.layers = layers; a.flags = flags; a.cap = cap; a.token_bytes = token_bytes;
    a.segs = reinterpret_cast<uint64_t*>(segs); a.page_table = page_table; a.total = total;
    kv_segments_kernel<<<map_grid(c, cap), MAP_THREADS, (size_t)batch->n_req * 4, (cudaStream_t)stream>>>(a);
    c->launches++;
    CU_TRY(cudaGetLastError());
    return GIFT_OK;
}

}  // extern "C"
