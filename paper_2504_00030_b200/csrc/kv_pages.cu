// Block tables and slot maps built on the device from the sequences' lengths (KV caching, paper Section 5).
//
// Three phases with a barrier between them: pages given back are pushed on the free stack, pages asked for
// are popped, rows are looked up.  Where a page goes follows from two prefix sums over the batch (released and wanted
// pages), so the result is that of the sequential walk in the order of the batch, whatever the launch.
//
// What bounds it is latency: a decoding step moves a few hundred words, an admission a few megabytes.  One
// thread-block cluster does the whole call in one launch: its barrier is a hardware instruction (a grid-wide one would
// need a second launch or a spin), every block computes the same prefix sums for itself (a batch's lengths are a
// few kilobytes in L2), and the pages and rows are dealt out over the cluster's threads.
#include "common.cuh"

namespace sv {

constexpr int KP_THREADS = 1024;       // one scan step covers this many sequences
constexpr int KP_PAGE = 16;

struct KvPagesLaunch {
    sv_kv_pages_params p;
};

struct KvPagesShared {
    int32_t rel[KP_THREADS];           // exclusive prefix of released / wanted pages within the chunk
    int32_t req[KP_THREADS];
    int32_t col[KP_THREADS];           // first column that changes hands
    int32_t warp_rel[32], warp_req[32];
    int32_t first_without;             // first sequence that goes without its pages
    int32_t served;                    // pages acquired
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// every thread of the cluster arrives; global writes before it are visible behind it (release / acquire)
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

// pages of one sequence: what it holds, what it needs, whether its numbers make sense
struct SeqPages {
    int held, need;
    bool ok;
};
__device__ __forceinline__ SeqPages seq_pages(const sv_kv_pages_params &p, int b)
{
    SeqPages s;
    const int len = __ldg(p.seq_len + b);
    s.held = __ldcg(p.n_held + b);
    s.need = len > 0 ? (len - 1) / KP_PAGE + 1 : 0;
    s.ok = len >= 0 && s.need <= p.block_table_stride && s.held >= 0 && s.held <= p.block_table_stride;
    return s;
}

// exclusive prefix sums of the chunk's released and wanted pages into shared memory; returns the chunk's totals
__device__ __forceinline__ int2 scan_chunk(KvPagesShared &sh, int rel, int req, int col)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int a = rel, c = req;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int ua = __shfl_up_sync(0xffffffffu, a, d), uc = __shfl_up_sync(0xffffffffu, c, d);
        if (lane >= d) {
            a += ua;
            c += uc;
        }
    }
    __syncthreads();                   // the previous chunk's arrays are no longer read
    if (lane == 31) {
        sh.warp_rel[warp] = a;
        sh.warp_req[warp] = c;
    }
    __syncthreads();
    int ta = sh.warp_rel[lane], tc = sh.warp_req[lane];       // every warp scans the warp totals
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int ua = __shfl_up_sync(0xffffffffu, ta, d), uc = __shfl_up_sync(0xffffffffu, tc, d);
        if (lane >= d) {
            ta += ua;
            tc += uc;
        }
    }
    const int before_a = warp > 0 ? __shfl_sync(0xffffffffu, ta, warp - 1) : 0;
    const int before_c = warp > 0 ? __shfl_sync(0xffffffffu, tc, warp - 1) : 0;
    sh.rel[threadIdx.x] = before_a + a - rel;
    sh.req[threadIdx.x] = before_c + c - req;
    sh.col[threadIdx.x] = col;
    const int2 total = make_int2(__shfl_sync(0xffffffffu, ta, 31), __shfl_sync(0xffffffffu, tc, 31));
    __syncthreads();
    return total;
}

// the sequence of the chunk whose share of the prefix sums holds entry e: the last one that starts at or before it
__device__ __forceinline__ int owner_of(const int32_t *ex, int e)
{
    int lo = 0;
#pragma unroll
    for (int step = KP_THREADS / 2; step > 0; step >>= 1)
        if (ex[lo + step] <= e) lo += step;
    return lo;
}

__global__ void __launch_bounds__(KP_THREADS)
kv_pages_kernel(const __grid_constant__ KvPagesLaunch a)
{
    pdl_enter();
    __shared__ KvPagesShared sh;
    const sv_kv_pages_params &p = a.p;
    const int tid = threadIdx.x, rank = (int)cluster_rank();
    const int threads = (int)cluster_size() * KP_THREADS, me = rank * KP_THREADS + tid;
    const int batch = p.batch;
    const int n_pages = (int)p.n_pages;
    uint32_t bad = 0;

    int n_free = __ldcg(p.n_free);
    if (n_free < 0 || n_free > n_pages) {
        bad |= SV_DEV_BAD_PAGE;
        n_free = min(max(n_free, 0), n_pages);
    }
    // ---- release
    long long released = 0;
    for (int b0 = 0; b0 < batch; b0 += KP_THREADS) {
        int rel = 0, req = 0, col = 0;
        if (b0 + tid < batch) {
            const SeqPages s = seq_pages(p, b0 + tid);
            if (s.ok) {
                rel = max(s.held - s.need, 0);
                req = max(s.need - s.held, 0);
                col = min(s.held, s.need);
            } else {
                bad |= SV_DEV_BAD_LEN;
            }
        }
        const int total = scan_chunk(sh, rel, req, col).x;
        for (int e = me; e < total; e += threads) {
            const int s = owner_of(sh.rel, e);
            int32_t *entry = p.block_table + (long long)(b0 + s) * p.block_table_stride + sh.col[s] + (e - sh.rel[s]);
            const int page = __ldcg(entry);
            if (page < 0 || page >= n_pages) bad |= SV_DEV_BAD_PAGE;
            const long long at = n_free + released + e;
            if (at < n_pages) p.free_list[at] = page;
            else bad |= SV_DEV_BAD_PAGE;
            *entry = -1;
        }
        released += total;
    }
    const int have = (int)min((long long)n_free + released, (long long)n_pages);
    cluster_sync();
    // ---- acquire
    int taken = 0, without = batch;
    for (int b0 = 0; b0 < batch && without == batch; b0 += KP_THREADS) {
        int req = 0, col = 0;
        if (b0 + tid < batch) {
            const SeqPages s = seq_pages(p, b0 + tid);
            if (s.ok) {
                req = max(s.need - s.held, 0);
                col = min(s.held, s.need);
            }
        }
        if (tid == 0) sh.first_without = batch;
        const int total = scan_chunk(sh, 0, req, col).y;
        if (req > 0 && taken + sh.req[tid] + req > have) atomicMin(&sh.first_without, b0 + tid);
        __syncthreads();
        without = sh.first_without;
        const int served = without < batch ? sh.req[without - b0] : total;
        for (int e = me; e < served; e += threads) {
            const int s = owner_of(sh.req, e);
            p.block_table[(long long)(b0 + s) * p.block_table_stride + sh.col[s] + (e - sh.req[s])] =
                __ldcg(p.free_list + have - 1 - taken - e);
        }
        taken += served;
    }
    if (without < batch) bad |= SV_DEV_NO_PAGES;
    if (me == 0) *p.n_free = have - taken;
    cluster_sync();
    // ---- held pages and rows: a warp per sequence
    const bool rows = p.slot_map != nullptr || p.positions != nullptr;
    const int lane = tid & 31;
    for (int b = me >> 5; b < batch; b += threads >> 5) {
        SeqPages s = seq_pages(p, b);
        if (s.ok && (b < without || s.need < s.held)) s.held = s.need;
        __syncwarp();
        if (lane == 0 && s.ok) p.n_held[b] = s.held;
        if (!rows) continue;
        const int len = __ldg(p.seq_len + b);
        int g = __ldg(p.gamma + b);
        if (g < 0 || g > p.gamma_max) {
            bad |= SV_DEV_BAD_GAMMA;
            g = min(max(g, 0), p.gamma_max);
        }
        bool there = s.ok && len > 0 && s.need <= s.held;
        if (s.ok && len > 0 && len <= g) {
            bad |= SV_DEV_BAD_LEN;
            there = false;
        }
        const long long lo = max(__ldg(p.cu_q + b), 0), hi = min((long long)__ldg(p.cu_q + b + 1), (long long)p.n_rows);
        const int32_t *table = p.block_table + (long long)b * p.block_table_stride;
        for (long long r = lo + lane; r < hi; r += 32) {
            int pos = -1;
            long long slot = -1;
            if (there && r - lo <= g) {
                pos = len - g - 1 + (int)(r - lo);
                const int page = __ldcg(table + pos / KP_PAGE);
                if (page >= 0 && page < n_pages) slot = (long long)page * KP_PAGE + pos % KP_PAGE;
                else bad |= SV_DEV_BAD_PAGE;
            }
            if (p.slot_map != nullptr) p.slot_map[r] = slot;
            if (p.positions != nullptr) p.positions[r] = slot >= 0 ? pos : -1;
        }
    }
    // ---- rows of no sequence
    if (rows) {
        const long long first = min((long long)max(__ldg(p.cu_q), 0), (long long)p.n_rows);
        const long long last = max(__ldg(p.cu_q + batch), 0);
        for (long long r = me; r < first; r += threads) {
            if (p.slot_map != nullptr) p.slot_map[r] = -1;
            if (p.positions != nullptr) p.positions[r] = -1;
        }
        for (long long r = last + me; r < p.n_rows; r += threads) {
            if (p.slot_map != nullptr) p.slot_map[r] = -1;
            if (p.positions != nullptr) p.positions[r] = -1;
        }
    }
    if (bad != 0) set_status(p.device_status, bad);
}

}  // namespace sv

extern "C" sv_status spec_kv_pages_update(const sv_kv_pages_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr) return SV_EINVAL;
    if (p->seq_len == nullptr || p->block_table == nullptr || p->n_held == nullptr || p->free_list == nullptr ||
        p->n_free == nullptr)
        return SV_EINVAL;
    if (p->batch <= 0 || p->block_table_stride <= 0 || p->n_pages <= 0 || p->gamma_max < 0 || p->n_rows < 0)
        return SV_EINVAL;
    if (p->slot_map != nullptr || p->positions != nullptr) {
        if (p->gamma == nullptr || p->cu_q == nullptr || p->n_rows == 0) return SV_EINVAL;
    }
    if (p->page_size != KP_PAGE) return SV_EUNSUPPORTED;
    // page and row counts are summed in 32 bits
    if (p->n_pages > 0x7fffffffLL || p->n_rows > 0x7fffffffLL || p->block_table_stride > 0x7fffffffLL / p->batch)
        return SV_EUNSUPPORTED;
    KvPagesLaunch a;
    a.p = *p;
    const int blocks = 8;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = KP_THREADS;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    ++g_launches;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_pages_kernel, a);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess ? SV_OK : SV_ECUDA;
}
