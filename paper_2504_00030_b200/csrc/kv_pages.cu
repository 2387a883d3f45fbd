// Block tables and slot maps built on the device from the sequences' lengths (KV caching, paper Section 5).
//
// Where a page goes follows from two prefix sums over the batch (released and wanted pages), so the result is that of
// the sequential walk in the order of the batch, whatever the launch.  An acquired page is found without waiting for the
// releases: an index below the old top of the stack is read from the stack, one above it names an entry that is
// being released and is read from the block table.  Reads therefore see the state before the call throughout, and
// what would overwrite it (-1 in released entries, held pages, the top of the stack) is written behind the one barrier.
// Only a call that both releases and acquires many pages has a second one, behind which all are read from the stack.
//
// What bounds it is latency: a decoding step moves a few hundred words, an admission a few megabytes.  One
// thread-block cluster does the whole call in one launch, up to KP_ONE_CLUSTER sequences: its barrier is a hardware
// instruction (a grid-wide one would need a second launch or a spin), every block computes the same prefix sums for itself
// (a batch's lengths are a few kilobytes in L2), and the pages and rows are dealt out over the cluster's threads.
#include "common.cuh"

namespace sv {

constexpr int KP_THREADS = 1024;
constexpr int KP_PAGE = 16;
constexpr int KP_MAX_BATCH = 8192;     // prefix sums of the whole batch stay in shared memory (16 bytes a sequence)
constexpr int KP_CLUSTER = 8;          // blocks of the cluster (the portable size)
// Largest batch that one cluster serves alone; above it the pages are moved by the whole GPU and a second launch closes
// the books.  Measured, us a call, one launch / two: 128 sequences that decode 5.2 / 7.1, 384 6.8 / 7.6, 512 7.8 / 7.9,
// 1024 11.8 / 9.1; half of the batch replaced by other prompts at 8192 tokens on average: 64 sequences 5.3 / 7.2,
// 256 9.7 / 7.9, 384 11.8 / 8.2, 512 14.8 / 8.8, 1024 31 / 10.8.  Decoding is what most calls do.
constexpr int KP_ONE_CLUSTER = 384;
static_assert(KP_ONE_CLUSTER <= KP_THREADS, "one sequence a thread");
constexpr size_t kp_bytes(int batch) { return (size_t)(4 * batch + 3) * sizeof(int32_t); }      // prefix sums and first columns
constexpr size_t KP_SMEM = 40 * 1024;  // what a kernel may have without asking (48 KB, its static arrays among them)
static_assert(kp_bytes(KP_ONE_CLUSTER) <= KP_SMEM, "one cluster's kernel never asks");

struct KvPagesLaunch {
    sv_kv_pages_params p;
    int search;                        // first step of a thread's binary search: the largest power of two <= batch
};

// every thread of the cluster arrives; global writes before it are visible behind it
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// The last sequence whose exclusive prefix is at most e.  ex[0] = 0 <= e and ex[batch] = the total; for e below the
// total that sequence is the owner of entry e.
__device__ __forceinline__ int owner_of(const int32_t *ex, int batch, int search, int e)
{
    int lo = 0;
    for (int step = search; step > 0; step >>= 1)
        if (lo + step < batch && ex[lo + step] <= e) lo += step;
    return lo;
}

// the same for a whole warp, 32 candidates a step
__device__ __forceinline__ int warp_owner_of(const int32_t *ex, int batch, int e, int lane)
{
    int lo = 0;
    for (int stride = batch > 1024 ? 1024 : batch > 32 ? 32 : 1; stride > 0; stride >>= 5) {
        const int i = lo + lane * stride;
        lo += (__popc(__ballot_sync(0xffffffffu, i < batch && ex[i] <= e)) - 1) * stride;
    }
    return lo;
}

// What every block knows about the batch: prefix sums in shared memory and the totals that follow from them.
// UNIT: columns of one sequence that a warp moves at a time.
template <int UNIT>
struct Pages {
    const int32_t *rel;                // [batch + 1] exclusive prefix of released pages
    const int32_t *req;                // [batch + 1] exclusive prefix of wanted pages
    const int32_t *unit;               // [batch + 1] exclusive prefix of units (UNIT columns that change hands)
    const int32_t *col;                // [batch] first column that changes hands, -1: sequence left alone
    int n_free;                        // top of the stack before the call
    int have;                          // and after the releases
    int from_stack;                    // acquired pages below this index are read from the stack
    int batch, search;

    // page that is acquired as number e
    __device__ __forceinline__ int acquired(const sv_kv_pages_params &p, int e) const
    {
        const int at = have - 1 - e;
        if (at < from_stack) return __ldcg(p.free_list + at);
        const int s = owner_of(rel, batch, search, at - n_free);
        return __ldcg(p.block_table + (long long)s * p.block_table_stride + col[s] + (at - n_free - rel[s]));
    }

    // body(sequence, first of its changed columns that the unit holds) for each unit of this warp, from unit `begin` on
    template <typename F>
    __device__ __forceinline__ void for_units(int begin, int warp, int warps, int lane, F &&body) const
    {
        const int total = unit[batch];
        for (int u = begin + warp; u < total; u += warps) {
            const int s = warp_owner_of(unit, batch, u, lane);
            body(s, (u - unit[s]) * UNIT);
        }
    }
};

// WHOLE: the call in one launch by one cluster.  MOVE: what comes before the barrier, by a grid of any size; CLOSE: what
// comes behind it, by one cluster in a second launch.
enum { KP_WHOLE, KP_MOVE, KP_CLOSE };

// Pages that a thread has under way.  One cluster has more sequences than it has warps for their parts: 128 that decode take 5.5 us
// with 8 pages a thread, 5.2 with 4; half of 64 replaced 5.9 and 5.4, of 256 9.3 and 9.7.  The whole GPU: half of 1024 10.8 and 13.3.
constexpr int kp_unroll(int part) { return part == KP_WHOLE ? 4 : 8; }

template <int PART>
__global__ void __launch_bounds__(KP_THREADS)
kv_pages_kernel(const __grid_constant__ KvPagesLaunch a)
{
    // The closing launch may start, and make its prefix sums, before the first one has ended: what they read is not written by it,
    // and every block of it has waited for the kernels in front of the call before this launch may start (whose results are
    // read from L2: this launch has not waited itself).  A closing block (32 registers a thread) does not fit beside a moving one
    // (40) in a multiprocessor's 65536, so its sums run beside the last moving blocks only, where others have ended.
    if (PART != KP_CLOSE) pdl_enter();
    extern __shared__ int32_t kp_smem[];
    __shared__ int32_t warp_rel[32], warp_req[32], warp_unit[32];
    const sv_kv_pages_params &p = a.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int threads = gridDim.x * KP_THREADS, me = blockIdx.x * KP_THREADS + tid;     // a cluster is a whole grid
    const int my_warp = me >> 5, warps = threads >> 5;
    constexpr int UNROLL = kp_unroll(PART), UNIT = 32 * UNROLL;
    const int batch = p.batch, n_pages = (int)p.n_pages;
    int32_t *rel = kp_smem, *req = rel + batch + 1, *unit = req + batch + 1, *col = unit + batch + 1;
    uint32_t bad = 0;

    Pages<UNIT> pg;
    pg.n_free = __ldcg(p.n_free);
    if (pg.n_free < 0 || pg.n_free > n_pages) {
        bad |= SV_DEV_BAD_PAGE;
        pg.n_free = min(max(pg.n_free, 0), n_pages);
    }
    // ---- prefix sums: a thread has `items` neighbouring sequences
    const int items = PART == KP_WHOLE ? 1 : (batch + KP_THREADS - 1) / KP_THREADS;
    int my_rel = 0, my_req = 0, my_unit = 0, my_col = -1;
#pragma unroll 4
    for (int i = 0; i < items; ++i) {
        const int b = tid * items + i;
        if (b >= batch) break;
        const int len = PART == KP_CLOSE ? __ldcg(p.seq_len + b) : p.seq_len[b], held = __ldcg(p.n_held + b);
        const int need = len > 0 ? (len - 1) / KP_PAGE + 1 : 0;
        int n_rel = 0, n_req = 0;
        my_col = -1;
        if (len >= 0 && need <= p.block_table_stride && held >= 0 && held <= p.block_table_stride) {
            n_rel = max(held - need, 0);
            n_req = max(need - held, 0);
            my_col = min(held, need);
        } else {
            bad |= SV_DEV_BAD_LEN;
        }
        col[b] = my_col;
        if (items > 1) {
            rel[b] = n_rel;
            req[b] = n_req;
        }
        my_rel += n_rel;
        my_req += n_req;
        my_unit += (n_rel + n_req + UNIT - 1) / UNIT;     // one of the two is zero
    }
    int sum_rel = my_rel, sum_req = my_req, sum_unit = my_unit;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u0 = __shfl_up_sync(0xffffffffu, sum_rel, d), u1 = __shfl_up_sync(0xffffffffu, sum_req, d),
                  u2 = __shfl_up_sync(0xffffffffu, sum_unit, d);
        if (lane >= d) {
            sum_rel += u0;
            sum_req += u1;
            sum_unit += u2;
        }
    }
    if (lane == 31) {
        warp_rel[warp] = sum_rel;
        warp_req[warp] = sum_req;
        warp_unit[warp] = sum_unit;
    }
    __syncthreads();
    int t_rel = warp_rel[lane], t_req = warp_req[lane], t_unit = warp_unit[lane];     // every warp scans the 32 totals
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u0 = __shfl_up_sync(0xffffffffu, t_rel, d), u1 = __shfl_up_sync(0xffffffffu, t_req, d),
                  u2 = __shfl_up_sync(0xffffffffu, t_unit, d);
        if (lane >= d) {
            t_rel += u0;
            t_req += u1;
            t_unit += u2;
        }
    }
    const int prev = warp > 0 ? warp - 1 : 0;
    const int before_rel = __shfl_sync(0xffffffffu, t_rel, prev), before_req = __shfl_sync(0xffffffffu, t_req, prev),
              before_unit = __shfl_sync(0xffffffffu, t_unit, prev);
    const int base_rel = __shfl_sync(0xffffffffu, t_rel, 31), base_req = __shfl_sync(0xffffffffu, t_req, 31),
              base_unit = __shfl_sync(0xffffffffu, t_unit, 31);                       // totals of the batch
    int at_rel = (warp > 0 ? before_rel : 0) + sum_rel - my_rel, at_req = (warp > 0 ? before_req : 0) + sum_req - my_req,
        at_unit = (warp > 0 ? before_unit : 0) + sum_unit - my_unit;
#pragma unroll 4
    for (int i = 0; i < items; ++i) {
        const int b = tid * items + i;
        if (b >= batch) break;
        const int n_rel = items > 1 ? rel[b] : my_rel, n_req = items > 1 ? req[b] : my_req;
        rel[b] = at_rel;
        req[b] = at_req;
        unit[b] = at_unit;
        at_rel += n_rel;
        at_req += n_req;
        at_unit += (n_rel + n_req + UNIT - 1) / UNIT;
    }
    if (tid == 0) {
        rel[batch] = base_rel;
        req[batch] = base_req;
        unit[batch] = base_unit;
    }
    __syncthreads();
    if (PART == KP_CLOSE) {
        cluster_arrive();              // this block has read what the last lines write
        pdl_enter();
    }
    pg.rel = rel;
    pg.req = req;
    pg.unit = unit;
    pg.col = col;
    pg.batch = batch;
    pg.search = a.search;
    pg.have = (int)min((long long)pg.n_free + base_rel, (long long)n_pages);
    pg.from_stack = pg.n_free;
    if ((long long)pg.n_free + base_rel > n_pages) bad |= SV_DEV_BAD_PAGE;
    // the first sequence that goes without its pages: the one in whose share the last page has been handed out
    int without = batch, served = base_req;
    if (base_req > pg.have) {
        without = owner_of(req, batch, a.search, pg.have);
        served = req[without];
        bad |= SV_DEV_NO_PAGES;
    }
    // Released entries that land below this index of the stack are not handed out again, so nobody reads them and they become -1
    // at once.  (One cluster alone leaves all of them for the end, which measured 0.7 us faster for 128 sequences.)
    const int untouched = PART == KP_WHOLE ? 0 : pg.have - served;
    if (PART != KP_CLOSE) {
        // ---- released pages onto the stack
        if (base_rel > 0) {
            pg.for_units(0, my_warp, warps, lane, [&](int s, int first) {
                const int n = rel[s + 1] - rel[s], at = pg.n_free + rel[s];
                int32_t *from = p.block_table + (long long)s * p.block_table_stride + col[s];
                int page[UNROLL];
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int j = first + u * 32 + lane;
                    page[u] = j < n ? __ldcg(from + j) : 0;
                }
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int j = first + u * 32 + lane;
                    if (j >= n) continue;
                    if (page[u] < 0 || page[u] >= n_pages) bad |= SV_DEV_BAD_PAGE;
                    if (j < n_pages - at) p.free_list[at + j] = page[u];
                    if (PART != KP_WHOLE && j < untouched - at) from[j] = -1;
                }
            });
            // A page that is read as an entry being released costs a binary search; for more than a few a thread, the
            // barrier (about a microsecond) is cheaper.
            if (PART == KP_WHOLE && served > threads) {
                cluster_arrive();
                cluster_wait();
                pg.from_stack = pg.have;
            }
        }
        // ---- acquired pages into the table
        if (served > 0) {
            pg.for_units(0, my_warp, warps, lane, [&](int s, int first) {
                const int n = s < without ? req[s + 1] - req[s] : 0, e = req[s];
                int32_t *to = p.block_table + (long long)s * p.block_table_stride + col[s];
                int page[UNROLL];
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int j = first + u * 32 + lane;
                    page[u] = j < n ? pg.acquired(p, e + j) : 0;
                }
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int j = first + u * 32 + lane;
                    if (j < n) to[j] = page[u];
                }
            });
        }
        // ---- rows: a warp per sequence
        if (p.slot_map != nullptr || p.positions != nullptr) {
            // from the other end of the cluster, whose warps have few pages to move
            for (int b = warps - 1 - my_warp; b < batch; b += warps) {
                const int len = p.seq_len[b];
                int g = p.gamma[b];
                const long long lo = max(p.cu_q[b], 0), hi = min((long long)p.cu_q[b + 1], (long long)p.n_rows);
                if (g < 0 || g > p.gamma_max) {
                    bad |= SV_DEV_BAD_GAMMA;
                    g = min(max(g, 0), p.gamma_max);
                }
                const int c0 = col[b], wanted = req[b + 1] - req[b];
                const int held = c0 + (rel[b + 1] - rel[b]);
                bool there = c0 >= 0 && len > 0 && (wanted == 0 || b < without);
                if (c0 >= 0 && len > 0 && len <= g) {
                    bad |= SV_DEV_BAD_LEN;
                    there = false;
                }
                for (long long r = lo + lane; r < hi; r += 32) {
                    int pos = -1;
                    long long slot = -1;
                    if (there && r - lo <= g) {
                        pos = len - g - 1 + (int)(r - lo);
                        const int c = pos / KP_PAGE;
                        const int page = c < held ? __ldcg(p.block_table + (long long)b * p.block_table_stride + c)
                                                  : pg.acquired(p, req[b] + c - held);
                        if (page >= 0 && page < n_pages) slot = (long long)page * KP_PAGE + pos % KP_PAGE;
                        else bad |= SV_DEV_BAD_PAGE;
                    }
                    if (p.slot_map != nullptr) p.slot_map[r] = slot;
                    if (p.positions != nullptr) p.positions[r] = slot >= 0 ? pos : -1;
                }
            }
            // rows of no sequence
            const long long first = min((long long)max(p.cu_q[0], 0), (long long)p.n_rows);
            const long long last = max(p.cu_q[batch], 0);
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
    if (PART == KP_MOVE) return;
    // ---- nobody reads the old state any more
    if (PART == KP_WHOLE) cluster_arrive();
    cluster_wait();
    if (untouched - pg.n_free < base_rel) {            // released entries that acquisitions may have read
        const int from = max(untouched - pg.n_free, 0);
        pg.for_units(PART == KP_WHOLE ? 0 : unit[owner_of(rel, batch, a.search, from)], my_warp, warps, lane, [&](int s, int first) {
            const int n = min(rel[s + 1] - rel[s] - first, UNIT);
            int32_t *entry = p.block_table + (long long)s * p.block_table_stride + col[s] + first;
            for (int j = lane; j < n; j += 32)
                if (rel[s] + first + j >= from) entry[j] = -1;
        });
    }
    for (int b = me; b < batch; b += threads) {
        const int n_req = req[b + 1] - req[b], n_rel = rel[b + 1] - rel[b];
        if (n_rel > 0) p.n_held[b] = col[b];
        if (n_req > 0 && b < without) p.n_held[b] = col[b] + n_req;
    }
    if (me == 0) *p.n_free = pg.have - served;
}

// Lets a kernel of the two-launch form have the prefix sums of any batch in shared memory.  The limit belongs to the kernel, not to
// the call, and host threads share it: it is the same for every batch, so that none lowers it under another one's launch.
template <int PART>
static bool allow_smem()
{
    if (cudaFuncSetAttribute(kv_pages_kernel<PART>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kp_bytes(KP_MAX_BATCH)) == cudaSuccess) return true;
    (void)cudaGetLastError();
    return false;
}

template <int PART>
static sv_status launch_pages(const KvPagesLaunch &a, int blocks, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = KP_THREADS;
    cfg.dynamicSmemBytes = kp_bytes(a.p.batch);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PART == KP_MOVE ? 1 : 2;
    ++g_launches;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_pages_kernel<PART>, a);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess ? SV_OK : SV_ECUDA;
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
    // pages and rows are counted in 32 bits, with room for a loop's last step; the top of the stack and what is given back, added
    // up, as well
    if (p->batch > KP_MAX_BATCH) return SV_EUNSUPPORTED;
    if (p->n_pages >= 1LL << 30 || p->n_rows > 0x7fffffffLL || p->block_table_stride > (1LL << 30) / p->batch)
        return SV_EUNSUPPORTED;
    KvPagesLaunch a;
    a.p = *p;
    a.search = 1;
    while (2 * a.search <= p->batch) a.search *= 2;
    if (p->batch <= KP_ONE_CLUSTER) return launch_pages<KP_WHOLE>(a, KP_CLUSTER, (cudaStream_t)stream);
    // before the first launch: a refusal leaves the state as it was
    if (kp_bytes(p->batch) > KP_SMEM && !(allow_smem<KP_MOVE>() && allow_smem<KP_CLOSE>())) return SV_ECUDA;
    const sv_status st = launch_pages<KP_MOVE>(a, sm_count(), (cudaStream_t)stream);
    return st != SV_OK ? st : launch_pages<KP_CLOSE>(a, KP_CLUSTER, (cudaStream_t)stream);
}
