// Attention over parts of the cache (tcgen05, sm_100a): the kernel behind spec_verify_attn_pages and
// spec_verify_attn_prefix.
//
// Work.  An owner is what has keys of its own: a sequence, a (sequence, kv head) with its page list, or a group of
// sequences with its shared prefix.  An owner's query rows -- positions times the group's query heads -- are cut into
// tiles of 128 rows, NL tiles to a pair; a pair walks the owner's keys in tiles of TILE tokens.  The key tiles of all
// pairs form one list that is shared out over the grid by cost (lengths and lists live on the device, so every block
// finds its share in its prologue); a block's piece of a pair is a segment.  A segment that covers its pair writes the
// output, one that does not leaves its unnormalised rows (fp32 O, running maximum and sum) in the workspace.
//
// NL = 1: one row tile, 113 KB of shared memory and half of the tensor memory, so that two blocks share a multiprocessor:
//   the one streams while the other changes pairs.  Taken where a pair has at most 128 rows (G (gamma_max+1) <= 128): there
//   the keys are read for few rows and HBM is the limit.
// NL = 2: two row tiles that share the key tiles, one block a multiprocessor; while the tensor core works for one of them
//   the softmax warps of the other have the exponentials.  Taken for more rows and for the groups, where the tensor core and
//   the exponentials are the limit.
// A key tile has 64 tokens, so that every row tile has two S buffers in tensor memory (2 * 64 columns beside O's 128): the
// scores of the next tile are there when the softmax of this one is done.  (128 tokens and one buffer, whose S = Q K^T is a
// quarter cheaper on the tensor core: 600 us for the groups of 128 sequences behind three prefixes where this took 520 beside it.)
//
// Warps: 0 = TMA of K, 2 = TMA of V, 1 and 3 = MMA issuers of the row tiles (1 owns the tensor memory; with one row tile 3
// brings the queries of pairs of up to 32 rows ahead); then four softmax warps per row tile (thread = row = TMEM lane).  All
// hand-offs are mbarriers; every wait is bounded, an expired wait sets SV_DEV_TIMEOUT and drains the block.
//
// Measured (B200, device time of the call, 128-dim heads; at 1965 MHz, and in brackets where calls in a row for a second have
// brought the clock to 1400 to 1490): lists of 128 pages for one row of each of 128 sequences 189 us (221; 173 us of bytes at a
// copy's rate); of 64 pages a row for 17 rows of 64 heads 254 us (369; 163 us of bytes: rows of different sequences fill 136 of
// 256, the chain S -> softmax -> P V of a row tile sets the pace); one token over 64 pages 13.5 us (latency of two launches).
#pragma once

#include "attn_common.cuh"
#include "attn_softmax.cuh"
#include "f32x2.cuh"
#include "tc_ptx.cuh"
#include "work_share.cuh"

#include <math_constants.h>

namespace sv {

enum SegKind { SEG_LIST = 0, SEG_SEQ = 1, SEG_GROUP = 2 };

constexpr int SEG_MAX_GRID = 1024;
constexpr int SEG_PITCH = 128;                 // floats between rows of a partial (both head sizes)
constexpr int SEG_RING = 12;                   // most ring slots
constexpr int SEG_TILE = 64;                   // tokens of a key tile
constexpr int SEG_S_BUFS = 2;                  // S buffers of a row tile
constexpr int SEG_Q_AHEAD = 32;                // most rows of a pair whose queries are brought ahead

__host__ __device__ inline size_t seg_slot_floats(int rows) { return (size_t)rows * (SEG_PITCH + 2); }

// What the plan of spec_verify_attn_prefix leaves for its attention launches.
struct PrefixPlan {
    int32_t *grp_pages;      // [n_groups] shared pages (0: nothing is shared)
    int32_t *grp_rep;        // [n_groups] a member: its block table row has the pages
    int32_t *grp_n;          // [n_groups] positions of all members
    int32_t *grp_base;       // [n_groups] first of them in row_list
    int2 *row_list;          // query row of each position, group by group, and b * (gamma_max+1) + i
    int32_t *seq_pages;      // [batch] shared pages in front of the sequence (0: none)
    float *part_o;           // what the groups leave for the sequences: unnormalised fp32 O of position b * (gamma_max+1) + i and
    float2 *part_ml;         // head, [positions * hq][128], and its running maximum and sum
};

struct SegLaunch {
    sv_attn_params p;
    int64_t n_pool_pages;
    int group;               // query heads per kv head
    int ppl;                 // positions of a row tile: 128 / group
    int n_slots;             // K/V ring slots
    int q_ahead;             // the query rows of the next pair are brought by a warp of their own (two buffers of 32 rows)
    int n_owners;
    const int32_t *page_list;      // SEG_LIST
    const uint64_t *row_mask;
    const int32_t *n_list;
    int64_t list_stride;
    const int32_t *seq_group;      // of the plan kernel
    PrefixPlan plan;
    int32_t *bounds;         // [grid + 1]: first tile of every block
    int32_t *desc;           // [grid * 4]: a block's last segment, if its pair begins there and goes on: owner (else -1), pair
                             // of the owner, slot of the partial, the pair's end in the list of tiles
    float *part;             // partials: block * 2 + (0: the block's first segment, 1: its last)
};

// The walk over (owner, pair of the owner, tile).
struct SegCursor {
    int o, s, t;             // owner, pair of the owner, tile of the pair
    int n_sub, n_tiles;      // pairs of the owner, tiles of each
    int b, h, chunk;         // sequence (SEG_GROUP: group), kv head, row chunk
    int R, L;                // positions of the owner, length (SEG_GROUP: of the prefix)
    int n_pages, page0;      // pages to read: entries of the list, or of the table from page0 on
};

// Pairs and tiles of owner c.o (0 tiles: nothing to do); fills the owner's part of the cursor.
template <int KIND, int NL>
__device__ __forceinline__ void seg_owner(const SegLaunch &a, SegCursor &c, bool report)
{
    constexpr int PPT = SEG_TILE / 16;
    const sv_attn_params &p = a.p;
    const int ppp = NL * a.ppl;
    c.n_sub = c.n_tiles = 0;
    c.page0 = 0;
    if (KIND == SEG_GROUP) {
        c.b = c.o;
        c.R = a.plan.grp_n[c.o];
        c.n_pages = a.plan.grp_pages[c.o];
        c.L = c.n_pages * 16;
        if (c.R <= 0 || c.n_pages <= 0) return;
        c.n_sub = p.hkv * ((c.R + ppp - 1) / ppp);
        c.n_tiles = (c.n_pages + PPT - 1) / PPT;
        return;
    }
    c.b = KIND == SEG_LIST ? c.o / p.hkv : c.o;
    int g = p.gamma[c.b];
    c.L = p.seq_len[c.b];
    int n = KIND == SEG_LIST ? a.n_list[c.o] : a.plan.seq_pages[c.b];
    if (g < 0 || g > p.gamma_max) {
        if (report) set_status(p.device_status, SV_DEV_BAD_GAMMA);
        g = min(max(g, 0), p.gamma_max);
    }
    c.R = g + 1;
    if (c.L < c.R || c.L > p.max_seq_len || (c.L + 15) / 16 > p.block_table_stride) {        // in this order: the sum stays in range
        if (report) set_status(p.device_status, SV_DEV_BAD_LEN);
        return;
    }
    const int chunks = (c.R + ppp - 1) / ppp;
    if (KIND == SEG_LIST) {
        if (n < 0 || n > a.list_stride) {
            if (report) set_status(p.device_status, SV_DEV_BAD_LEN);
            n = (int)min((long long)max(n, 0), (long long)a.list_stride);
        }
        c.n_pages = n;
        c.n_sub = chunks;
        c.n_tiles = max(1, (n + PPT - 1) / PPT);       // an empty list still has outputs
    } else {
        c.page0 = n;
        c.n_pages = (c.L + 15) / 16 - n;
        c.n_sub = p.hkv * chunks;
        c.n_tiles = (c.n_pages + PPT - 1) / PPT;
    }
}

template <int KIND, int NL>
__device__ __forceinline__ void seg_pair(const SegLaunch &a, SegCursor &c)
{
    const int ppp = NL * a.ppl;
    if (KIND == SEG_LIST) {
        c.h = c.o - c.b * a.p.hkv;
        c.chunk = c.s;
    } else {
        const int chunks = (c.R + ppp - 1) / ppp;
        c.h = c.s / chunks;
        c.chunk = c.s - c.h * chunks;
    }
}

template <int KIND, int NL>
__device__ __forceinline__ void seg_next(const SegLaunch &a, SegCursor &c)
{
    c.t = 0;
    if (++c.s >= c.n_sub) {
        c.s = 0;
        c.n_tiles = 0;
        while (c.n_tiles == 0 && ++c.o < a.n_owners) seg_owner<KIND, NL>(a, c, false);
        if (c.o >= a.n_owners) { c.n_tiles = c.n_sub = 1; c.R = 1; c.b = c.h = c.chunk = 0; return; }     // past the end: never used
    }
    seg_pair<KIND, NL>(a, c);
}

// The calling block's share, by the whole block (NT threads); every block publishes its first tile.
template <int KIND, int NL, int NT>
__device__ __forceinline__ void seg_plan(const SegLaunch &a, int pair_cost, WorkShare *sh, SegCursor *start, long long (*red)[NT / 32])
{
    SegCursor c;
    plan_work_share<NT>(
        a.n_owners, pair_cost,
        [&](int o, bool first) {
            c.o = o;
            seg_owner<KIND, NL>(a, c, first && blockIdx.x == 0);
            return OwnerWork{c.n_sub, c.n_tiles};
        },
        [&]() { *start = c; }, sh, red);
    if (threadIdx.x == 0) {
        a.bounds[blockIdx.x] = (int)sh->t_begin;
        if (blockIdx.x + 1 == gridDim.x) a.bounds[gridDim.x] = (int)sh->total;
        a.desc[blockIdx.x * 4] = -1;
    }
}

template <int KIND, int NL>
__device__ __forceinline__ void seg_start(const SegLaunch &a, const WorkShare &sh, const SegCursor &start, SegCursor &c)
{
    c = start;                                                 // only called by blocks with tiles
    c.s = sh.s; c.t = sh.t;
    seg_pair<KIND, NL>(a, c);
    if (c.t >= c.n_tiles) seg_next<KIND, NL>(a, c);
}

struct SegShared {
    uint64_t full[SEG_RING];     // ring slot filled by TMA
    uint64_t empty[SEG_RING];    // ring slot consumed by the tensor core
    uint64_t s_full[4];          // S ready (row tile * 2 + parity of the key tile)
    uint64_t p_full[4];          // P written
    uint64_t o_done[4];          // P V finished
    uint64_t q_full[2];          // query rows are in shared memory: (q_ahead) of the buffer, else of the row tile
    uint64_t q_empty[2];         // (q_ahead) and were read for the last time
    uint64_t drained[2];         // a row tile's instructions are through (after an expired wait)
    uint32_t tmem_base;
    int abort_flag;
    WorkShare share;
    SegCursor start;             // of the owner that the block begins in
};

// Place in the ring of the tiles' K (first = 0) or V (first = 1): the items K, V of tile 0, K, V of tile 1 ... take the slots in
// turn.  Advanced by additions: divisions by the slot count cost the MMA warp more cycles than its instructions took.
struct RingPos {
    int slot;
    uint32_t use;            // times the ring has wrapped
    __device__ __forceinline__ explicit RingPos(int first) : slot(first), use(0) {}
    __device__ __forceinline__ void next(int n_slots)
    {
        slot += 2;
        if (slot >= n_slots) { slot -= n_slots; ++use; }
    }
};

// bounded_wait whose outcome a warp agrees on, so that it stays together when a wait is given up
__device__ __forceinline__ bool seg_wait(uint32_t bar, uint32_t parity, int *abort_flag, uint32_t *status)
{
    return __all_sync(0xffffffffu, bounded_wait(bar, parity, abort_flag, status));
}

// eight float32 of a partial row (32-byte aligned) at a time: a whole sector of the memory, where 16 bytes a thread would
// touch each sector twice
__device__ __forceinline__ void store8(float *dst, const uint32_t *o)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]),
                 "r"(o[5]), "r"(o[6]), "r"(o[7])
                 : "memory");
}
__device__ __forceinline__ void load8(const float *src, uint32_t *x)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7])
                 : "l"(src));
}

// the larger of three
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// The online softmax of one row's TILE scores, as softmax_tile, with the keys that the row may see given per page:
// lim[j] is the last visible slot of the tile's page j (below 0: none; 15 or more: all).
template <int TILE, int O_CHUNKS, typename WaitPV>
__device__ __forceinline__ bool seg_softmax(uint32_t s_addr, uint32_t o_addr, const int (&lim)[TILE / 16], float c_scale,
                                            bool first_tile, float &m_ref, float &l_sum, WaitPV &&wait_prev_pv)
{
    uint32_t s[TILE];
#pragma unroll
    for (int ch = 0; ch < TILE / 32; ++ch) tc_ld32_nowait(s_addr + ch * 32, s + ch * 32);
    tc_wait_ld();
    bool partial = false, none = false;
#pragma unroll
    for (int j = 0; j < TILE / 16; ++j) {
        partial |= lim[j] >= 0 && lim[j] < 15;
        none |= lim[j] < 0;
    }
    if (partial) {
#pragma unroll
        for (int c = 0; c < TILE; ++c)
            if ((c & 15) > lim[c >> 4]) s[c] = 0xff800000u;     // -inf
    } else if (none) {
#pragma unroll
        for (int c = 0; c < TILE; ++c)
            if (lim[c >> 4] < 0) s[c] = 0xff800000u;
    }
    float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, m2 = -CUDART_INF_F, m3 = -CUDART_INF_F;
#pragma unroll
    for (int c = 0; c < TILE; c += 8) {
        m0 = max3(m0, __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
        m1 = max3(m1, __uint_as_float(s[c + 2]), __uint_as_float(s[c + 3]));
        m2 = max3(m2, __uint_as_float(s[c + 4]), __uint_as_float(s[c + 5]));
        m3 = max3(m3, __uint_as_float(s[c + 6]), __uint_as_float(s[c + 7]));
    }
    const float m_tile = fmaxf(max3(m0, m1, m2), m3) * c_scale;
    float factor = 1.f;
    bool rescale = false;
    if ((m_tile > m_ref + RESCALE_THRESHOLD || m_ref == -CUDART_INF_F) && m_tile > -CUDART_INF_F) {
        rescale = m_ref > -CUDART_INF_F;
        factor = rescale ? ex2_approx(m_ref - m_tile) : 1.f;
        m_ref = m_tile;
    }
    const float m_use = (m_ref == -CUDART_INF_F) ? 0.f : m_ref;
    if (rescale) l_sum *= factor;
    // tensor-memory accesses are warp-wide: if any row of the warp has to rescale, the whole warp goes through (factor 1)
    if (__any_sync(0xffffffffu, rescale && !first_tile)) {
        if (!wait_prev_pv()) return false;
        tc_fence_after();
        const float f = (rescale && !first_tile) ? factor : 1.f;
#pragma unroll
        for (int ch = 0; ch < O_CHUNKS; ++ch) {
            uint32_t o[32];
            tc_ld32(o_addr + ch * 32, o);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tc_st32(o_addr + ch * 32, o);
        }
    }
    // P = 2^(s*c - m_ref) as bf16 pairs over S: the tensor core multiplies bf16, so each weight is rounded, by at most 2^-8 of it
    // and independently from key to key; an output is off by at most 2^-8 of the weighted sum of |v|, next to its own rounding
    // (2^-8 of it).  The sums stay fp32 and unrounded, so the log-sum-exp has none of it
    const uint64_t c2 = pair2(c_scale, c_scale), m2n = pair2(-m_use, -m_use);
    uint64_t sum = 0;                                  // two float32 zeros
#pragma unroll
    for (int ch = 0; ch < TILE / 32; ++ch) {
        uint32_t pk[16];
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
            float x0, x1;
            split2(fma2(pair2(__uint_as_float(s[ch * 32 + c]), __uint_as_float(s[ch * 32 + c + 1])), c2, m2n), x0, x1);
            const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
            sum = add2(sum, pair2(e0, e1));
            pk[c >> 1] = pack_bf16(e0, e1);
        }
        asm volatile(
            "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
            "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(s_addr + ch * 16),
            "r"(pk[0]), "r"(pk[1]), "r"(pk[2]), "r"(pk[3]), "r"(pk[4]), "r"(pk[5]), "r"(pk[6]), "r"(pk[7]), "r"(pk[8]),
            "r"(pk[9]), "r"(pk[10]), "r"(pk[11]), "r"(pk[12]), "r"(pk[13]), "r"(pk[14]), "r"(pk[15])
            : "memory");
    }
    float sum0, sum1;
    split2(sum, sum0, sum1);
    l_sum += sum0 + sum1;
    return true;
}

// What a row's sum makes of its output and log-sum-exp.  A sum of 0 is a row without keys, which lists alone can leave: zeros and
// -inf; elsewhere all scores are -inf, 0 / 0.  A sum that is no number (a NaN or an infinite score) stays one in both.
template <int KIND>
__device__ __forceinline__ float seg_inv(float l)
{
    return KIND == SEG_LIST && l == 0.f ? 0.f : 1.f / l;
}
template <int KIND>
__device__ __forceinline__ float seg_lse(float m, float l)
{
    if (KIND != SEG_LIST && l == 0.f) return CUDART_NAN_F;
    return (m + log2f(l)) * 0.6931471805599453f;
}

// a pair's start and end, in key tiles
__host__ __device__ constexpr int seg_pair_cost(int kind) { return kind == SEG_LIST ? 3 : kind == SEG_SEQ ? 8 : 12; }

template <int NL> struct SegConfig {
    static constexpr int THREADS = 128 + 128 * NL;
    static constexpr int BLOCKS = NL == 1 ? 2 : 1;             // blocks per multiprocessor
    static constexpr uint32_t TMEM_COLS = NL == 1 ? 256 : 512;
};

template <int KIND, int NL, int D>
__global__ void __launch_bounds__(SegConfig<NL>::THREADS, SegConfig<NL>::BLOCKS)
attn_seg_kernel(const __grid_constant__ SegLaunch a, const __grid_constant__ CUtensorMap k_map,
                const __grid_constant__ CUtensorMap v_map)
{
    constexpr int TILE = SEG_TILE, NT = SegConfig<NL>::THREADS;
    constexpr int NB = SEG_S_BUFS;
    constexpr int PPT = TILE / 16;                             // pages per tile
    constexpr int HALF = TILE * 128;                           // bytes of a tile's 64 dims
    constexpr int SLOT_BYTES = TILE * D * 2;
    constexpr int Q_BYTES = 128 * D * 2;
    constexpr uint32_t TMEM_COLS = SegConfig<NL>::TMEM_COLS;
    constexpr int O_COL0 = NL * NB * TILE;                     // the row tiles' S buffers, then their O
    constexpr int OCH = D / 32;
    extern __shared__ __align__(1024) uint8_t seg_smem[];
    const sv_attn_params &p = a.p;
    if ((smem_u32(seg_smem) & 1023u) != 0) {                       // never seen; refuse rather than compute garbage
        pdl_enter();
        if (threadIdx.x == 0) set_status(p.device_status, SV_DEV_TIMEOUT);
        return;
    }
    const int n_slots = a.n_slots;
    // Query rows: a tile of 128 per row tile, or, with q_ahead, two buffers of 32 rows.  The instructions read 128 rows all
    // the same: what lies behind the buffers (ring, barriers) gives rows of S that nobody looks at.
    const bool q_ahead = NL == 1 && a.q_ahead != 0;
    const int q_half = q_ahead ? SEG_Q_AHEAD * 128 : 16384;        // bytes between the 64-dim halves of the rows
    uint8_t *q_smem = seg_smem;
    uint8_t *ring = seg_smem + (q_ahead ? 2 * SEG_Q_AHEAD * D * 2 : NL * Q_BYTES);
    SegShared *sh = reinterpret_cast<SegShared *>(ring + (size_t)n_slots * SLOT_BYTES);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = a.group, ppl = a.ppl;

    // in front of the wait for the launch before: what needs nothing of it (not the tensor memory, which that one may hold)
    if (tid == 0) {
        for (int i = 0; i < n_slots; ++i) {
            mbar_init(smem_u32(&sh->full[i]), 1);
            mbar_init(smem_u32(&sh->empty[i]), NL);            // every row tile's MMA warp
        }
        for (int i = 0; i < NB * NL; ++i) {
            mbar_init(smem_u32(&sh->s_full[i]), 1);
            mbar_init(smem_u32(&sh->p_full[i]), 128);
            mbar_init(smem_u32(&sh->o_done[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->q_full[i]), q_ahead ? 1 : 128);
            mbar_init(smem_u32(&sh->q_empty[i]), 1);
        }
        for (int i = 0; i < NL; ++i) mbar_init(smem_u32(&sh->drained[i]), 1);
        sh->abort_flag = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_enter();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                     "r"(TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the plan's sums share the queries' memory, which nothing touches before the barrier below
    seg_plan<KIND, NL, NT>(a, seg_pair_cost(KIND), &sh->share, &sh->start, reinterpret_cast<long long(*)[NT / 32]>(seg_smem));
    tc_fence_before();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    tc_fence_after();

    const long long t_begin = sh->share.t_begin, t_end = sh->share.t_end;
    const uint32_t tmem = sh->tmem_base;
    int *abort_flag = &sh->abort_flag;
    uint32_t *status = p.device_status;

    if (warp < 4) {
        // of the block's registers (128 or 168 a thread at launch): 56 + 200 = 2 * 128, 56 + 2 * 224 = 3 * 168
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (t_end > t_begin && (warp == 0 || warp == 2)) {
            // ================================================================ TMA producers: warp 0 K, warp 2 V
            SegCursor cur;
            seg_start<KIND, NL>(a, sh->share, sh->start, cur);
            const bool is_v = warp == 2;
            constexpr int HV = D / 64;                         // 64-dim halves of a page
            const int page_in_tile = lane / HV, half = lane % HV;
            uint32_t u = 0;                                    // tiles of this block so far
            RingPos at(is_v ? 1 : 0);
            bool ok = true;
            int ids = 0;                                       // lane l: page of entry ids_base + l
            for (long long tg = t_begin; tg < t_end && ok;) {
                const int seg_tiles = (int)min((long long)(cur.n_tiles - cur.t), t_end - tg);
                SegCursor nxt = cur;                           // the next pair, looked up while this one's tiles are under way
                const int32_t *table;
                {
                    const int tb = KIND == SEG_GROUP ? a.plan.grp_rep[cur.o] : cur.b;
                    table = p.block_table + (long long)tb * p.block_table_stride;
                }
                const int32_t *list = KIND == SEG_LIST ? a.page_list + (long long)cur.o * a.list_stride : nullptr;
                const int seq_pages = (cur.L + 15) / 16;
                int ids_base = -1;
                for (int ti = 0; ti < seg_tiles; ++ti, ++u, at.next(n_slots)) {
                    const int e0 = (cur.t + ti) * PPT;
                    if (ids_base < 0 || e0 + PPT > ids_base + 32) {          // the next 32 page ids
                        ids_base = e0;
                        const int e = e0 + lane;
                        int phys = (int)a.n_pool_pages;        // out of range: TMA fills zeros, no traffic
                        if (e < cur.n_pages) {
                            int lp = cur.page0 + e;
                            if (KIND == SEG_LIST) lp = list[e];
                            int id = -1;
                            if (KIND != SEG_LIST || (lp >= 0 && lp < seq_pages)) id = table[lp];
                            if (id < 0 || id >= a.n_pool_pages) set_status(status, SV_DEV_BAD_PAGE);
                            else phys = id;
                        }
                        ids = phys;
                    }
                    const int phys = __shfl_sync(0xffffffffu, ids, (e0 - ids_base + page_in_tile) & 31);
                    const uint32_t full = smem_u32(&sh->full[at.slot]);
                    if (at.use > 0) ok = seg_wait(smem_u32(&sh->empty[at.slot]), (at.use - 1) & 1, abort_flag, status);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(full, SLOT_BYTES);
                    __syncwarp();
                    if (lane < PPT * HV) {
                        const uint32_t dst = smem_u32(ring + at.slot * SLOT_BYTES + half * HALF + page_in_tile * 2048);
                        tma_load_4d(dst, is_v ? &v_map : &k_map, half * 64, 0, cur.h, phys, full);
                    }
                    if (ti == 0) seg_next<KIND, NL>(a, nxt);
                }
                tg += seg_tiles;
                cur = nxt;                                     // a segment that ends inside its pair is the block's last
            }
            if (!ok && lane == 0) {
                // given up: the copies under way end before the block does (each slot's last use by this warp)
                for (uint32_t k = 0; k < (uint32_t)n_slots && k < u; ++k) {
                    const uint32_t item = 2 * (u - 1 - k) + (is_v ? 1 : 0);
                    if (item + n_slots < 2 * u) break;
                    const uint32_t bar = smem_u32(&sh->full[item % (uint32_t)n_slots]), par = (item / (uint32_t)n_slots) & 1;
                    for (int it = 0; it < (1 << 20) && !mbar_try_wait(bar, par); ++it) { }
                }
            }
        } else if (t_end > t_begin && (warp == 1 || NL == 2)) {
            // ================================================================ MMA issuers: a warp per row tile
            // An issuing warp spends about half of its time on waits (130 cycles each, also for what is there already), and
            // the tensor core's queue is short: with one warp for both row tiles a step of 64 keys took 2570 cycles
            // where the instructions take 1290.
            const int l = NL == 2 && warp == 3 ? 1 : 0;
            const uint32_t idesc_qk = instr_desc(false, TILE), idesc_pv = instr_desc(true, D);
            SegCursor cur;
            seg_start<KIND, NL>(a, sh->share, sh->start, cur);
            uint32_t seg_no = 0, cnt = 0;                      // segments and tiles in which this row tile has rows, so far
            RingPos k_at(0), v_at(1);                          // of the next Q K^T and the next P V
            // What steers the loops and makes up the descriptors goes through a warp-wide reduction, whose result the
            // compiler knows to be the same in all lanes: the operands of the instructions then stay in uniform registers,
            // where otherwise each instruction waits for its operands to be moved there.
            const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem);
            int left = __reduce_max_sync(0xffffffffu, (int)(t_end - t_begin));
            bool ok = true;
            while (left > 0 && ok) {
                const int seg_tiles = __reduce_max_sync(0xffffffffu, min(cur.n_tiles - cur.t, left));
                const int n_pos = cur.R - cur.chunk * NL * ppl;
                const uint32_t o_there = KIND == SEG_SEQ && __reduce_max_sync(0xffffffffu, cur.page0 > 0 && cur.t == 0) ? 1u : 0u;
                const bool active = NL == 1 || l == 0 || __reduce_max_sync(0xffffffffu, n_pos > ppl ? 1 : 0) != 0;
                SegCursor nxt = cur;
                const int qb = q_ahead ? (int)(seg_no & 1) : 0;
                if (active) {                                  // a row tile without rows brings no queries and counts no segment
                    ok = q_ahead ? seg_wait(smem_u32(&sh->q_full[qb]), (seg_no >> 1) & 1, abort_flag, status)
                                 : seg_wait(smem_u32(&sh->q_full[l]), seg_no & 1, abort_flag, status);
                    if (!ok) break;
                    tc_fence_after();
                    ++seg_no;
                }
                const uint64_t qd = smem_desc(smem_u32(q_smem + (q_ahead ? qb * SEG_Q_AHEAD * D * 2 : l * Q_BYTES)), 16, 1024);
                auto issue_qk = [&](int ti) {
                    ok = ok && seg_wait(smem_u32(&sh->full[k_at.slot]), k_at.use & 1, abort_flag, status);
                    if (!ok) return;
                    tc_fence_after();
                    const int buf = l * NB + (int)((cnt + ti) % NB);
                    const uint64_t kd = smem_desc(smem_u32(ring + k_at.slot * SLOT_BYTES), 16, 1024);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            tc_mma_ss(tm + buf * TILE, qd + (((ks >> 2) * q_half + (ks & 3) * 32) >> 4),
                                      kd + (((ks >> 2) * HALF + (ks & 3) * 32) >> 4), idesc_qk, ks > 0);
                        tc_commit(smem_u32(&sh->s_full[buf]));
                        tc_commit(smem_u32(&sh->empty[k_at.slot]));            // K tile consumed
                        if (q_ahead && ti == seg_tiles - 1) tc_commit(smem_u32(&sh->q_empty[qb]));
                    }
                    __syncwarp();
                    k_at.next(n_slots);
                };
                if (active) {
                    issue_qk(0);
                    if (NB > 1 && seg_tiles > 1) issue_qk(1);
                }
                seg_next<KIND, NL>(a, nxt);
                if (active) {
                    for (int ti = 0; ti < seg_tiles && ok; ++ti) {
                        const uint32_t g = cnt + ti;
                        const int buf = l * NB + (int)(g % NB);
                        ok = seg_wait(smem_u32(&sh->p_full[buf]), (g / NB) & 1, abort_flag, status);
                        if (ok) ok = seg_wait(smem_u32(&sh->full[v_at.slot]), v_at.use & 1, abort_flag, status);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t vd = smem_desc(smem_u32(ring + v_at.slot * SLOT_BYTES), HALF, 1024);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < TILE / 16; ++ks)
                                tc_mma_ts(tm + O_COL0 + l * 128, tm + buf * TILE + ks * 8, vd + (uint64_t)(ks * (2048 >> 4)),
                                          idesc_pv, (ti > 0 || ks > 0) ? 1u : o_there);
                            tc_commit(smem_u32(&sh->o_done[buf]));
                            tc_commit(smem_u32(&sh->empty[v_at.slot]));        // V tile consumed
                        }
                        __syncwarp();
                        v_at.next(n_slots);
                        if (ti + NB < seg_tiles) issue_qk(ti + NB);
                    }
                    cnt += seg_tiles;
                } else {                                       // no rows in this row tile: pass the tiles on
                    for (int ti = 0; ti < seg_tiles && ok; ++ti) {
                        ok = seg_wait(smem_u32(&sh->full[k_at.slot]), k_at.use & 1, abort_flag, status);
                        if (ok && lane == 0) mbar_arrive(smem_u32(&sh->empty[k_at.slot]));
                        if (ok) ok = seg_wait(smem_u32(&sh->full[v_at.slot]), v_at.use & 1, abort_flag, status);
                        if (ok && lane == 0) mbar_arrive(smem_u32(&sh->empty[v_at.slot]));
                        k_at.next(n_slots);
                        v_at.next(n_slots);
                    }
                }
                left -= seg_tiles;
                cur = nxt;
            }
            if (!ok) {                                         // given up: let the issued instructions finish
                if (elect_one()) tc_commit(smem_u32(&sh->drained[l]));
                __syncwarp();
                for (int it = 0; it < (1 << 20) && !mbar_try_wait(smem_u32(&sh->drained[l]), 0); ++it) { }
            }
        }
        else if (NL == 1 && t_end > t_begin && warp == 3 && q_ahead) {         // groups have two row tiles
            // ================================================================ query rows of the next pair
            SegCursor cur;
            seg_start<KIND, NL>(a, sh->share, sh->start, cur);
            constexpr int CH = D / 8, RPI = 32 / CH;           // 16-byte chunks of a row; rows that one load of the warp covers
            const int ch = lane % CH, r0 = lane / CH;
            bool ok = true;
            uint32_t seg_no = 0;
            for (long long tg = t_begin; tg < t_end && ok; ++seg_no) {
                const int seg_tiles = (int)min((long long)(cur.n_tiles - cur.t), t_end - tg);
                const int qb = seg_no & 1;
                const int pos0 = cur.chunk * ppl, n_rows = min(cur.R - pos0, ppl) * G;
                if (seg_no >= 2) ok = seg_wait(smem_u32(&sh->q_empty[qb]), ((seg_no >> 1) - 1) & 1, abort_flag, status);
                if (!ok) break;
                uint8_t *dst = q_smem + qb * SEG_Q_AHEAD * D * 2 + (ch >> 3) * q_half;
#pragma unroll 1
                for (int b0 = 0; b0 < n_rows; b0 += 4 * RPI) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = b0 + k * RPI + r0, i = r / G;
                        v[k] = make_uint4(0, 0, 0, 0);
                        if (r < n_rows) {
                            const int at = p.cu_q[cur.b] + pos0 + i;
                            const long long q_row = (long long)at * p.hq + (long long)cur.h * G + (r - i * G);
                            v[k] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) + q_row * D) + ch);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = b0 + k * RPI + r0;               // up to the next multiple of 4 * RPI, at most SEG_Q_AHEAD
                        *reinterpret_cast<uint4 *>(dst + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = v[k];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->q_full[qb]));
                tg += seg_tiles;
                cur.t += seg_tiles;
                if (cur.t == cur.n_tiles) seg_next<KIND, NL>(a, cur);
            }
        }
    } else {
        if (NL == 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        if (t_end > t_begin) {
            // ================================================================ softmax / epilogue, a thread per row
            const int l = NL == 2 ? (warp - 4) >> 2 : 0;       // row tile
            const int quarter = warp & 3;
            const int r = quarter * 32 + lane;                 // row of the tile = TMEM lane
            const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
            const uint32_t o_addr = tmem + lane_addr + O_COL0 + l * 128;
            const float c_scale = p.sm_scale * 1.4426950408889634f;          // scores in log2 units
            const int ri = r / G, hh = r - ri * G;             // position and head of the row within its tile
            SegCursor cur;
            seg_start<KIND, NL>(a, sh->share, sh->start, cur);
            uint32_t cnt = 0, seg_no = 0;                      // tiles of this row tile so far
            bool ok = true;
            int q0 = KIND == SEG_GROUP ? 0 : p.cu_q[cur.b];
            // List entries: lane l holds entry f_e + l of owner f_o and its mask.  With two row tiles they are brought ahead (17 rows
            // of 64 heads for 128 sequences: 261 -> 253 us); with one, where a second block works meanwhile, the more code cost
            // more than the waits (13 rows of one head, 40 kv heads: 180 -> 191 us).
            constexpr bool AHEAD = NL == 2;
            int f_o = -1, f_e = 0, f_lp = -1;
            unsigned long long f_mk = 0;
            auto fetch = [&](const SegCursor &w, int e0) {
                f_o = w.o;
                f_e = e0;
                f_lp = -1;
                f_mk = 0;
                if (e0 + lane < w.n_pages) {
                    const long long at = (long long)w.o * a.list_stride + e0 + lane;
                    f_lp = __ldg(a.page_list + at);
                    f_mk = __ldg(reinterpret_cast<const unsigned long long *>(a.row_mask) + at);
                }
            };
            for (long long tg = t_begin; tg < t_end && ok; ++seg_no) {
                const int seg_tiles = (int)min((long long)(cur.n_tiles - cur.t), t_end - tg);
                const int pos0 = cur.chunk * NL * ppl + l * ppl;               // first position of the row tile
                const int n_pos = min(cur.R - pos0, ppl);
                const bool tile_active = n_pos > 0;
                const bool warp_active = tile_active && quarter * 32 < n_pos * G;
                const bool row_ok = ri < n_pos;
                const int i = pos0 + ri;
                long long q_row = 0, part_row = 0;             // of the queries and outputs, and of the groups' partials
                if (row_ok) {
                    int2 at;
                    if (KIND == SEG_GROUP) at = a.plan.row_list[a.plan.grp_base[cur.o] + i];
                    else at = make_int2(q0 + i, cur.b * (p.gamma_max + 1) + i);
                    q_row = (long long)at.x * p.hq + (long long)cur.h * G + hh;
                    part_row = (long long)at.y * p.hq + (long long)cur.h * G + hh;
                }
                // ---- this thread's query row into shared memory.  Every instruction that read the rows before has
                // completed: this thread has seen the last S that they gave.
                if (!q_ahead && warp_active) {
                    // D / 8 lanes for a row: whole lines, where a thread for each row would touch 32 lines a load
                    constexpr int LPR = D / 8, RPI = 32 / LPR;
                    const int ch = lane % LPR, sub = lane / LPR;
                    uint4 v[32 / RPI];
#pragma unroll
                    for (int k = 0; k < 32 / RPI; ++k) {
                        const int from = k * RPI + sub;                        // the warp's row: the lane that knows its place
                        const long long qr = __shfl_sync(0xffffffffu, q_row, from);
                        const int have = __shfl_sync(0xffffffffu, (int)row_ok, from);
                        v[k] = have ? __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) + qr * D) + ch) : make_uint4(0, 0, 0, 0);
                    }
                    uint8_t *dst = q_smem + l * Q_BYTES + (ch >> 3) * 16384;
#pragma unroll
                    for (int k = 0; k < 32 / RPI; ++k) {
                        const int rr = quarter * 32 + k * RPI + sub;
                        *reinterpret_cast<uint4 *>(dst + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4)) = v[k];
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (!q_ahead && tile_active) mbar_arrive(smem_u32(&sh->q_full[l]));
                SegCursor nxt = cur;
                seg_next<KIND, NL>(a, nxt);
                int nxt_q0 = 0;                                // under way while this pair is worked on
                if (KIND != SEG_GROUP && nxt.o < a.n_owners) nxt_q0 = p.cu_q[nxt.b];
                const bool whole = cur.t == 0 && seg_tiles == cur.n_tiles;
                const int last = KIND == SEG_GROUP ? cur.L - 1 : cur.L - cur.R + i;       // last visible key of the row
                const int seq_pages = (cur.L + 15) / 16;
                const bool far = p.gamma_max >= 32;            // masks have bits above the 32nd
                int e_base = -32, e_lp = -1;                   // lane l: entry e_base + l of the list and its mask
                uint32_t e_lo = 0, e_hi = 0;
                float m_ref = -CUDART_INF_F, l_sum = 0.f;
                // behind a shared prefix the row begins with what its group left
                const bool joins = KIND == SEG_SEQ && cur.page0 > 0 && cur.t == 0;
                if (joins && warp_active) {
                    if (row_ok) {
                        const float2 ml = a.plan.part_ml[part_row];
                        m_ref = ml.x;
                        l_sum = ml.y;
                    }
                    const float *src = a.plan.part_o + part_row * SEG_PITCH;
#pragma unroll
                    for (int ch = 0; ch < OCH; ch += 2) {
                        uint32_t x[2][32];
#pragma unroll
                        for (int c = 0; c < 64; c += 8) {
#pragma unroll
                            for (int z = 0; z < 8; ++z) x[c >> 5][(c & 31) + z] = 0;
                            if (row_ok) load8(src + ch * 32 + c, &x[c >> 5][c & 31]);
                        }
                        tc_st32(o_addr + ch * 32, x[0]);
                        tc_st32(o_addr + ch * 32 + 32, x[1]);
                    }
                    tc_wait_st();                              // the first tile's maximum may have them read again at once
                }
                if (tile_active) {
                    for (int ti = 0; ti < seg_tiles && ok; ++ti, ++cnt) {
                        const int buf = l * NB + (int)(cnt % NB);
                        const uint32_t phase = (cnt / NB) & 1;
                        int lim[PPT];
                        if (KIND == SEG_LIST) {
                            const int e0 = (cur.t + ti) * PPT;
                            if (warp_active && (e0 < e_base || e0 >= e_base + 32)) {
                                if (!AHEAD || f_o != cur.o || f_e != e0) fetch(cur, e0);
                                e_base = e0;
                                e_lp = f_lp;
                                const bool have = f_lp >= 0 && f_lp < seq_pages;
                                e_lo = have ? (uint32_t)f_mk : 0;
                                e_hi = have ? (uint32_t)(f_mk >> 32) : 0;
                                if (AHEAD) {                   // under way while these are worked on: the segment's next, or the next pair's first
                                    if (ti + 32 / PPT < seg_tiles) fetch(cur, e0 + 32);
                                    else if (nxt.o < a.n_owners) fetch(nxt, 0);
                                }
                            }
#pragma unroll
                            for (int j = 0; j < PPT; ++j) {
                                const int src = (e0 - e_base + j) & 31;
                                const int lp = __shfl_sync(0xffffffffu, e_lp, src);
                                uint32_t mk = __shfl_sync(0xffffffffu, e_lo, src);
                                if (far) {
                                    const uint32_t hi = __shfl_sync(0xffffffffu, e_hi, src);
                                    if (i >= 32) mk = hi;
                                }
                                lim[j] = row_ok && ((mk >> (i & 31)) & 1) ? max(last - lp * 16, -1) : -1;
                            }
                        } else {
                            const int tok0 = (cur.page0 + (cur.t + ti) * PPT) * 16;        // the longest sequence leaves room for a tile
#pragma unroll
                            for (int j = 0; j < PPT; ++j) lim[j] = last - tok0 - j * 16;
                        }
                        ok = seg_wait(smem_u32(&sh->s_full[buf]), phase, abort_flag, status);
                        if (!ok) break;
                        if (!warp_active) {                    // all 32 rows are padding
                            mbar_arrive(smem_u32(&sh->p_full[buf]));
                            continue;
                        }
                        tc_fence_after();
                        ok = seg_softmax<TILE, OCH>(tmem + lane_addr + buf * TILE, o_addr, lim, c_scale, ti == 0 && !joins, m_ref, l_sum, [&]() {
                            const uint32_t g = cnt - 1;
                            return seg_wait(smem_u32(&sh->o_done[l * NB + (int)(g % NB)]), (g / NB) & 1, abort_flag, status);
                        });
                        if (!ok) break;
                        tc_wait_st();
                        tc_fence_before();
                        mbar_arrive(smem_u32(&sh->p_full[buf]));
                    }
                    if (!ok) break;
                    // the last P V.  It writes all rows: where the next pair's rows may begin with a partial, a warp without
                    // rows in this pair has to see it end too
                    if (warp_active || KIND == SEG_SEQ) {
                        const uint32_t g = cnt - 1;
                        ok = seg_wait(smem_u32(&sh->o_done[l * NB + (int)(g % NB)]), (g / NB) & 1, abort_flag, status);
                    }
                    if (!ok) break;
                    tc_fence_after();
                }
                if (!warp_active) {
                    // nothing to write
                } else if (KIND != SEG_GROUP && whole) {
                    // rolled loops here and below: the roles' code competes for the instruction cache (13 rows of one head, 40 kv
                    // heads, 9 pairs a block: 182 us unrolled, 172 rolled when it was tried)
                    const float inv = seg_inv<KIND>(l_sum);
                    __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(p.o) + q_row * D;
#pragma unroll 1
                    for (int ch = 0; ch < OCH; ++ch) {
                        uint32_t o[32];
                        tc_ld32(o_addr + ch * 32, o);
                        if (row_ok) {
#pragma unroll
                            for (int c = 0; c < 32; c += 8) {
                                uint4 w;
                                w.x = pack_bf16(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv);
                                w.y = pack_bf16(__uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
                                w.z = pack_bf16(__uint_as_float(o[c + 4]) * inv, __uint_as_float(o[c + 5]) * inv);
                                w.w = pack_bf16(__uint_as_float(o[c + 6]) * inv, __uint_as_float(o[c + 7]) * inv);
                                *reinterpret_cast<uint4 *>(dst + ch * 32 + c) = w;
                            }
                        }
                    }
                    if (row_ok && p.lse != nullptr) p.lse[q_row] = seg_lse<KIND>(m_ref, l_sum);
                } else {
                    // unnormalised: a whole pair of a group to the positions' rows, a piece of a pair to a slot of this block
                    const bool to_rows = KIND == SEG_GROUP && whole;
                    float *slot = a.part + ((size_t)blockIdx.x * 2 + (seg_no == 0 ? 0 : 1)) * seg_slot_floats(NL * 128);
                    const int row = l * 128 + r;
                    float *dst = to_rows ? a.plan.part_o + part_row * SEG_PITCH : slot + (size_t)row * SEG_PITCH;
#pragma unroll 1
                    for (int ch = 0; ch < OCH; ++ch) {
                        uint32_t o[32];
                        tc_ld32(o_addr + ch * 32, o);
                        if (row_ok) {
#pragma unroll
                            for (int c = 0; c < 32; c += 8) store8(dst + ch * 32 + c, o + c);
                        }
                    }
                    if (row_ok) {
                        // A sum that is no number goes with the highest maximum: with -inf (all scores NaN) the merge would take
                        // the part for one without keys
                        const float m_part = l_sum != l_sum ? CUDART_INF_F : m_ref;
                        if (to_rows) {
                            a.plan.part_ml[part_row] = make_float2(m_part, l_sum);
                        } else {
                            slot[(size_t)NL * 128 * SEG_PITCH + row] = m_part;
                            slot[(size_t)NL * 128 * SEG_PITCH + NL * 128 + row] = l_sum;
                        }
                    }
                }
                tc_fence_before();
                if (l == 0 && r == 0 && cur.t == 0 && seg_tiles < cur.n_tiles) {
                    // the pair goes on in the next blocks: the combine kernel merges its parts
                    *reinterpret_cast<int4 *>(a.desc + blockIdx.x * 4) =
                        make_int4(cur.o, cur.s, blockIdx.x * 2 + (seg_no == 0 ? 0 : 1), (int)(tg + cur.n_tiles));
                }
                tg += seg_tiles;
                cur = nxt;
                q0 = nxt_q0;
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

// ---------------------------------------------------------------------------- pairs that were split over blocks
constexpr int SEG_COMBINE_WARPS = 8;

// Merges the pairs that begin in a block of the main kernel and go on behind it.  The work -- eight rows of a pair, a warp
// each, `chunks` times for a pair -- is dealt out over all blocks, since few pairs may have many parts; P parts of a row are in flight at a time.  A
// group's rows go where its whole pairs' rows are.
template <int KIND, int NL, int D>
__global__ void __launch_bounds__(SEG_COMBINE_WARPS * 32)
attn_seg_combine_kernel(const __grid_constant__ SegLaunch a, int main_grid, int chunks)
{
    constexpr int SLOT_ROWS = NL * 128, NT = SEG_COMBINE_WARPS * 32;
    static_assert(SEG_MAX_GRID / 32 == 32 && SEG_MAX_GRID % NT == 0, "a warp holds the counts of all words");
    pdl_enter();
    __shared__ int s_split[SEG_MAX_GRID];      // blocks in which a split pair begins
    __shared__ int s_n;
    const sv_attn_params &p = a.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.group;
    {                                          // in order, so that all blocks deal out the same list
        __shared__ int s_count[SEG_MAX_GRID / 32];
        bool have[SEG_MAX_GRID / NT];
        unsigned mine[SEG_MAX_GRID / NT];
#pragma unroll
        for (int j = 0; j < SEG_MAX_GRID / NT; ++j) have[j] = j * NT + tid < main_grid && a.desc[(j * NT + tid) * 4] >= 0;
#pragma unroll
        for (int j = 0; j < SEG_MAX_GRID / NT; ++j) {
            mine[j] = __ballot_sync(0xffffffffu, have[j]);
            if (lane == 0) s_count[j * SEG_COMBINE_WARPS + warp] = __popc(mine[j]);
        }
        __syncthreads();
        const int n = s_count[lane];           // SEG_MAX_GRID / 32 = 32 words
        int upto = n;
#pragma unroll
        for (int dd = 1; dd < 32; dd <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, dd);
            if (lane >= dd) upto += x;
        }
#pragma unroll
        for (int j = 0; j < SEG_MAX_GRID / NT; ++j) {
            const int at = __shfl_sync(0xffffffffu, upto - n, j * SEG_COMBINE_WARPS + warp);
            if (have[j]) s_split[at + __popc(mine[j] & ((1u << lane) - 1))] = j * NT + tid;
        }
        if (warp == 0 && lane == 31) s_n = upto;
    }
    __syncthreads();
    const bool lane_on = 4 * lane < D;
    constexpr size_t slot_floats = (size_t)SLOT_ROWS * (SEG_PITCH + 2);
    for (int u = blockIdx.x; u < s_n * chunks; u += gridDim.x) {
        const int begin = s_split[u / chunks], k = u % chunks * SEG_COMBINE_WARPS + warp;
        const int4 d = *reinterpret_cast<const int4 *>(a.desc + begin * 4);
        SegCursor cur;
        cur.o = d.x; cur.s = d.y; cur.t = 0;
        seg_owner<KIND, NL>(a, cur, false);
        seg_pair<KIND, NL>(a, cur);
        const int pos0 = cur.chunk * NL * a.ppl, n_pos = min(cur.R - pos0, NL * a.ppl);
        if (k >= n_pos * G) continue;
        const int in = k / G, hh = k - in * G, i = pos0 + in;
        const int tile = in / a.ppl, row = tile * 128 + (in - tile * a.ppl) * G + hh;
        // where the row goes: to the positions' partials of a group, or to the outputs
        const int at = KIND == SEG_GROUP ? a.plan.row_list[a.plan.grp_base[cur.o] + i].y : p.cu_q[cur.b] + i;
        const long long dst_row = (long long)at * p.hq + (long long)cur.h * G + hh;
        float m_run = -CUDART_INF_F, l_run = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int P = NL == 1 ? 8 : 4;
        // P partials into the running one; -inf: not there, or no keys for the row
        auto merge = [&](const float (&m)[P], const float (&l)[P], const float4 (&v)[P]) {
            float m_new = m_run;
#pragma unroll
            for (int j = 0; j < P; ++j) m_new = fmaxf(m_new, m[j]);
            if (m_new == -CUDART_INF_F) return;
            const float w_old = exp2f(m_run - m_new);
            acc.x *= w_old; acc.y *= w_old; acc.z *= w_old; acc.w *= w_old;
            l_run *= w_old;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                if (m[j] == -CUDART_INF_F) continue;
                const float w = exp2f(m[j] - m_new);
                l_run += w * l[j];
                acc.x += w * v[j].x; acc.y += w * v[j].y; acc.z += w * v[j].z; acc.w += w * v[j].w;
            }
            m_run = m_new;
        };
        auto take = [&](const float *slot, float &m, float &l, float4 &v) {
            m = slot[(size_t)SLOT_ROWS * SEG_PITCH + row];
            l = slot[(size_t)SLOT_ROWS * SEG_PITCH + SLOT_ROWS + row];
            v = lane_on ? reinterpret_cast<const float4 *>(slot + (size_t)row * SEG_PITCH)[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
        };
        // the first part, then the first slots of the blocks behind it whose tiles begin before the
        // pair ends
        bool first = true;
        for (int c0 = begin + 1; first || c0 < main_grid; c0 += 32) {
            const int c = c0 + lane;
            const int lo = c < main_grid ? a.bounds[c] : 0x7fffffff, hi = c < main_grid ? a.bounds[c + 1] : 0;
            unsigned have = __ballot_sync(0xffffffffu, lo < d.w && hi > lo);       // empty blocks hold nothing
            while (first || have != 0) {
                float m[P], l[P];
                float4 v[P];
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    m[j] = -CUDART_INF_F;
                    l[j] = 0.f;
                    v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (j == 0 && first) {
                        take(a.part + (size_t)d.z * slot_floats, m[j], l[j], v[j]);
                    } else if (have != 0) {
                        take(a.part + (size_t)(c0 + __ffs(have) - 1) * 2 * slot_floats, m[j], l[j], v[j]);
                        have &= have - 1;
                    }
                }
                merge(m, l, v);
                first = false;
            }
            if (__any_sync(0xffffffffu, lo >= d.w)) break;
        }
        if (KIND == SEG_GROUP) {
            if (lane_on) reinterpret_cast<float4 *>(a.plan.part_o + dst_row * SEG_PITCH)[lane] = acc;
            if (lane == 0) a.plan.part_ml[dst_row] = make_float2(m_run, l_run);
            continue;
        }
        const float inv = seg_inv<KIND>(l_run);
        if (lane_on) {
            uint2 w;
            w.x = pack_bf16(acc.x * inv, acc.y * inv);
            w.y = pack_bf16(acc.z * inv, acc.w * inv);
            reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.o) + dst_row * D)[lane] = w;
        }
        if (lane == 0 && p.lse != nullptr) p.lse[dst_row] = seg_lse<KIND>(m_run, l_run);
    }
}

// ---------------------------------------------------------------------------- host side
inline int seg_nl(int rows) { return rows <= 128 ? 1 : 2; }
inline int seg_grid(int nl) { return sm_count() * (nl == 1 ? 2 : 1); }
// Longest sequence: the positions of its last tile fit an int.
constexpr int SEG_MAX_LEN = 0x7fffffff - SEG_TILE;
// Whether the key tiles of `pairs` pairs with at most `pages` pages each can be numbered with 31 bits, as the launches number them.
inline bool seg_tiles_fit(long long pairs, long long pages)
{
    const long long tiles = pages / (SEG_TILE / 16) + 1;
    return pairs <= 0x7fffffffLL / tiles;
}
// pairs of a sequence and kv head
inline long long seg_chunks(int group, int gamma_max)
{
    const int ppp = 128 / group * seg_nl(group * (gamma_max + 1));
    return (gamma_max + ppp) / ppp;
}
inline size_t seg_round(size_t n) { return (n + 255) & ~(size_t)255; }
// Partial rows move 32 bytes at a time, a caller's workspace begins on any 16: the tables and partials begin on the next 32.
constexpr size_t SEG_WS_SLACK = 16;
inline uint8_t *seg_workspace(void *w) { return reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(w) + 31) & ~(uintptr_t)31); }
// bounds, descriptors and partials of one launch
inline size_t seg_table_bytes() { return seg_round((SEG_MAX_GRID + 1) * sizeof(int32_t)) + seg_round(SEG_MAX_GRID * 4 * sizeof(int32_t)); }
inline size_t seg_part_bytes(int nl) { return (size_t)seg_grid(nl) * 2 * seg_slot_floats(nl * 128) * sizeof(float); }

template <int KIND, int NL, int D>
sv_status launch_seg(SegLaunch &a, int grid, cudaStream_t stream)
{
    constexpr int slot_bytes = SEG_TILE * D * 2;
    // shared memory of a multiprocessor less 1 KB that each block takes by itself
    const size_t budget = 228 * 1024 / SegConfig<NL>::BLOCKS - 1024;
    a.q_ahead = NL == 1 && a.group * (a.p.gamma_max + 1) <= SEG_Q_AHEAD;
    const size_t fixed = (a.q_ahead ? (size_t)2 * SEG_Q_AHEAD : (size_t)NL * 128) * D * 2 + ((sizeof(SegShared) + 15) & ~(size_t)15);
    a.n_slots = (int)((budget - fixed) / slot_bytes);
    if (a.n_slots > SEG_RING) a.n_slots = SEG_RING;
    if (a.n_slots < 4) return SV_EUNSUPPORTED;
    const size_t smem = fixed + (size_t)a.n_slots * slot_bytes;
    // the limit is all that a block may have, not this call's part of it: calls of several threads would lower it for one another
    // between here and the launch
    if (cudaFuncSetAttribute(attn_seg_kernel<KIND, NL, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)budget) != cudaSuccess)
        return SV_ECUDA;
    return launch_kernel(true, attn_seg_kernel<KIND, NL, D>, grid, SegConfig<NL>::THREADS, smem, stream, a, a.p.pool->k_map,
                         a.p.pool->v_map);
}

template <int KIND, int NL, int D>
sv_status launch_seg_combine(const SegLaunch &a, int grid, cudaStream_t stream)
{
    // a pair's rows: a group's fill their tiles, a sequence has at most G (gamma_max+1)
    int rows = NL * 128;
    if (KIND != SEG_GROUP && a.group * (a.p.gamma_max + 1) < rows) rows = a.group * (a.p.gamma_max + 1);
    return launch_kernel(true, attn_seg_combine_kernel<KIND, NL, D>, sm_count() * (NL == 1 ? 4 : 6), SEG_COMBINE_WARPS * 32, 0, stream, a, grid,
                         (rows + SEG_COMBINE_WARPS - 1) / SEG_COMBINE_WARPS);
}

}  // namespace sv
