// Selection of the pages that each row of a draft block reads (spec_page_select), two kernels.
//
// page_score_kernel.  The score of a page estimates the most that any of its keys can give with the row's queries (a bound but for
// the roundings to 8 bits, half a step of each),
//     max over the group's heads h of  sum_d max(q_hd M_d, q_hd m_d),
// with the queries in 8 bits (one scale per row and kv head, which no comparison needs) and the page's bounds M, m in 8
// bits times the page's scale.  max(q M, q m) = max(q, 0) M + min(q, 0) m, so it is an integer matrix product of depth
// 2 head_dim: 128 pages (tensor-memory lanes) times rows * heads (columns), tcgen05.mma kind::i8 with int32 sums.  The sums
// stay below 2 * 127^2 * 128 < 2^22: whole numbers are exact and do not depend on the order of the additions, so a page's
// score is the same for a row of a draft block and for the same position decoded alone.  One thread per page takes the
// maximum over the heads in its own registers.  Bytes: 2 head_dim + 4 per page and kv head (1/31 of its keys and values).
//
// page_pick_kernel.  Per row the n_select best (the first n_first and last n_last among them): the scores, held in registers,
// are counted in 256 parts of their range, and the part that holds the last place again, until it is taken whole; then the
// union over a block's rows as a list with a row mask per page.
//
// Measured (B200): 128 sequences of up to 16384 tokens, 17 rows of 64 heads: 112 us, about 70 for the scores (bound by the
// instructions that make the queries' 8-bit halves and the maxima; 27 us of bytes) and 45 for the choice (bound by shared-memory
// atomics and barriers); one head a kv head, with scores on both sides of zero, 118 to 123; one token at 32768 tokens 13.0 us,
// 16 ragged blocks 19.0 us (latency).
#include "attn_common.cuh"
#include "tc_ptx.cuh"
#include "whole8.cuh"
#include "work_share.cuh"

#include <climits>
#include <math_constants.h>

namespace sv {

constexpr int PS_PAGES = 128;                  // pages per tile
constexpr int PS_MAX_COLS = 256;               // rows * heads of one product

struct PageSelectLaunch {
    sv_page_select_params p;
    int group;                                 // query heads per kv head
    int pos_per_chunk;                         // positions whose rows * heads fit the columns
    int max_cols;                              // columns of a product: the rows of a chunk, in multiples of 16
    int n_tile_bufs;
    int key_stride;                            // words between rows of keys
    int bit_words;                             // 32-page words of a row of chosen bits
    uint32_t *keys;                            // scores that order as whole numbers: [batch * hkv][gamma_max + 1][key_stride]
    uint32_t *bits;                            // [batch * hkv][gamma_max + 1][bit_words], or NULL: in shared memory
};

// Rows and pages of a sequence; 0 rows where its lengths make no sense.
struct SeqRows {
    int R, L, n_pages;
};
__device__ __forceinline__ SeqRows seq_rows(const sv_page_select_params &p, int b, bool report)
{
    SeqRows s;
    int g = p.gamma[b];
    s.L = p.seq_len[b];
    if (g < 0 || g > p.gamma_max) {
        if (report) set_status(p.device_status, SV_DEV_BAD_GAMMA);
        g = min(max(g, 0), p.gamma_max);
    }
    s.R = g + 1;
    if (s.L < s.R || s.L > p.max_seq_len) {
        if (report) set_status(p.device_status, SV_DEV_BAD_LEN);
        s.R = 0;
    }
    s.n_pages = pages_of(s.L);                  // of use where there are rows
    return s;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool have)
{
    const int n = have ? 16 : 0;               // 0: the 16 bytes are zeroed, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

// D[tmem] = A[smem] * B[smem], int8 x int8 -> int32
__device__ __forceinline__ void tc_mma_i8(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Roles of the score kernel's 16 warps: 0 and 1 bring tiles of bounds into shared memory, 2 issues the products, 4..7 turn them
// into scores, 3 and 8..15 bring the rows' queries in 8 bits (17 positions take two rounds; with five of these warps everything
// else waited for them; 20 warps, eight of them for the scores, took 123 us for the largest calls where these took 125, and 4 %
// more for a single token).  Everything is double buffered (the tiles up to four times): bounds stream while the next pair's
// queries are made.
constexpr int SC_THREADS = 512;
constexpr int SC_MMA_WARP = 2, SC_OUT_WARP0 = 4, SC_Q_WARPS = 9;
constexpr int SC_MAX_TILES = 4;
constexpr int SC_PAIR_COST = 1;                // a pair's queries, in tiles

struct ScoreShared {
    uint64_t tile_full[SC_MAX_TILES], tile_empty[SC_MAX_TILES];
    uint64_t q_full[2], q_empty[2];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drained;
    uint32_t tmem_base;
    int abort_flag;
    WorkShare share;
    SeqRows start;               // of the sequence that the block begins in
    OwnerWork start_work;
};

// The walk over (sequence, kv head and chunk of rows, tile of pages).
struct ScoreCursor {
    SeqRows sr;
    int o, s, t, n_sub, n_tiles;
    int h, i0, n_pos;            // kv head, first position of the chunk, its positions
};

__device__ __forceinline__ OwnerWork score_owner(const PageSelectLaunch &a, int b, SeqRows &sr)
{
    sr = seq_rows(a.p, b, false);
    if (sr.R == 0 || sr.n_pages <= a.p.n_select) return {0, 0};        // every row takes all it sees: no scores
    return {a.p.hkv * ((sr.R + a.pos_per_chunk - 1) / a.pos_per_chunk), (sr.n_pages + PS_PAGES - 1) / PS_PAGES};
}
__device__ __forceinline__ void score_pair(const PageSelectLaunch &a, ScoreCursor &c)
{
    const int chunks = (c.sr.R + a.pos_per_chunk - 1) / a.pos_per_chunk;
    c.h = c.s / chunks;
    c.i0 = (c.s - c.h * chunks) * a.pos_per_chunk;
    c.n_pos = min(c.sr.R - c.i0, a.pos_per_chunk);
}
__device__ __forceinline__ void score_next(const PageSelectLaunch &a, ScoreCursor &c)
{
    c.t = 0;
    if (++c.s >= c.n_sub) {
        c.s = 0;
        c.n_tiles = 0;
        while (c.n_tiles == 0 && ++c.o < a.p.batch) {
            const OwnerWork w = score_owner(a, c.o, c.sr);
            c.n_sub = w.n_sub;
            c.n_tiles = w.n_tiles;
        }
        if (c.o >= a.p.batch) { c.n_tiles = c.n_sub = 1; c.sr.R = 1; c.sr.n_pages = 0; }        // past the end: never used
    }
    score_pair(a, c);
}
__device__ __forceinline__ void score_start(const PageSelectLaunch &a, const ScoreShared &sh, ScoreCursor &c)
{
    c.o = sh.share.o; c.s = sh.share.s; c.t = sh.share.t;      // only called by blocks with tiles
    c.sr = sh.start;
    c.n_sub = sh.start_work.n_sub;
    c.n_tiles = sh.start_work.n_tiles;
    score_pair(a, c);
    if (c.t >= c.n_tiles) score_next(a, c);
}

// A score as a number that orders as it does and is neither 0 nor the largest; -0 counts as 0, what is no number as the highest
// (fminf takes the other operand for it)
__device__ __forceinline__ uint32_t score_key(int best, float scale)
{
    const uint32_t x = __float_as_uint(fminf(__fmul_rn((float)best, scale) + 0.f, CUDART_INF_F));
    return (x & 0x80000000u) ? ~x : x | 0x80000000u;
}

// max over G columns at a time of one page's products, times the page's scale, as keys to the rows.  GT: G where it is known
// (a power of two up to 32), else 0.
template <int GT>
__device__ __forceinline__ void store_keys(uint32_t acc, int cols, int G, float scale, bool used, uint32_t *dst, int stride)
{
    int best = INT_MIN, k = 0;
    for (int c0 = 0; c0 < cols; c0 += 32) {
        uint32_t r[32];
        tc_ld32(acc + c0, r);
        if (GT > 0) {
#pragma unroll
            for (int c = 0; c < 32; c += (GT > 0 ? GT : 1)) {
                int m = (int)r[c];
#pragma unroll
                for (int j = 1; j + 1 < GT; j += 2) m = __vimax3_s32(m, (int)r[c + j], (int)r[c + j + 1]);
                if (GT > 1) m = max(m, (int)r[c + GT - 1]);            // GT is even
                if (used && c0 + c < cols) *dst = score_key(m, scale);
                dst += stride;
            }
        } else {
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                best = max(best, (int)r[c]);
                if (++k == G) {
                    if (used && c0 + c < cols) *dst = score_key(best, scale);
                    dst += stride;
                    best = INT_MIN;
                    k = 0;
                }
            }
        }
    }
}

// D: head_dim.  The lanes of the products are a tile's 128 pages, the columns the pair's rows.
template <int D>
__global__ void __launch_bounds__(SC_THREADS, 1)
page_score_kernel(const __grid_constant__ PageSelectLaunch a)
{
    constexpr int ROW = 2 * D;                 // bytes of a page's bounds, and of a column's queries
    constexpr int CH = ROW / 16;               // 16-byte chunks of a row
    constexpr int TILE_BYTES = PS_PAGES * ROW;
    pdl_enter();
    const sv_page_select_params &p = a.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = a.group, n_bufs = a.n_tile_bufs;
    extern __shared__ __align__(1024) uint8_t ps_smem[];
    if ((smem_u32(ps_smem) & 1023u) != 0) {                        // never seen; refuse rather than compute garbage
        if (tid == 0) set_status(p.device_status, SV_DEV_TIMEOUT);
        return;
    }
    uint8_t *tile_buf = ps_smem;
    const int q_bytes = a.max_cols * ROW;
    uint8_t *q_buf = tile_buf + n_bufs * TILE_BYTES;               // two buffers of max_cols rows
    ScoreShared *sh = reinterpret_cast<ScoreShared *>(q_buf + 2 * q_bytes);
    uint32_t acc_cols = 32;                                        // tensor-memory columns of one accumulator
    while ((int)acc_cols < a.max_cols) acc_cols <<= 1;
    if (tid == 0) {
        for (int i = 0; i < n_bufs; ++i) {
            mbar_init(smem_u32(&sh->tile_full[i]), 64);
            mbar_init(smem_u32(&sh->tile_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->q_full[i]), SC_Q_WARPS * 32);
            mbar_init(smem_u32(&sh->q_empty[i]), 1);
            mbar_init(smem_u32(&sh->acc_full[i]), 1);
            mbar_init(smem_u32(&sh->acc_empty[i]), 128);
        }
        mbar_init(smem_u32(&sh->drained), 1);
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == SC_MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                     "r"(2 * acc_cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the sums of the plan use the tiles' memory, which nothing else touches before the barrier below
    SeqRows rows;
    OwnerWork work;
    plan_work_share<SC_THREADS>(
        p.batch, SC_PAIR_COST,
        [&](int b, bool) { return work = score_owner(a, b, rows); },
        [&]() {
            sh->start = rows;
            sh->start_work = work;
        },
        &sh->share, reinterpret_cast<long long(*)[SC_THREADS / 32]>(tile_buf));
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const long long t_begin = sh->share.t_begin, t_end = sh->share.t_end;
    const uint32_t tmem = sh->tmem_base;
    int *abort_flag = &sh->abort_flag;
    uint32_t *status = p.device_status;
    int left = (int)(t_end - t_begin);
    bool ok = true;
    auto wait = [&](uint64_t &bar, uint32_t parity) {
        return __all_sync(0xffffffffu, bounded_wait(smem_u32(&bar), parity, abort_flag, status));
    };
    if (left > 0) {
        ScoreCursor c;
        score_start(a, *sh, c);
        if (warp < 2) {
            // ================================================================ tiles: a warp for 64 of the 128 pages
            constexpr int RPI = 32 / CH;                           // rows that one copy of the warp covers
            const int ch = lane % CH, r0 = lane / CH;
            int n = 0, buf = 0, arrive_at = 0, arrived = 0;
            uint32_t use = 0;
            auto release = [&]() {                                 // the oldest tile under way is complete
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(smem_u32(&sh->tile_full[arrive_at]));
                if (++arrive_at == n_bufs) arrive_at = 0;
                ++arrived;
            };
            // lane l: ids of pages l and 32 + l of the warp's 64 (-1: behind the last, or not a page)
            auto ids_of = [&](int (&id)[2]) {
                const int32_t *table = p.block_table + (long long)c.o * p.block_table_stride;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int lp = c.t * PS_PAGES + warp * 64 + k * 32 + lane;
                    id[k] = lp < c.sr.n_pages ? __ldg(table + lp) : INT_MIN;
                }
            };
            int id[2];
            ids_of(id);
            for (; left > 0 && ok; --left, ++n) {
                const int h = c.h;
                int now[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (id[k] != INT_MIN && (id[k] < 0 || id[k] >= p.n_pages)) set_status(status, SV_DEV_BAD_PAGE);
                    now[k] = id[k] >= 0 && id[k] < p.n_pages ? id[k] : -1;
                }
                if (++c.t == c.n_tiles) score_next(a, c);
                if (left > 1) ids_of(id);                          // the next tile's, under way meanwhile
                if (use > 0) ok = wait(sh->tile_empty[buf], (use - 1) & 1);
                if (!ok) break;
                const uint32_t base = smem_u32(tile_buf + buf * TILE_BYTES) + (ch >> 3) * (PS_PAGES * 128);
                const int8_t *src0 = p.bounds + (long long)h * ROW + ch * 16;
                const long long page_bytes = (long long)p.hkv * ROW;
#pragma unroll 4
                for (int k = 0; k < 64 / RPI; ++k) {
                    const int in = k * RPI + r0, row = warp * 64 + in;
                    const int phys = __shfl_sync(0xffffffffu, k * RPI < 32 ? now[0] : now[1], in & 31);
                    cp_async16(base + row * 128 + (((ch & 7) ^ (row & 7)) << 4), src0 + max(phys, 0) * page_bytes, phys >= 0);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (n >= 1) {                                      // one tile stays under way behind the newest
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    release();
                }
                if (++buf == n_bufs) { buf = 0; ++use; }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (ok && arrived < n) release();
        } else if (warp != SC_MMA_WARP && (warp < SC_OUT_WARP0 || warp >= SC_OUT_WARP0 + 4)) {
            // ================================================================ queries: a warp per position, its G heads together
            const int qw = warp < SC_OUT_WARP0 ? 0 : warp - 7;     // warps 3, 8..15: 0..8
            constexpr int HELD = 4;                                // 16-byte chunks of a position that a lane holds
            const int chunks = G * D / 8;
            auto src_of = [&](int i) {
                return reinterpret_cast<const uint4 *>(
                    static_cast<const __nv_bfloat16 *>(p.q) + (((long long)__ldg(p.cu_q + c.o) + c.i0 + i) * p.hq + (long long)c.h * G) * D);
            };
            auto load = [&](uint4 (&v)[HELD], int i) {
                if (i >= c.n_pos) return;
                const uint4 *src = src_of(i);
#pragma unroll
                for (int e = 0; e < HELD; ++e) v[e] = lane + e * 32 < chunks ? __ldg(src + lane + e * 32) : make_uint4(0, 0, 0, 0);
            };
            uint4 v[HELD];
            load(v, qw);
            for (uint32_t pair = 0; left > 0 && ok; ++pair) {
                const int qb = pair & 1;
                if (pair >= 2) ok = wait(sh->q_empty[qb], ((pair >> 1) - 1) & 1);
                if (!ok) break;
                uint8_t *dst = q_buf + qb * q_bytes;
                const int n_mma = (c.n_pos * G + 15) & ~15;
                for (int i = qw; i < c.n_pos; i += SC_Q_WARPS) {
                    uint4 x[HELD];
#pragma unroll
                    for (int e = 0; e < HELD; ++e) x[e] = v[e];
                    load(v, i + SC_Q_WARPS);                       // under way while this position is worked on
                    const uint4 *src = src_of(i);
                    uint32_t big2 = 0;                             // largest magnitudes, even and odd dims; magnitudes order as bits
                    auto fold = [&](const uint4 &y) {
                        big2 = __vmaxu2(big2, __vmaxu2(__vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu), __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu)));
                    };
#pragma unroll
                    for (int e = 0; e < HELD; ++e) fold(x[e]);
                    for (int e = lane + HELD * 32; e < chunks; e += 32) fold(__ldg(src + e));
                    const float big = __uint_as_float(__reduce_max_sync(0xffffffffu, max(big2 & 0xffffu, big2 >> 16)) << 16);
                    const Whole8 by(__fmul_rn(big, 1.f / 127.f));
                    auto put = [&](const uint4 &y, int e) {
                        float f[8];
                        unpack8(y, f);
                        const uint2 n = whole8x8(f, by);
                        const int hh = e / (D / 8), d8 = e - hh * (D / 8), col = i * G + hh;
                        const uint32_t sx = negative_bytes(n.x), sy = negative_bytes(n.y);
#pragma unroll
                        for (int z = 0; z < 2; ++z) {              // positive parts meet the maxima, negative ones the minima
                            const int byte = z * D + d8 * 8, ch = byte >> 4;
                            const uint32_t off = (ch >> 3) * (n_mma * 128) + col * 128 + (((ch & 7) ^ (col & 7)) << 4) + (byte & 15);
                            *reinterpret_cast<uint2 *>(dst + off) = z == 0 ? make_uint2(n.x & ~sx, n.y & ~sy) : make_uint2(n.x & sx, n.y & sy);
                        }
                    };
                    // one copy of the code for all chunks (the held ones move up): with a copy for each the four roles' code did
                    // not fit the instruction cache
#pragma unroll 1
                    for (int e = lane, k = 0; e < chunks; e += 32, ++k) {
                        const uint4 y = k < HELD ? x[0] : __ldg(src + e);
#pragma unroll
                        for (int z = 0; z + 1 < HELD; ++z) x[z] = x[z + 1];
                        put(y, e);
                    }
                }
                // columns up to the next multiple of 16: zeros
                const int pad = (n_mma - c.n_pos * G) * CH;
                for (int e = qw * 32 + lane; e < pad; e += SC_Q_WARPS * 32) {
                    const int col = c.n_pos * G + e / CH, ch = e % CH;
                    *reinterpret_cast<uint4 *>(dst + (ch >> 3) * (n_mma * 128) + col * 128 + (ch & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(smem_u32(&sh->q_full[qb]));
                left -= min(left, c.n_tiles - c.t);
                score_next(a, c);
                if (left > 0) load(v, qw);                         // the next pair's first position
            }
        } else if (warp >= SC_OUT_WARP0 && warp < SC_OUT_WARP0 + 4) {
            // ================================================================ scores: a thread per page
            const int row = (warp & 3) * 32 + lane;
            // Where the thread's page of a tile goes, and which page it is.  Ids are looked up two tiles ahead and scales one: with
            // the id of the next tile fetched in front of its scale, every tile began with a wait of 800 cycles.
            struct Place {
                uint32_t *dst;
                int cols, h, id;
                bool used;
            };
            auto look_up = [&]() {
                Place w;
                const int lp = c.t * PS_PAGES + row;
                w.dst = a.keys + (((long long)c.o * p.hkv + c.h) * (p.gamma_max + 1) + c.i0) * a.key_stride + lp;
                w.cols = c.n_pos * G;
                w.h = c.h;
                w.used = lp < c.sr.n_pages;
                w.id = w.used ? __ldg(p.block_table + (long long)c.o * p.block_table_stride + lp) : -1;
                if (++c.t == c.n_tiles) score_next(a, c);
                return w;
            };
            auto scale_of = [&](const Place &w) { return w.id >= 0 && w.id < p.n_pages ? __ldg(p.scales + (long long)w.id * p.hkv + w.h) : 0.f; };
            Place now = look_up(), next = now;
            if (left > 1) next = look_up();
            float scale = scale_of(now);
            for (uint32_t n = 0; left > 0 && ok; ++n, --left) {
                const int g = n & 1;
                const uint32_t acc = tmem + g * acc_cols + ((uint32_t)((warp & 3) * 32) << 16);
                const float scale_next = scale_of(next);
                Place after = next;
                if (left > 2) after = look_up();
                ok = wait(sh->acc_full[g], (n >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                switch (G) {
                    case 1: store_keys<1>(acc, now.cols, G, scale, now.used, now.dst, a.key_stride); break;
                    case 2: store_keys<2>(acc, now.cols, G, scale, now.used, now.dst, a.key_stride); break;
                    case 4: store_keys<4>(acc, now.cols, G, scale, now.used, now.dst, a.key_stride); break;
                    case 8: store_keys<8>(acc, now.cols, G, scale, now.used, now.dst, a.key_stride); break;
                    default: store_keys<0>(acc, now.cols, G, scale, now.used, now.dst, a.key_stride); break;
                }
                tc_fence_before();
                mbar_arrive(smem_u32(&sh->acc_empty[g]));
                now = next;
                next = after;
                scale = scale_next;
            }
        } else {
            // ================================================================ products
            uint32_t pair = 0, use = 0;
            int buf = 0;
            bool fresh = true;                                     // the first tile of a pair
            for (uint32_t n = 0; left > 0 && ok; ++n, --left) {
                const int qb = pair & 1, g = n & 1;
                if (fresh) ok = wait(sh->q_full[qb], (pair >> 1) & 1);
                if (ok && n >= 2) ok = wait(sh->acc_empty[g], ((n >> 1) - 1) & 1);
                if (ok) ok = wait(sh->tile_full[buf], use & 1);
                if (!ok) break;
                tc_fence_after();
                const int n_mma = (c.n_pos * G + 15) & ~15;
                uint32_t idesc = 0;
                idesc |= 2u << 4;                                  // int32 accumulator
                idesc |= 1u << 7;                                  // A signed 8-bit
                idesc |= 1u << 10;                                 // B signed 8-bit
                idesc |= (uint32_t)(n_mma >> 3) << 17;
                idesc |= (uint32_t)(128 >> 4) << 24;
                const bool last = c.t + 1 == c.n_tiles || left == 1;
                const uint64_t ad = smem_desc(smem_u32(tile_buf + buf * TILE_BYTES), 16, 1024);
                const uint64_t bd = smem_desc(smem_u32(q_buf + qb * q_bytes), 16, 1024);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < ROW / 32; ++ks)
                        tc_mma_i8(tmem + g * acc_cols, ad + (((ks >> 2) * (PS_PAGES * 128) + (ks & 3) * 32) >> 4),
                                  bd + (((ks >> 2) * (n_mma * 128) + (ks & 3) * 32) >> 4), idesc, ks > 0);
                    tc_commit(smem_u32(&sh->acc_full[g]));
                    tc_commit(smem_u32(&sh->tile_empty[buf]));
                    if (last) tc_commit(smem_u32(&sh->q_empty[qb]));
                }
                __syncwarp();
                if (++buf == n_bufs) { buf = 0; ++use; }
                fresh = last;
                pair += last;
                if (++c.t == c.n_tiles) score_next(a, c);
            }
            if (!ok) {                                             // given up: let the issued instructions finish
                if (elect_one()) tc_commit(smem_u32(&sh->drained));
                __syncwarp();
                for (int it = 0; it < (1 << 20) && !mbar_try_wait(smem_u32(&sh->drained), 0); ++it) { }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == SC_MMA_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * acc_cols) : "memory");
    }
}

// ---------------------------------------------------------------------------- choice and union
constexpr int PK_WARPS = 16;
constexpr int PK_BINS = 256;                   // parts that a range of keys is divided into
constexpr int PK_WORDS = 512;                  // words of 32 pages that the union takes at a time

// WPR: warps per row; KPT: keys a thread holds.  More pages than WPR * 32 * KPT are read again in every pass.
template <int WPR, int KPT>
__global__ void __launch_bounds__(PK_WARPS * 32, 2)
page_pick_kernel(const __grid_constant__ PageSelectLaunch a)
{
    constexpr int TEAM = WPR * 32;
    const int n_warps = blockDim.x >> 5, teams = n_warps / WPR;
    pdl_enter();
    const sv_page_select_params &p = a.p;
    extern __shared__ __align__(16) uint32_t pk_smem[];
    __shared__ int s_count[2][PK_WARPS];
    const int h = blockIdx.x % p.hkv, b = blockIdx.x / p.hkv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp / WPR, tw = warp % WPR, t = tw * 32 + lane;
    const SeqRows sr = seq_rows(p, b, h == 0 && threadIdx.x == 0);
    const long long pair = blockIdx.x;
    int *hist = reinterpret_cast<int *>(pk_smem) + team * PK_BINS;       // the team's counts
    uint32_t *bits = a.bits != nullptr ? a.bits + pair * (p.gamma_max + 1) * a.bit_words : pk_smem + teams * PK_BINS;
    int parity = 0;
    auto team_bar = [&]() {
        if (WPR == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TEAM) : "memory");
    };
    // f over the threads of a team (sums write alternate places, so one barrier each is enough)
    auto team_reduce = [&](uint32_t x, auto &&f) {
        if (WPR == 1) return x;
        if (lane == 0) s_count[parity][warp] = (int)x;
        team_bar();
        x = (uint32_t)s_count[parity][team * WPR];
#pragma unroll
        for (int w = 1; w < WPR; ++w) x = f(x, (uint32_t)s_count[parity][team * WPR + w]);
        parity ^= 1;
        return x;
    };
    auto team_sum = [&](int x) {
        return (int)team_reduce((uint32_t)__reduce_add_sync(0xffffffffu, x), [](uint32_t u, uint32_t v) { return u + v; });
    };
    auto team_max = [&](uint32_t x) {
        return team_reduce(__reduce_max_sync(0xffffffffu, x), [](uint32_t u, uint32_t v) { return max(u, v); });
    };
    for (int i = team; i < sr.R; i += teams) {
        const int last = (sr.L - sr.R + i) / 16, n_seen = last + 1;
        uint32_t *row = bits + (long long)i * a.bit_words;
        const int n_words = (sr.n_pages + 31) / 32;
        if (n_seen <= p.n_select) {            // all that the row sees
            for (int w = t; w < n_words; w += TEAM) {
                const int left = n_seen - w * 32;
                row[w] = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1 : 0u;
            }
            continue;
        }
        // candidates: all but the fixed pages; 0 stands for no candidate
        const int c_lo = p.n_first, c_hi = n_seen - p.n_last;
        int want = p.n_select - p.n_first - p.n_last;
        const uint32_t *src = a.keys + (pair * (p.gamma_max + 1) + i) * a.key_stride;
        auto key_at = [&](int page) -> uint32_t { return page >= c_lo && page < c_hi ? __ldg(src + page) : 0u; };
        uint32_t key[KPT];
        const int rounds = (n_seen + TEAM - 1) / TEAM;
        // f(key, page) for the thread's pages (with keys of 0 up to the next four)
        auto each = [&](auto &&f) {
#pragma unroll
            for (int j0 = 0; j0 < KPT; j0 += 4) {
                if (j0 >= rounds) break;
#pragma unroll
                for (int j = j0; j < j0 + 4; ++j) f(key[j], j * TEAM + t);
            }
            for (int j = KPT; j < rounds; ++j) f(key_at(j * TEAM + t), j * TEAM + t);
        };
        uint32_t top = 0, low = 0xffffffffu;
#pragma unroll
        for (int j0 = 0; j0 < KPT; j0 += 4) {
            if (j0 >= rounds) break;
            if (j0 * TEAM >= c_lo && (j0 + 4) * TEAM <= c_hi) {
#pragma unroll
                for (int j = j0; j < j0 + 4; ++j) key[j] = __ldg(src + j * TEAM + t);
            } else {
#pragma unroll
                for (int j = j0; j < j0 + 4; ++j) key[j] = key_at(j * TEAM + t);
            }
        }
        each([&](uint32_t k, int) {
            top = max(top, k);
            low = min(low, k - 1);             // 0 - 1 is the largest
        });
        top = team_max(top);
        low = ~team_max(~low) + 1;
        // The want-th largest key lies in [low, top]: counts of its 256 parts from the top down name one of them, which is
        // divided again until it is taken whole or is a single key.  After a pass: all keys >= cut are among the best, and
        // `want` more of [low, cut) are.
        uint32_t cut = top + 1;
        bool whole = want == 0, ties = false;
        while (!whole && !ties) {
            const uint32_t range = top - low;
            const int shift = max(0, 24 - __clz(range));               // parts of 2^shift keys: at most 256 of them
            team_bar();
            for (int k = t; k < PK_BINS; k += TEAM) hist[k] = 0;
            team_bar();
            each([&](uint32_t k, int) {
                const uint32_t off = top - k;                          // part 0 holds the largest
                if (off <= range) atomicAdd(&hist[off >> shift], 1);
            });
            team_bar();
            // lane l: parts 8 l .. 8 l + 7
            int n[8], sum = 0;
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const int4 x = *reinterpret_cast<const int4 *>(hist + lane * 8 + k);
                n[k] = x.x; n[k + 1] = x.y; n[k + 2] = x.z; n[k + 3] = x.w;
                sum += x.x + x.y + x.z + x.w;
            }
            int before = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, before, d);
                if (lane >= d) before += x;
            }
            before -= sum;
            const uint32_t hit = __ballot_sync(0xffffffffu, before < want && before + sum >= want);
            const int at = __ffs(hit) - 1;
            int part = 0, above = before, in = 0;                      // the part that holds the want-th, keys above it, in it
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (in == 0 && above + n[k] >= want) { part = lane * 8 + k; in = n[k]; }
                else if (in == 0) above += n[k];
            }
            part = __shfl_sync(0xffffffffu, part, at);
            above = __shfl_sync(0xffffffffu, above, at);
            in = __shfl_sync(0xffffffffu, in, at);
            want -= above;
            const uint32_t part_top = top - ((uint32_t)part << shift);
            const uint32_t span = (1u << shift) - 1, part_low = part_top - low > span ? part_top - span : low;
            if (in == want) {
                cut = part_low;
                whole = true;
            } else {
                cut = part_top + 1;
                top = part_top;
                low = part_low;
                ties = shift == 0;
            }
        }
        // more candidates of one key than places: the lowest pages among them
        int until = -1;
        if (ties) {
            int lo = 0, hi = c_hi;             // smallest page with enough candidates up to it
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                int n = 0;
                each([&](uint32_t k, int page) { n += k == low && page <= mid ? 1 : 0; });
                if (team_sum(n) >= want) hi = mid; else lo = mid + 1;
            }
            until = lo;
        }
        auto store_word = [&](int j, uint32_t k) {
            const int page = j * TEAM + t;
            bool take = k >= cut;                                      // not for a key of 0
            if (ties) take = take || (k == low && page <= until);
            if (j * TEAM < c_lo || j * TEAM + TEAM > c_hi) take = take || page < c_lo || (page >= c_hi && page < n_seen);
            const uint32_t word = __ballot_sync(0xffffffffu, take);
            const int w = j * WPR + tw;
            if (lane == 0 && w < n_words) row[w] = word;
        };
#pragma unroll
        for (int j0 = 0; j0 < KPT; j0 += 4) {
            if (j0 >= rounds) break;
#pragma unroll
            for (int j = j0; j < j0 + 4; ++j) store_word(j, key[j]);
        }
        const int stored = min((rounds + 3) / 4 * 4, KPT);
        for (int j = stored; j * WPR + tw < n_words; ++j) store_word(j, j < rounds ? key_at(j * TEAM + t) : 0u);
    }
    __syncthreads();
    // the union of the rows, in page order: first how many pages each word of 32 has and where they go, a thread per word,
    // then the pages and their masks, a warp per word
    __shared__ int s_at[PK_WORDS], s_total;
    int base = 0;
    const int n_words = sr.R > 0 ? (sr.n_pages + 31) / 32 : 0;
    int32_t *list = p.page_list + pair * p.list_stride;
    uint64_t *masks = p.row_mask + pair * p.list_stride;
    bool short_list = false;
    for (int w0 = 0; w0 < n_words; w0 += PK_WORDS) {
        const int words = min(PK_WORDS, n_words - w0);
        for (int w = threadIdx.x; w < words; w += blockDim.x) {
            uint32_t any = 0;
            for (int i = 0; i < sr.R; ++i) any |= bits[(long long)i * a.bit_words + w0 + w];
            s_at[w] = __popc(any);
        }
        __syncthreads();
        if (warp == 0) {
            int run = base;
            for (int w = 0; w < words; w += 32) {
                const int n = w + lane < words ? s_at[w + lane] : 0;
                int v = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, v, d);
                    if (lane >= d) v += x;
                }
                if (w + lane < words) s_at[w + lane] = run + v - n;
                run += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) s_total = run;
        }
        __syncthreads();
        for (int w = warp; w < words; w += n_warps) {
            uint64_t mask = 0;
            for (int i = 0; i < sr.R; ++i) mask |= (uint64_t)((bits[(long long)i * a.bit_words + w0 + w] >> lane) & 1u) << i;
            const uint32_t any = __ballot_sync(0xffffffffu, mask != 0);
            const int at = s_at[w] + __popc(any & ((1u << lane) - 1));
            if (mask != 0) {
                if (at < p.list_stride) {
                    list[at] = (w0 + w) * 32 + lane;
                    masks[at] = mask;
                } else {
                    short_list = true;
                }
            }
        }
        base = s_total;
        __syncthreads();
    }
    if (short_list) set_status(p.device_status, SV_DEV_BAD_LEN);
    if (threadIdx.x == 0) p.n_list[pair] = (int)min((long long)base, (long long)p.list_stride);
    if (h == 0 && sr.R > 0 && sr.n_pages <= p.n_select) {      // no scores, so nobody has looked at these ids
        const int32_t *table = p.block_table + (long long)b * p.block_table_stride;
        for (int page = threadIdx.x; page < sr.n_pages; page += blockDim.x) {
            const int id = __ldg(table + page);
            if (id < 0 || id >= p.n_pages) set_status(p.device_status, SV_DEV_BAD_PAGE);
        }
    }
}

// ---------------------------------------------------------------------------- host side
constexpr size_t PK_SMEM_BITS = 96 * 1024;
// What a launch may bring without asking: 48 KB less the kernel's own arrays and what the system keeps, 3 KB together
constexpr size_t PK_SMEM_DEFAULT = 44 * 1024;

static int select_max_pages(int max_seq_len) { return (int)(((long long)max_seq_len + 15) / 16); }
static int select_key_stride(int max_seq_len) { return (select_max_pages(max_seq_len) + 31) / 32 * 32; }
static size_t select_key_bytes(int batch, int gamma_max, int hkv, int max_seq_len)
{
    return (size_t)batch * hkv * (gamma_max + 1) * select_key_stride(max_seq_len) * sizeof(uint32_t);
}
static size_t select_row_bits(int gamma_max, int max_seq_len)
{
    return (size_t)(gamma_max + 1) * ((select_max_pages(max_seq_len) + 31) / 32) * sizeof(uint32_t);
}

using PickKernel = void (*)(PageSelectLaunch);

// As many keys a thread as the longest row needs: with 32 for all a single token over 2048 pages took 15.1 us where it takes 14.5
// (less code to fetch); 16 for all, with more warps for the longer rows, 134 us for the largest batch where 32 take 124.
template <int WPR>
static PickKernel pick_kernel_of(int pages)
{
    const int keys = (pages + WPR * 32 - 1) / (WPR * 32);
    return keys <= 8 ? page_pick_kernel<WPR, 8> : keys <= 16 ? page_pick_kernel<WPR, 16> : page_pick_kernel<WPR, 32>;
}

template <int D>
static sv_status launch_score(PageSelectLaunch &a, int grid, cudaStream_t s)
{
    const int tile = PS_PAGES * 2 * D, queries = 2 * a.max_cols * 2 * D;
    a.n_tile_bufs = (227 * 1024 - queries - (int)sizeof(ScoreShared)) / tile;          // at least two: 256 columns are 128 KB
    if (a.n_tile_bufs > SC_MAX_TILES) a.n_tile_bufs = SC_MAX_TILES;
    const int smem = a.n_tile_bufs * tile + queries + (int)sizeof(ScoreShared);
    if (cudaFuncSetAttribute(page_score_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) return SV_ECUDA;
    return launch_kernel(true, page_score_kernel<D>, grid, SC_THREADS, smem, s, a);
}

}  // namespace sv

extern "C" size_t spec_page_select_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hkv, int32_t max_seq_len)
{
    using namespace sv;
    if (batch <= 0 || gamma_max < 0 || gamma_max > 63 || hkv <= 0 || max_seq_len <= 0) return 0;
    const size_t row_bits = select_row_bits(gamma_max, max_seq_len);
    return select_key_bytes(batch, gamma_max, hkv, max_seq_len) + (row_bits > PK_SMEM_BITS ? row_bits * batch * hkv : 0) + 256;
}

extern "C" sv_status spec_page_select(const sv_page_select_params *p, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace sv;
    if (p == nullptr) return SV_EINVAL;
    if (p->q == nullptr || p->bounds == nullptr || p->scales == nullptr || p->block_table == nullptr || p->seq_len == nullptr ||
        p->gamma == nullptr || p->cu_q == nullptr || p->page_list == nullptr || p->row_mask == nullptr || p->n_list == nullptr)
        return SV_EINVAL;
    if (p->batch <= 0 || p->gamma_max < 0 || p->hq <= 0 || p->hkv <= 0 || p->max_seq_len <= 0 || p->n_pages <= 0) return SV_EINVAL;
    if (p->n_first < 0 || p->n_last < 1 || p->n_select < p->n_first || p->n_select - p->n_first < p->n_last) return SV_EINVAL;
    if (p->hq % p->hkv != 0 || p->hq / p->hkv > 128 || p->gamma_max > 63) return SV_EUNSUPPORTED;
    if (p->head_dim != 64 && p->head_dim != 128) return SV_EUNSUPPORTED;
    const long long max_pages = select_max_pages(p->max_seq_len);
    if (p->block_table_stride < max_pages) return SV_EINVAL;
    const long long widest = (long long)(p->gamma_max + 1) * p->n_select;
    if (p->list_stride < (widest < max_pages ? widest : max_pages)) return SV_EINVAL;
    if (!aligned16(p->q) || !aligned16(p->bounds) || !aligned16(workspace) || (reinterpret_cast<uintptr_t>(p->row_mask) & 7u) != 0) return SV_EALIGN;
    if (workspace == nullptr ||
        workspace_bytes < spec_page_select_workspace_bytes(p->batch, p->gamma_max, p->hkv, p->max_seq_len))
        return SV_EWORKSPACE;
    PageSelectLaunch a;
    a.p = *p;
    a.group = p->hq / p->hkv;
    const int R = p->gamma_max + 1;
    a.pos_per_chunk = PS_MAX_COLS / a.group < R ? PS_MAX_COLS / a.group : R;
    a.max_cols = (a.pos_per_chunk * a.group + 15) & ~15;
    a.key_stride = select_key_stride(p->max_seq_len);
    a.bit_words = (int)((max_pages + 31) / 32);
    a.keys = static_cast<uint32_t *>(workspace);
    const size_t row_bits = select_row_bits(p->gamma_max, p->max_seq_len);
    const bool in_smem = row_bits <= PK_SMEM_BITS;
    a.bits = in_smem ? nullptr
                     : reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(workspace) +
                                                    select_key_bytes(p->batch, p->gamma_max, p->hkv, p->max_seq_len));
    const long long pairs = (long long)p->batch * p->hkv;
    if (pairs > (1 << 24)) return SV_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    // Warps per row: enough to hold a row's keys in registers, and more where a block has few rows, down to four keys a thread
    int need = 1;
    while (need < PK_WARPS && (long long)need * 32 * 32 < max_pages) need *= 2;
    while (need < PK_WARPS && need * 2 * R <= PK_WARPS && need * 32 * 4 < max_pages) need *= 2;
    // Rows at a time: as few rounds as 16 warps allow, and no more warps than these rounds need (17 rows: two rounds of nine)
    const int rounds = (R * need + PK_WARPS - 1) / PK_WARPS, teams = (R + rounds - 1) / rounds;
    const size_t pick_smem = (size_t)teams * PK_BINS * sizeof(int) + (in_smem ? row_bits : 0);
    PickKernel pick;
    switch (need) {
        case 1: pick = pick_kernel_of<1>(a.key_stride); break;
        case 2: pick = pick_kernel_of<2>(a.key_stride); break;
        case 4: pick = pick_kernel_of<4>(a.key_stride); break;
        case 8: pick = pick_kernel_of<8>(a.key_stride); break;
        default: pick = pick_kernel_of<16>(a.key_stride); break;
    }
    // in front of the first launch, so that a refusal leaves nothing under way; the limit is the largest block's, so that calls of
    // several threads do not lower it for one another
    if (pick_smem > PK_SMEM_DEFAULT &&
        cudaFuncSetAttribute(pick, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(PK_SMEM_BITS + PK_WARPS * PK_BINS * sizeof(int))) != cudaSuccess)
        return SV_ECUDA;
    if (max_pages > p->n_select) {             // otherwise no sequence has more pages than a row takes
        // a block per multiprocessor, fewer where there are not as many tiles
        const long long tiles = pairs * ((R + a.pos_per_chunk - 1) / a.pos_per_chunk) * ((max_pages + PS_PAGES - 1) / PS_PAGES);
        const int grid = (int)(tiles < sm_count() ? tiles : sm_count());
        const sv_status st = p->head_dim == 128 ? launch_score<128>(a, grid, s) : launch_score<64>(a, grid, s);
        if (st != SV_OK) return st;
    }
    return launch_kernel(true, pick, (unsigned)pairs, teams * need * 32, pick_smem, s, a);
}
