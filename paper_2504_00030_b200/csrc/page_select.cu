// Selection of the pages that each row of a draft block reads (spec_page_select), two kernels.
//
// page_score_kernel.  The score of a page is an upper estimate of what any of its keys can give with the row's queries,
//     max over the group's heads h of  sum_d max(q_hd M_d, q_hd m_d),
// with the queries in 8 bits (one scale per row and kv head, which no comparison needs) and the page's bounds M, m in 8
// bits times the page's scale.  max(q M, q m) = max(q, 0) M + min(q, 0) m, so it is an integer matrix product of depth
// 2 head_dim: 128 pages (tensor-memory lanes) times rows * heads (columns), tcgen05.mma kind::i8 with int32 sums.  The sums
// stay below 2 * 127^2 * 128 < 2^22: whole numbers are exact and do not depend on the order of the additions, so a page's
// score is the same for a row of a draft block and for the same position decoded alone.  One thread per page takes the
// maximum over the heads in its own registers.  Bytes: 2 head_dim + 4 per page and kv head (1/31 of its keys and values).
//
// page_pick_kernel.  Per row the n_select best (the first n_first and last n_last among them) by bisection over the bits
// of the scores, held in registers; then the union over a block's rows as a list with a row mask per page.
#include "attn_common.cuh"
#include "tc_ptx.cuh"

#include <climits>

namespace sv {

constexpr int PS_PAGES = 128;                  // pages per tile
constexpr int PS_MAX_COLS = 256;               // rows * heads of one product

struct PageSelectLaunch {
    sv_page_select_params p;
    int group;                                 // query heads per kv head
    int pos_per_chunk;                         // positions whose rows * heads fit the columns
    int n_chunks;
    int tiles_per_block;
    int max_pages;                             // of a sequence
    int score_stride;                          // floats between rows of scores
    int bit_words;                             // 32-page words of a row of chosen bits
    float *scores;                             // [batch * hkv][gamma_max + 1][score_stride]
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
    s.n_pages = (s.L + 15) / 16;
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

struct ScoreShared {
    uint64_t done;
    uint32_t tmem_base;
    int abort_flag;
};

// D: head_dim.  128 threads; thread t owns page t of a tile.
template <int D>
__global__ void __launch_bounds__(128)
page_score_kernel(const __grid_constant__ PageSelectLaunch a)
{
    constexpr int ROW = 2 * D;                 // bytes of a page's bounds, and of a column's queries
    constexpr int CH = ROW / 16;               // 16-byte chunks of a row
    constexpr int TILE_BYTES = PS_PAGES * ROW;
    pdl_enter();
    const sv_page_select_params &p = a.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.y, b = blockIdx.z / a.n_chunks, chunk = blockIdx.z - b * a.n_chunks;
    const SeqRows sr = seq_rows(p, b, false);
    const int i0 = chunk * a.pos_per_chunk, n_pos = min(sr.R - i0, a.pos_per_chunk);
    const int tile0 = blockIdx.x * a.tiles_per_block;
    if (n_pos <= 0 || tile0 * PS_PAGES >= sr.n_pages) return;
    if (sr.n_pages <= p.n_select) return;      // every row takes all it sees
    const int tiles = min(a.tiles_per_block, (sr.n_pages - tile0 * PS_PAGES + PS_PAGES - 1) / PS_PAGES);
    const int G = a.group, cols = n_pos * G, n_mma = (cols + 15) & ~15;

    extern __shared__ __align__(1024) uint8_t ps_smem[];
    uint8_t *tile_buf = ps_smem;                                   // two tiles
    uint8_t *q_buf = ps_smem + 2 * TILE_BYTES;                     // n_mma rows
    ScoreShared *sh = reinterpret_cast<ScoreShared *>(q_buf + (size_t)((a.pos_per_chunk * G + 15) & ~15) * ROW);
    if ((smem_u32(ps_smem) & 1023u) != 0) {                        // never seen; refuse rather than compute garbage
        if (tid == 0) set_status(p.device_status, SV_DEV_TIMEOUT);
        return;
    }
    uint32_t tmem_cols = 32;
    while ((int)tmem_cols < n_mma) tmem_cols <<= 1;
    if (tid == 0) {
        mbar_init(smem_u32(&sh->done), 1);
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                     "r"(tmem_cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const int32_t *table = p.block_table + (long long)b * p.block_table_stride;
    // a tile's bounds: chunk tid % CH of rows tid / CH + k * (128 / CH)
    auto fetch = [&](int t) {
        const int c = tid % CH;
        const uint32_t base = smem_u32(tile_buf + (t & 1) * TILE_BYTES) + (c >> 3) * (PS_PAGES * 128);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int row = tid / CH + k * (128 / CH);
            const int lp = (tile0 + t) * PS_PAGES + row;
            const int phys = lp < sr.n_pages ? table[lp] : -1;
            const bool have = phys >= 0 && phys < p.n_pages;
            if (lp < sr.n_pages && !have && c == 0) set_status(p.device_status, SV_DEV_BAD_PAGE);
            const int8_t *src = p.bounds + ((long long)(have ? phys : 0) * p.hkv + h) * ROW + c * 16;
            cp_async16(base + row * 128 + (((c & 7) ^ (row & 7)) << 4), src, have);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch(0);
    // the rows' queries in 8 bits: a warp per position, its G heads together (one scale)
    for (int i = warp; i < (n_mma + G - 1) / G; i += 4) {
        const bool used = i < n_pos;
        const __nv_bfloat162 *src = reinterpret_cast<const __nv_bfloat162 *>(
            static_cast<const __nv_bfloat16 *>(p.q) + (((long long)p.cu_q[b] + i0 + (used ? i : 0)) * p.hq + (long long)h * G) * D);
        float big = 0.f;
        if (used)
            for (int e = lane; e < G * D / 2; e += 32) {
                const float2 f = __bfloat1622float2(src[e]);
                big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
        const float scale = __fmul_rn(big, 1.f / 127.f);
        for (int e = lane; e < G * D / 4; e += 32) {               // four dims of a head
            const int hh = e / (D / 4), d4 = e - hh * (D / 4), col = i * G + hh;
            if (col >= n_mma) break;
            uint32_t pos = 0, neg = 0;
            if (used && scale > 0.f) {
                const float2 f0 = __bfloat1622float2(src[e * 2]), f1 = __bfloat1622float2(src[e * 2 + 1]);
                const float f[4] = {f0.x, f0.y, f1.x, f1.y};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int n = min(max(__float2int_rn(__fdiv_rn(f[c], scale)), -127), 127);
                    pos |= (uint32_t)max(n, 0) << (8 * c);
                    neg |= (uint32_t)(min(n, 0) & 255) << (8 * c);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {                          // positive parts meet the maxima, negative ones the minima
                const int byte = s * D + d4 * 4, ch = byte >> 4;
                const uint32_t off = (ch >> 3) * (n_mma * 128) + col * 128 + (((ch & 7) ^ (col & 7)) << 4) + (byte & 15);
                *reinterpret_cast<uint32_t *>(q_buf + off) = s == 0 ? pos : neg;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    uint32_t idesc = 0;
    idesc |= 2u << 4;                          // int32 accumulator
    idesc |= 1u << 7;                          // A signed 8-bit
    idesc |= 1u << 10;                         // B signed 8-bit
    idesc |= (uint32_t)(n_mma >> 3) << 17;
    idesc |= (uint32_t)(128 >> 4) << 24;
    bool ok = true;
    for (int t = 0; t < tiles; ++t) {
        if (t + 1 < tiles) {
            fetch(t + 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();                     // the accumulator was read by the tile before
        if (__syncthreads_or(!ok)) break;      // a wait ran out: every thread leaves at the same barrier
        tc_fence_after();
        if (warp == 0) {
            if (elect_one()) {
                const uint64_t ad = smem_desc(smem_u32(tile_buf + (t & 1) * TILE_BYTES), 16, 1024);
                const uint64_t bd = smem_desc(smem_u32(q_buf), 16, 1024);
#pragma unroll
                for (int ks = 0; ks < ROW / 32; ++ks)
                    tc_mma_i8(tmem, ad + (((ks >> 2) * (PS_PAGES * 128) + (ks & 3) * 32) >> 4),
                              bd + (((ks >> 2) * (n_mma * 128) + (ks & 3) * 32) >> 4), idesc, ks > 0);
                tc_commit(smem_u32(&sh->done));
            }
            __syncwarp();
        }
        const int lp = (tile0 + t) * PS_PAGES + tid;
        const int phys = lp < sr.n_pages ? table[lp] : -1;
        const float scale = phys >= 0 && phys < p.n_pages ? p.scales[(long long)phys * p.hkv + h] : 0.f;
        ok = bounded_wait(smem_u32(&sh->done), t & 1, &sh->abort_flag, p.device_status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) continue;
        tc_fence_after();
        float *dst = a.scores + (((long long)b * p.hkv + h) * (p.gamma_max + 1) + i0) * a.score_stride + lp;
        int best = INT_MIN, k = 0;
        for (int c0 = 0; c0 < cols; c0 += 32) {
            uint32_t r[32];
            tc_ld32(tmem + ((uint32_t)(warp * 32) << 16) + c0, r);
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                best = max(best, (int)r[c]);
                if (++k == G) {
                    // past the last column: nothing more to store (columns beyond it are padding)
                    if (c0 + c < cols && lp < sr.n_pages) *dst = __fmul_rn((float)best, scale) + 0.f;     // -0 becomes 0
                    dst += a.score_stride;
                    best = INT_MIN;
                    k = 0;
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
    }
}

// ---------------------------------------------------------------------------- choice and union
constexpr int PK_WARPS = 16;

// WPR: warps per row (PK_WARPS / WPR rows at a time); KPT: scores a thread holds.  More pages than WPR * 32 * KPT are
// read again in every round.
template <int WPR, int KPT>
__global__ void __launch_bounds__(PK_WARPS * 32)
page_pick_kernel(const __grid_constant__ PageSelectLaunch a)
{
    constexpr int TEAM = WPR * 32, TEAMS = PK_WARPS / WPR;
    pdl_enter();
    const sv_page_select_params &p = a.p;
    extern __shared__ uint32_t pk_bits[];
    __shared__ int s_count[2][PK_WARPS];
    const int h = blockIdx.x % p.hkv, b = blockIdx.x / p.hkv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp / WPR, tw = warp % WPR, t = tw * 32 + lane;
    const SeqRows sr = seq_rows(p, b, h == 0 && threadIdx.x == 0);
    const long long pair = blockIdx.x;
    uint32_t *bits = a.bits != nullptr ? a.bits + pair * (p.gamma_max + 1) * a.bit_words : pk_bits;
    int parity = 0;
    // sum over the threads of a team
    auto team_sum = [&](int x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (WPR == 1) return x;
        if (lane == 0) s_count[parity][warp] = x;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TEAM) : "memory");
        x = 0;
#pragma unroll
        for (int w = 0; w < WPR; ++w) x += s_count[parity][team * WPR + w];
        parity ^= 1;                           // the next sum writes elsewhere, so one barrier a sum is enough
        return x;
    };
    for (int i = team; i < sr.R; i += TEAMS) {
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
        // candidates: all but the fixed pages; their keys order as the scores do, and 0 stands for no candidate
        const int c_lo = p.n_first, c_hi = n_seen - p.n_last, want = p.n_select - p.n_first - p.n_last;
        const float *src = a.scores + (pair * (p.gamma_max + 1) + i) * a.score_stride;
        auto key_at = [&](int page) -> uint32_t {
            if (page < c_lo || page >= c_hi) return 0u;
            const uint32_t x = __float_as_uint(src[page]);
            return (x & 0x80000000u) ? ~x : x | 0x80000000u;
        };
        uint32_t key[KPT];
        const int rounds = (n_seen + TEAM - 1) / TEAM;
#pragma unroll
        for (int j = 0; j < KPT; ++j) key[j] = j < rounds ? key_at(j * TEAM + t) : 0u;
        // f(key, page) summed over the team's pages
        auto count = [&](auto &&f) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < KPT; ++j) {
                if (j >= rounds) break;
                n += f(key[j], j * TEAM + t) ? 1 : 0;
            }
            for (int j = KPT; j < rounds; ++j) n += f(key_at(j * TEAM + t), j * TEAM + t) ? 1 : 0;
            return team_sum(n);
        };
        // the want-th largest key: its bits from the top (all candidates have keys above 0)
        uint32_t cut = 0;
        int above = 0;                         // keys >= cut, once that is known to be at least want
        bool exact = false;
        if (want > 0) {
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t cand = cut | (1u << bit);
                const int n = count([&](uint32_t k, int) { return k >= cand; });
                if (n >= want) {
                    cut = cand;
                    above = n;
                    if (n == want) { exact = true; break; }
                }
            }
        } else {
            cut = 0xffffffffu;
            exact = true;
        }
        // more candidates at the cut than places: the lowest pages among them
        int until = 0x7fffffff;
        if (!exact && above != want) {
            const int greater = count([&](uint32_t k, int) { return k > cut; });
            int lo = 0, hi = c_hi;             // smallest page with enough candidates up to it
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                const int n = count([&](uint32_t k, int page) { return k == cut && page <= mid; });
                if (greater + n >= want) hi = mid; else lo = mid + 1;
            }
            until = lo;
        }
        auto store_word = [&](int j, uint32_t k) {
            const int page = j * TEAM + t;
            const bool fixed = page < c_lo || (page >= c_hi && page < n_seen);
            const bool take = fixed || (want > 0 && (k > cut || (k == cut && page <= until)));
            const uint32_t word = __ballot_sync(0xffffffffu, take);
            const int w = j * WPR + tw;
            if (lane == 0 && w < n_words) row[w] = word;
        };
        const int all_rounds = (n_words + WPR - 1) / WPR;          // the pages behind the row's last one too
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
            if (j >= all_rounds) break;
            store_word(j, key[j]);
        }
        for (int j = KPT; j < all_rounds; ++j) store_word(j, j < rounds ? key_at(j * TEAM + t) : 0u);
    }
    __syncthreads();
    // the union of the rows, in page order: a warp per word, lane = page
    __shared__ int s_word[PK_WARPS];
    int base = 0;
    const int n_words = sr.R > 0 ? (sr.n_pages + 31) / 32 : 0;
    int32_t *list = p.page_list + pair * p.list_stride;
    uint64_t *masks = p.row_mask + pair * p.list_stride;
    bool short_list = false;
    for (int w0 = 0; w0 < n_words; w0 += PK_WARPS) {
        const int w = w0 + warp;
        uint64_t mask = 0;
        if (w < n_words)
            for (int i = 0; i < sr.R; ++i) mask |= (uint64_t)((bits[(long long)i * a.bit_words + w] >> lane) & 1u) << i;
        const uint32_t any = __ballot_sync(0xffffffffu, mask != 0);
        if (lane == 0) s_word[warp] = __popc(any);
        __syncthreads();
        int before = base, total = 0;
#pragma unroll
        for (int k = 0; k < PK_WARPS; ++k) {
            const int n = s_word[k];
            if (k < warp) before += n;
            total += n;
        }
        const int at = before + __popc(any & ((1u << lane) - 1));
        if (mask != 0) {
            if (at < p.list_stride) {
                list[at] = w * 32 + lane;
                masks[at] = mask;
            } else {
                short_list = true;
            }
        }
        base += total;
        __syncthreads();
    }
    if (short_list) set_status(p.device_status, SV_DEV_BAD_LEN);
    if (threadIdx.x == 0) p.n_list[pair] = (int)min((long long)base, (long long)p.list_stride);
}

// ---------------------------------------------------------------------------- host side
constexpr size_t PK_SMEM_BITS = 96 * 1024;

static int select_max_pages(int max_seq_len) { return (int)(((long long)max_seq_len + 15) / 16); }
static int select_score_stride(int max_seq_len) { return (select_max_pages(max_seq_len) + 31) / 32 * 32; }
static size_t select_score_bytes(int batch, int gamma_max, int hkv, int max_seq_len)
{
    return (size_t)batch * hkv * (gamma_max + 1) * select_score_stride(max_seq_len) * sizeof(float);
}
static size_t select_row_bits(int gamma_max, int max_seq_len)
{
    return (size_t)(gamma_max + 1) * ((select_max_pages(max_seq_len) + 31) / 32) * sizeof(uint32_t);
}

template <int WPR, int KPT>
static sv_status launch_pick(const PageSelectLaunch &a, size_t smem, cudaStream_t s)
{
    if (smem > 48 * 1024 &&
        cudaFuncSetAttribute(page_pick_kernel<WPR, KPT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PK_SMEM_BITS) != cudaSuccess)
        return SV_ECUDA;
    return launch_kernel(true, page_pick_kernel<WPR, KPT>, (unsigned)(a.p.batch * a.p.hkv), PK_WARPS * 32, smem, s, a);
}

template <int D>
static sv_status launch_score(const PageSelectLaunch &a, dim3 grid, cudaStream_t s)
{
    const size_t smem = 2 * (size_t)PS_PAGES * 2 * D + (size_t)((a.pos_per_chunk * a.group + 15) & ~15) * 2 * D + sizeof(ScoreShared);
    if (cudaFuncSetAttribute(page_score_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)(2 * PS_PAGES * 2 * D + PS_MAX_COLS * 2 * D + sizeof(ScoreShared))) != cudaSuccess)
        return SV_ECUDA;
    return launch_kernel(true, page_score_kernel<D>, grid, 128, smem, s, a);
}

}  // namespace sv

extern "C" size_t spec_page_select_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hkv, int32_t max_seq_len)
{
    using namespace sv;
    if (batch <= 0 || gamma_max < 0 || gamma_max > 63 || hkv <= 0 || max_seq_len <= 0) return 0;
    const size_t row_bits = select_row_bits(gamma_max, max_seq_len);
    return select_score_bytes(batch, gamma_max, hkv, max_seq_len) + (row_bits > PK_SMEM_BITS ? row_bits * batch * hkv : 0) + 256;
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
    a.n_chunks = (R + a.pos_per_chunk - 1) / a.pos_per_chunk;
    a.max_pages = (int)max_pages;
    a.score_stride = select_score_stride(p->max_seq_len);
    a.bit_words = (int)((max_pages + 31) / 32);
    a.scores = static_cast<float *>(workspace);
    const size_t row_bits = select_row_bits(p->gamma_max, p->max_seq_len);
    const bool in_smem = row_bits <= PK_SMEM_BITS;
    a.bits = in_smem ? nullptr
                     : reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(workspace) +
                                                    select_score_bytes(p->batch, p->gamma_max, p->hkv, p->max_seq_len));
    const long long pairs = (long long)p->batch * p->hkv;
    if (pairs > 0x7fffffffLL || (long long)p->batch * a.n_chunks > 65535 || p->hkv > 65535) return SV_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    // Tiles per block: a block spends about as long on its queries as on a tile, so up to four tiles share them where there
    // are enough blocks to fill the GPU a few times over.
    const long long tiles = (max_pages + PS_PAGES - 1) / PS_PAGES;
    a.tiles_per_block = 1;
    while (a.tiles_per_block < 4 && pairs * a.n_chunks * tiles / (2 * a.tiles_per_block) >= 4LL * sm_count()) a.tiles_per_block *= 2;
    const dim3 grid((unsigned)((tiles + a.tiles_per_block - 1) / a.tiles_per_block), (unsigned)p->hkv, (unsigned)(p->batch * a.n_chunks));
    if (max_pages > p->n_select) {             // otherwise no sequence has more pages than a row takes
        const sv_status st = p->head_dim == 128 ? launch_score<128>(a, grid, s) : launch_score<64>(a, grid, s);
        if (st != SV_OK) return st;
    }
    // Warps per row: enough to hold a row's scores in registers, and all of a block's where it has few rows.
    int need = 1;
    while (need < PK_WARPS && (long long)need * 32 * 32 < max_pages) need *= 2;
    while (need < PK_WARPS && need * 2 * R <= PK_WARPS) need *= 2;
    const size_t smem = in_smem ? row_bits : 0;
    switch (need) {
        case 1: return launch_pick<1, 32>(a, smem, s);
        case 2: return launch_pick<2, 32>(a, smem, s);
        case 4: return launch_pick<4, 32>(a, smem, s);
        case 8: return launch_pick<8, 32>(a, smem, s);
        default: return launch_pick<16, 32>(a, smem, s);
    }
}
