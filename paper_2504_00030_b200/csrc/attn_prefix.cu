// The verify attention of a batch whose sequences share long prefixes (spec_verify_attn_prefix).
//
// softmax over the keys of a row splits into parts: with m, l and o of the shared prefix (computed for all rows of a group
// at once) and of the sequence's own keys, the row is (2^(m1-m) o1 + 2^(m2-m) o2) / (2^(m1-m) l1 + 2^(m2-m) l2).  Launches:
//   plan      the members of each group and where their rows are;
//   groups    the prefixes: 256 rows of any members meet each key tile (tensor-core bound; a rows * heads * head_dim fp32
//             partial per group is written and read once, 520 bytes a row and head);
//   sequences the rest of every sequence: its rows begin with the group's partial O, maximum and sum in place of zeros;
//   combine   behind either of the two: pairs that were split over blocks.
// Measured (B200): 64 tokens behind one prompt of 8192 77 us (26 us of bytes; five launches; 268 by the verify attention), 128
// blocks of up to 17 rows of 64 heads behind three prefixes of up to 12000 tokens 643 us at 1965 MHz, 446 of them the groups (331
// us for all products at the tensor core's full rate), and 770 after a second of such calls (1690 MHz): there the verify
// attention, which reads the prefixes for every sequence, takes 651 and 704.
#include "attn_seg.cuh"

namespace sv {

constexpr int PLAN_THREADS = 256;
constexpr int MAX_PREFIX_BATCH = 8192;

// Block g: group g.  Two passes over the batch: how many members and rows, then where each member's rows go.
__global__ void __launch_bounds__(PLAN_THREADS)
prefix_plan_kernel(const __grid_constant__ SegLaunch a, const int32_t *prefix_len, int n_groups)
{
    pdl_enter();
    const sv_attn_params &p = a.p;
    const PrefixPlan &pl = a.plan;
    const int g = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ int s_sum[3][PLAN_THREADS / 32], s_rep;
    const int len = prefix_len[g];
    int pages = len / 16;
    if (len < 0 || pages > p.block_table_stride) {
        if (tid == 0) set_status(p.device_status, SV_DEV_BAD_LEN);
        pages = 0;
    }
    if (tid == 0) s_rep = 0x7fffffff;
    // rows of sequence b (0: skipped), its group
    auto rows_of = [&](int b, int &gid) {
        gid = a.seq_group[b];
        if (gid < -1 || gid >= n_groups) {
            if (g == 0) set_status(p.device_status, SV_DEV_BAD_LEN);
            gid = -1;
        }
        const int gam = min(max(p.gamma[b], 0), p.gamma_max), L = p.seq_len[b];
        if (L < gam + 1 || L > p.max_seq_len || (L + 15) / 16 > p.block_table_stride) return 0;
        return gam + 1;
    };
    int before = 0, rows = 0, members = 0, rep = 0x7fffffff;
    for (int b = tid; b < p.batch; b += PLAN_THREADS) {
        int gid;
        const int R = rows_of(b, gid);
        if (gid >= 0 && gid < g) before += R;
        if (gid == g && R > 0 && p.seq_len[b] - R >= 16 * pages) {
            rows += R;
            ++members;
            rep = min(rep, b);
        }
        if (g == 0 && gid < 0) pl.seq_pages[b] = 0;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    rows = __reduce_add_sync(0xffffffffu, rows);
    members = __reduce_add_sync(0xffffffffu, members);
    rep = __reduce_min_sync(0xffffffffu, rep);
    __syncthreads();
    if (lane == 0) {
        s_sum[0][warp] = before; s_sum[1][warp] = rows; s_sum[2][warp] = members;
        atomicMin(&s_rep, rep);
    }
    __syncthreads();
    before = rows = members = 0;
    for (int w = 0; w < PLAN_THREADS / 32; ++w) { before += s_sum[0][w]; rows += s_sum[1][w]; members += s_sum[2][w]; }
    if (members < 2) pages = 0;                        // nobody to share with
    if (tid == 0) {
        pl.grp_pages[g] = pages;
        pl.grp_rep[g] = members > 0 ? s_rep : 0;
        pl.grp_n[g] = pages > 0 ? rows : 0;
        pl.grp_base[g] = before;
    }
    int at0 = 0;
    for (int base = 0; base < p.batch; base += PLAN_THREADS) {
        const int b = base + tid;
        int R = 0, gid = -1;
        if (b < p.batch) R = rows_of(b, gid);
        const bool mine = b < p.batch && gid == g;
        const bool member = mine && R > 0 && pages > 0 && p.seq_len[b] - R >= 16 * pages;
        const int n = member ? R : 0;
        int v = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += t;
        }
        __syncthreads();
        if (lane == 31) s_sum[0][warp] = v;
        __syncthreads();
        int at = at0 + v - n;
        for (int w = 0; w < PLAN_THREADS / 32; ++w) {
            if (w < warp) at += s_sum[0][w];
            at0 += s_sum[0][w];
        }
        if (mine) pl.seq_pages[b] = member ? pages : 0;
        if (member)
            for (int i = 0; i < R; ++i) pl.row_list[before + at + i] = make_int2(p.cu_q[b] + i, b * (p.gamma_max + 1) + i);
    }
}

// ---------------------------------------------------------------------------- host side
enum { PX_GRP_PAGES, PX_GRP_REP, PX_GRP_N, PX_GRP_BASE, PX_ROW_LIST, PX_SEQ_PAGES, PX_PART_O, PX_PART_ML, PX_TABLES, PX_PART, PX_N };

struct PrefixLayout {
    size_t at[PX_N], bytes;
};

static PrefixLayout prefix_layout(int batch, int gamma_max, int hq, int hkv, int n_groups)
{
    const size_t w = sizeof(int32_t), positions = (size_t)batch * (gamma_max + 1);
    size_t sizes[PX_N];
    sizes[PX_GRP_PAGES] = sizes[PX_GRP_REP] = sizes[PX_GRP_N] = sizes[PX_GRP_BASE] = n_groups * w;
    sizes[PX_ROW_LIST] = positions * sizeof(int2);
    sizes[PX_SEQ_PAGES] = batch * w;
    sizes[PX_PART_O] = positions * hq * SEG_PITCH * sizeof(float);
    sizes[PX_PART_ML] = positions * hq * sizeof(float2);
    sizes[PX_TABLES] = seg_table_bytes();                                     // bounds, desc and parts of split pairs: those of the
    const size_t parts = seg_part_bytes(seg_nl(hq / hkv * (gamma_max + 1)));  // groups are done with before the sequences begin
    sizes[PX_PART] = parts > seg_part_bytes(2) ? parts : seg_part_bytes(2);
    PrefixLayout l;
    size_t at = 0;
    for (int i = 0; i < PX_N; ++i) {
        l.at[i] = at;
        at += seg_round(sizes[i]);
    }
    l.bytes = at;
    return l;
}

template <int D>
static sv_status launch_groups(SegLaunch &a, cudaStream_t s)
{
    const sv_status st = launch_seg<SEG_GROUP, 2, D>(a, seg_grid(2), s);
    return st != SV_OK ? st : launch_seg_combine<SEG_GROUP, 2, D>(a, seg_grid(2), s);
}

template <int NL>
static sv_status launch_sequences(SegLaunch &a, cudaStream_t s)
{
    const int grid = seg_grid(NL);
    sv_status st = a.p.head_dim == 128 ? launch_seg<SEG_SEQ, NL, 128>(a, grid, s) : launch_seg<SEG_SEQ, NL, 64>(a, grid, s);
    if (st != SV_OK) return st;
    return a.p.head_dim == 128 ? launch_seg_combine<SEG_SEQ, NL, 128>(a, grid, s) : launch_seg_combine<SEG_SEQ, NL, 64>(a, grid, s);
}

}  // namespace sv

extern "C" size_t spec_verify_attn_prefix_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hq, int32_t hkv, int32_t head_dim,
                                                          int32_t n_groups)
{
    using namespace sv;
    if (batch <= 0 || batch > MAX_PREFIX_BATCH || gamma_max < 0 || gamma_max > 4095 || hq <= 0 || hkv <= 0 || hq % hkv != 0 ||
        hq / hkv > 128 || (head_dim != 64 && head_dim != 128) || n_groups <= 0 || n_groups > batch)
        return 0;
    return SEG_WS_SLACK + prefix_layout(batch, gamma_max, hq, hkv, n_groups).bytes;
}

extern "C" sv_status spec_verify_attn_prefix(const sv_attn_prefix_params *p, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace sv;
    if (p == nullptr) return SV_EINVAL;
    const sv_attn_params &at = p->attn;
    sv_status st = check_attn_params(&at);
    if (st != SV_OK) return st;
    if (p->group == nullptr || p->prefix_len == nullptr || p->n_groups <= 0 || p->n_groups > at.batch) return SV_EINVAL;
    if (at.batch > MAX_PREFIX_BATCH || at.gamma_max > 4095 || at.hq / at.hkv > 128 || at.max_seq_len > SEG_MAX_LEN || !at.pool->has_maps)
        return SV_EUNSUPPORTED;
    // pairs of the sequences; the groups, whose pairs have two row tiles, have no more
    if (!seg_tiles_fit((long long)at.batch * at.hkv * seg_chunks(at.hq / at.hkv, at.gamma_max), at.max_seq_len / 16 + 1)) return SV_EUNSUPPORTED;
    if (workspace == nullptr ||
        workspace_bytes < spec_verify_attn_prefix_workspace_bytes(at.batch, at.gamma_max, at.hq, at.hkv, at.head_dim, p->n_groups))
        return SV_EWORKSPACE;
    if (!aligned16(workspace)) return SV_EALIGN;
    if (seg_grid(1) > SEG_MAX_GRID) return SV_EUNSUPPORTED;
    const PrefixLayout l = prefix_layout(at.batch, at.gamma_max, at.hq, at.hkv, p->n_groups);
    uint8_t *w = seg_workspace(workspace);
    auto ints = [&](int i) { return reinterpret_cast<int32_t *>(w + l.at[i]); };
    SegLaunch a = {};
    a.p = at;
    a.n_pool_pages = at.pool->n_pages;
    a.group = at.hq / at.hkv;
    a.ppl = 128 / a.group;
    a.seq_group = p->group;
    PrefixPlan &pl = a.plan;
    pl.grp_pages = ints(PX_GRP_PAGES);
    pl.grp_rep = ints(PX_GRP_REP);
    pl.grp_n = ints(PX_GRP_N);
    pl.grp_base = ints(PX_GRP_BASE);
    pl.row_list = reinterpret_cast<int2 *>(w + l.at[PX_ROW_LIST]);
    pl.seq_pages = ints(PX_SEQ_PAGES);
    pl.part_o = reinterpret_cast<float *>(w + l.at[PX_PART_O]);
    pl.part_ml = reinterpret_cast<float2 *>(w + l.at[PX_PART_ML]);
    a.bounds = ints(PX_TABLES);
    a.desc = reinterpret_cast<int32_t *>(w + l.at[PX_TABLES] + seg_round((SEG_MAX_GRID + 1) * sizeof(int32_t)));
    a.part = reinterpret_cast<float *>(w + l.at[PX_PART]);
    cudaStream_t s = (cudaStream_t)stream;
    st = launch_kernel(true, prefix_plan_kernel, p->n_groups, PLAN_THREADS, 0, s, a, p->prefix_len, p->n_groups);
    if (st != SV_OK) return st;
    a.n_owners = p->n_groups;
    st = at.head_dim == 128 ? launch_groups<128>(a, s) : launch_groups<64>(a, s);
    if (st != SV_OK) return st;
    a.n_owners = at.batch;
    return seg_nl(a.group * (at.gamma_max + 1)) == 1 ? launch_sequences<1>(a, s) : launch_sequences<2>(a, s);
}
