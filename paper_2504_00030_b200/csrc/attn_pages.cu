// Attention over the pages that a list names for every sequence and kv head, with a mask of the rows that read each
// (spec_verify_attn_pages): the kernel of attn_seg.cuh with lists as its owners.
#include "attn_seg.cuh"

namespace sv {

template <int NL>
static sv_status launch_pages(SegLaunch &a, int grid, cudaStream_t s)
{
    sv_status st = a.p.head_dim == 128 ? launch_seg<SEG_LIST, NL, 128>(a, grid, s) : launch_seg<SEG_LIST, NL, 64>(a, grid, s);
    if (st != SV_OK) return st;
    return a.p.head_dim == 128 ? launch_seg_combine<SEG_LIST, NL, 128>(a, grid, s) : launch_seg_combine<SEG_LIST, NL, 64>(a, grid, s);
}

}  // namespace sv

extern "C" size_t spec_verify_attn_pages_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hq, int32_t hkv, int32_t head_dim)
{
    using namespace sv;
    if (batch <= 0 || gamma_max < 0 || gamma_max > 63 || hq <= 0 || hkv <= 0 || hq % hkv != 0 || hq / hkv > 128 ||
        (head_dim != 64 && head_dim != 128))
        return 0;
    return SEG_WS_SLACK + seg_table_bytes() + seg_part_bytes(seg_nl(hq / hkv * (gamma_max + 1)));
}

extern "C" sv_status spec_verify_attn_pages(const sv_attn_pages_params *p, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace sv;
    if (p == nullptr) return SV_EINVAL;
    const sv_attn_params &at = p->attn;
    const sv_status st = check_attn_params(&at);
    if (st != SV_OK) return st;
    if (p->page_list == nullptr || p->row_mask == nullptr || p->n_list == nullptr || p->list_stride <= 0) return SV_EINVAL;
    if (at.gamma_max > 63 || at.hq / at.hkv > 128 || at.max_seq_len > SEG_MAX_LEN || !at.pool->has_maps) return SV_EUNSUPPORTED;
    if ((long long)at.batch * at.hkv > (1 << 24) || p->list_stride > (1 << 26)) return SV_EUNSUPPORTED;
    if (!seg_tiles_fit((long long)at.batch * at.hkv * seg_chunks(at.hq / at.hkv, at.gamma_max), p->list_stride)) return SV_EUNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(p->row_mask) & 7u) != 0) return SV_EALIGN;
    if (workspace == nullptr ||
        workspace_bytes < spec_verify_attn_pages_workspace_bytes(at.batch, at.gamma_max, at.hq, at.hkv, at.head_dim))
        return SV_EWORKSPACE;
    if (!aligned16(workspace)) return SV_EALIGN;
    SegLaunch a = {};
    a.p = at;
    a.n_pool_pages = at.pool->n_pages;
    a.group = at.hq / at.hkv;
    a.ppl = 128 / a.group;
    a.n_owners = at.batch * at.hkv;
    a.page_list = p->page_list;
    a.row_mask = p->row_mask;
    a.n_list = p->n_list;
    a.list_stride = p->list_stride;
    uint8_t *w = seg_workspace(workspace);
    a.bounds = reinterpret_cast<int32_t *>(w);
    a.desc = reinterpret_cast<int32_t *>(w + seg_round((SEG_MAX_GRID + 1) * sizeof(int32_t)));
    a.part = reinterpret_cast<float *>(w + seg_table_bytes());
    const int nl = seg_nl(a.group * (at.gamma_max + 1)), grid = seg_grid(nl);
    if (grid > SEG_MAX_GRID) return SV_EUNSUPPORTED;
    return nl == 1 ? launch_pages<1>(a, grid, (cudaStream_t)stream) : launch_pages<2>(a, grid, (cudaStream_t)stream);
}
