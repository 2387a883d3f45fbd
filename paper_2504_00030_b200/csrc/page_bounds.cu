// Bounds of every page's keys, kept beside the paged cache (KV caching, paper Section 5): per page and kv head the
// elementwise maximum and minimum of its keys in 8 bits with one scale, for spec_page_select.
//
// One warp per (page, kv head): its 16 keys are 4 KB (head_dim 128), eight 16-byte loads a lane, all in flight at once;
// a lane keeps the maxima and minima of its eight dims over its slots as packed bf16 (exact), the lanes that share
// dims combine by shuffle.  Bound by HBM on prompts (2 bytes read per key element, 1/8 of a byte written), by launch
// and two dependent loads (table entry, keys) on draft blocks.  Measured: 16 prompts of up to 8192 tokens 45 us (40.5 at a
// copy's rate), a block of one sequence 2.4 us.
#include "attn_common.cuh"
#include "common.cuh"
#include "whole8.cuh"

namespace sv {

constexpr int PB_WARPS = 8;

struct PageBoundsLaunch {
    sv_page_bounds_params p;
    const uint4 *k;
    long long n_pages;
    long long stride_page, stride_head, stride_slot;   // in 16-byte chunks
    int hkv;
    int pages_max;                                     // pages that max_new tokens may touch
    long long n_items;                                 // batch * pages_max * hkv
};

__device__ __forceinline__ __nv_bfloat162 as_bf2(uint32_t x) { return *reinterpret_cast<__nv_bfloat162 *>(&x); }

// D: head_dim.  D / 8 lanes hold a slot's dims, 32 / (D / 8) slots per load.
template <int D>
__global__ void __launch_bounds__(PB_WARPS * 32)
page_bounds_kernel(const __grid_constant__ PageBoundsLaunch a)
{
    constexpr int LANES = D / 8, SLOTS = 32 / LANES, LOADS = 16 / SLOTS;
    pdl_enter();
    const sv_page_bounds_params &p = a.p;
    const long long item = (long long)blockIdx.x * PB_WARPS + (threadIdx.x >> 5);
    if (item >= a.n_items) return;
    const int lane = threadIdx.x & 31;
    const long long bj = item / a.hkv;                 // heads innermost: a page's heads are neighbours in memory
    const int h = (int)(item - bj * a.hkv);
    const int b = (int)(bj / a.pages_max), j = (int)(bj - (long long)b * a.pages_max);
    const bool report = lane == 0 && h == 0 && j == 0;
    const int L = p.seq_len[b];
    if (L == 0) return;
    int first;
    if (p.gamma != nullptr) {
        int g = p.gamma[b];
        if (g < 0 || g >= p.max_new) {
            if (report) set_status(p.device_status, SV_DEV_BAD_GAMMA);
            g = min(max(g, 0), p.max_new - 1);
        }
        first = L - (g + 1);
    } else {
        first = p.first[b];
    }
    if (L < 0 || (long long)(L - 1) / 16 >= p.block_table_stride || first < 0 || (long long)L - first > p.max_new) {
        if (report) set_status(p.device_status, SV_DEV_BAD_LEN);
        return;
    }
    if (first >= L) return;                            // nothing new
    const int lp = first / 16 + j;
    if (lp * 16LL >= L) return;
    const int page = p.block_table[(long long)b * p.block_table_stride + lp];
    if (page < 0 || page >= a.n_pages) {
        if (lane == 0 && h == 0) set_status(p.device_status, SV_DEV_BAD_PAGE);
        return;
    }
    const int n_valid = min(16, L - lp * 16);
    const int dim8 = lane % LANES, slot0 = lane / LANES;
    const uint4 *src = a.k + page * a.stride_page + h * a.stride_head + dim8;
    uint4 v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int slot = min(slot0 + i * SLOTS, n_valid - 1);      // an unused slot: the last used one once more
        v[i] = __ldg(src + slot * a.stride_slot);
    }
    uint32_t hi[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, lo[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
    auto fold = [&](int c, uint32_t x, uint32_t y) {
        // a NaN stays: the page's scale becomes one, so that the choice takes the page for the highest
        const __nv_bfloat162 m = __hmax2_nan(as_bf2(hi[c]), as_bf2(x)), n = __hmin2_nan(as_bf2(lo[c]), as_bf2(y));
        hi[c] = *reinterpret_cast<const uint32_t *>(&m);
        lo[c] = *reinterpret_cast<const uint32_t *>(&n);
    };
#pragma unroll
    for (int i = 1; i < LOADS; ++i) {
        fold(0, v[i].x, v[i].x);
        fold(1, v[i].y, v[i].y);
        fold(2, v[i].z, v[i].z);
        fold(3, v[i].w, v[i].w);
    }
#pragma unroll
    for (int d = LANES; d < 32; d <<= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t x = __shfl_xor_sync(0xffffffffu, hi[c], d), y = __shfl_xor_sync(0xffffffffu, lo[c], d);
            fold(c, x, y);
        }
    // the first LANES lanes store the maxima, the next the minima
    const bool low = slot0 == 1;
    float x[8];
    uint32_t big = 0;                                  // largest magnitude: these order as bits, NaN above all
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float2 f = __bfloat1622float2(as_bf2(low ? lo[c] : hi[c]));
        x[2 * c] = f.x;
        x[2 * c + 1] = f.y;
        big = max(big, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
    }
#pragma unroll
    for (int d = 1; d < 2 * LANES; d <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, d));
    // every step rounds once to the nearest float32, so that the stored whole numbers are reproducible
    const float scale = __fmul_rn(__uint_as_float(big), 1.f / 127.f);
    const uint2 w = whole8x8(x, Whole8(scale));
    const long long at = (long long)page * a.hkv + h;
    if (slot0 < 2) *reinterpret_cast<uint2 *>(p.bounds + at * 2 * D + (low ? D : 0) + dim8 * 8) = w;
    if (lane == 0) p.scales[at] = scale;
}

}  // namespace sv

extern "C" sv_status spec_page_bounds_update(const sv_page_bounds_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr || p->pool == nullptr) return SV_EINVAL;
    if (p->bounds == nullptr || p->scales == nullptr || p->block_table == nullptr || p->seq_len == nullptr) return SV_EINVAL;
    if ((p->gamma == nullptr) == (p->first == nullptr)) return SV_EINVAL;
    if (p->batch <= 0 || p->block_table_stride <= 0 || p->max_new <= 0) return SV_EINVAL;
    const sv_kv_pool *pool = p->pool;
    if (pool->page_size != 16 || (pool->head_dim != 64 && pool->head_dim != 128)) return SV_EUNSUPPORTED;
    if (!aligned16(p->bounds) || (reinterpret_cast<uintptr_t>(p->scales) & 3u) != 0) return SV_EALIGN;
    PageBoundsLaunch a;
    a.p = *p;
    a.k = static_cast<const uint4 *>(pool->k);
    a.n_pages = pool->n_pages;
    a.stride_page = pool->strides[0] / 8;              // registration checked: multiples of 8 elements, dim stride 1
    a.stride_head = pool->strides[1] / 8;
    a.stride_slot = pool->strides[2] / 8;
    a.hkv = pool->hkv;
    long long pages = ((long long)p->max_new + 14) / 16 + 1;
    if (pages > p->block_table_stride) pages = p->block_table_stride;
    a.pages_max = (int)pages;
    a.n_items = (long long)p->batch * pages * pool->hkv;
    const long long blocks = (a.n_items + PB_WARPS - 1) / PB_WARPS;
    if (pages > 0x7fffffffLL || blocks > 0x7fffffffLL) return SV_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    return pool->head_dim == 128 ? launch_kernel(true, page_bounds_kernel<128>, (unsigned)blocks, PB_WARPS * 32, 0, s, a)
                                 : launch_kernel(true, page_bounds_kernel<64>, (unsigned)blocks, PB_WARPS * 32, 0, s, a);
}
