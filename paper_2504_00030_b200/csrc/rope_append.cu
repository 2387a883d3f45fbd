// Per-head norm of queries and keys, position rotation and cache append in one pass (KV caching, paper Section 5).
//
// y = x * w * rsqrt(mean(x^2) + eps), then z = y rotated by the row's angles; queries to the attention's input, keys and
// values to the row's slot of the paged cache.  Every element is read once and written once, so HBM bounds it: the
// norm's sum lives in the registers of the lanes that hold the head.
//
// A lane holds two 16-byte chunks (16 dims) of a head and D / 16 lanes hold the head.  Which two is chosen so that
// a rotated pair never leaves its lane: chunks j and j + rot/16 where the pairs are (f, f + rot/2), chunks 2j and 2j + 1
// where they are (2f, 2f + 1).  Either way the lane's eight pairs have the frequencies 8j .. 8j + 7, and only the norm's
// sum crosses lanes (two to four shuffles).
#include "attn_common.cuh"
#include "common.cuh"

namespace sv {

constexpr int RA_THREADS = 256;
constexpr int RA_PAGE = 16;
constexpr int RA_MAX_FREQ = 64;            // rot_dim <= head_dim <= 128

struct RopeAppendLaunch {
    sv_rope_append_params p;
    uint4 *k_pool;
    uint4 *v_pool;
    long long n_slots;
    long long stride_page, stride_head, stride_slot;   // in 16-byte chunks
    int hkv, lanes;                        // lanes that hold a head (head_dim / 16)
};

__device__ __forceinline__ uint4 ld_chunk(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void unpack8(const uint4 &v, float *x)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float *x)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);      // the one rounding
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// eight norm weights of a chunk
__device__ __forceinline__ void load_weights(const void *w, int f32, int chunk, float *x)
{
    if (f32) {
        const float4 *s = static_cast<const float4 *>(w) + 2 * chunk;
        const float4 a = __ldg(s), b = __ldg(s + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        unpack8(__ldg(static_cast<const uint4 *>(w) + chunk), x);
    }
}

// GL: lanes given to a head (a power of two >= head_dim / 16)
template <int GL>
__global__ void __launch_bounds__(RA_THREADS)
rope_append_kernel(const __grid_constant__ RopeAppendLaunch a)
{
    pdl_enter();
    __shared__ float2 turn[RA_MAX_FREQ];               // (cos, sin) of the row's angles
    const sv_rope_append_params &p = a.p;
    const long long row = blockIdx.x;
    const long long slot = __ldg(p.slot_map + row);
    if (slot < 0) return;
    if (slot >= a.n_slots) {
        if (threadIdx.x == 0) set_status(p.device_status, SV_DEV_BAD_PAGE);
        return;
    }
    const int tid = threadIdx.x, j = tid % GL;
    const int nf = p.rot_dim / 2, pair_lanes = p.rot_dim / 16;
    const bool live = j < a.lanes, turned = j < pair_lanes;
    int c0 = 2 * j, c1 = 2 * j + 1;                    // this lane's chunks
    if (turned && !p.interleaved) {
        c0 = j;
        c1 = j + pair_lanes;
    }
    for (int f = tid; f < nf; f += RA_THREADS) {
        const int axis = p.freq_axis != nullptr ? min((int)__ldg(p.freq_axis + f), p.n_axes - 1) : 0;
        const int pos = __ldg(p.positions + (long long)axis * p.n_rows + row);
        // whole turns drop out in float64; what is left is below half a turn
        double t = (double)pos * (__ldg(p.inv_freq + f) * 0.15915494309189535);
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        turn[f] = make_float2(c * p.rope_scale, s * p.rope_scale);
    }
    __syncthreads();
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 v = turned ? turn[8 * j + i] : make_float2(1.f, 0.f);
        cs[i] = v.x;
        sn[i] = v.y;
    }
    const long long cache = (slot / RA_PAGE) * a.stride_page + (slot % RA_PAGE) * a.stride_slot;
    const int heads = p.hq + 2 * a.hkv;
    const int chunks = 2 * a.lanes;
    // all lanes of a warp make the same number of rounds (the norm's shuffles)
    for (int h0 = 0; h0 < heads; h0 += RA_THREADS / GL) {
        const int h = h0 + tid / GL;
        const uint4 *src = nullptr;
        uint4 *dst = nullptr;
        const void *weight = nullptr;
        bool rotate = turned;
        if (live && h < heads) {
            if (h < p.hq) {
                src = static_cast<const uint4 *>(p.q) + row * (p.q_stride / 8) + (long long)h * chunks;
                dst = static_cast<uint4 *>(p.q_out) + (row * p.hq + h) * chunks;
                weight = p.q_weight;
            } else if (h < p.hq + a.hkv) {
                src = static_cast<const uint4 *>(p.k_new) + row * (p.k_stride / 8) + (long long)(h - p.hq) * chunks;
                dst = a.k_pool + cache + (h - p.hq) * a.stride_head;
                weight = p.k_weight;
            } else {
                src = static_cast<const uint4 *>(p.v_new) + row * (p.v_stride / 8) + (long long)(h - p.hq - a.hkv) * chunks;
                dst = a.v_pool + cache + (h - p.hq - a.hkv) * a.stride_head;
                rotate = false;
            }
        }
        uint4 v0 = make_uint4(0, 0, 0, 0), v1 = v0;
        if (src != nullptr) {
            v0 = ld_chunk(src + c0);
            v1 = ld_chunk(src + c1);
        }
        float x[16];
        unpack8(v0, x);
        unpack8(v1, x + 8);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
#pragma unroll
        for (int m = GL / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        if (src == nullptr) continue;
        if (weight != nullptr) {
            const float r = rsqrtf(ss / (float)(16 * a.lanes) + p.eps);
            float w[16];
            load_weights(weight, p.weights_f32, c0, w);
            load_weights(weight, p.weights_f32, c1, w + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
        }
        if (rotate) {
            if (p.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = x[2 * i], v = x[2 * i + 1];
                    x[2 * i] = u * cs[i] - v * sn[i];
                    x[2 * i + 1] = v * cs[i] + u * sn[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = x[i], v = x[8 + i];
                    x[i] = u * cs[i] - v * sn[i];
                    x[8 + i] = v * cs[i] + u * sn[i];
                }
            }
        }
        if (weight == nullptr && !rotate) {            // values, and what is neither normalised nor turned: the same bits
            dst[c0] = v0;
            dst[c1] = v1;
        } else {
            dst[c0] = pack8(x);
            dst[c1] = pack8(x + 8);
        }
    }
}

// [a, a + na) and [b, b + nb) share a byte
static bool overlap(const void *a, long long na, const void *b, long long nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

}  // namespace sv

extern "C" sv_status spec_rope_append(const sv_rope_append_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr || p->pool == nullptr || p->n_rows < 0) return SV_EINVAL;
    const sv_kv_pool &pool = *p->pool;
    if (p->hq <= 0 || p->n_axes <= 0 || p->rot_dim < 0 || p->rot_dim > pool.head_dim || !(p->eps >= 0.f)) return SV_EINVAL;
    if (pool.head_dim % 16 != 0 || p->rot_dim % 16 != 0) return SV_EUNSUPPORTED;
    if (p->n_rows > 0x7fffffffLL) return SV_EUNSUPPORTED;
    const long long q_row = (long long)p->hq * pool.head_dim, kv_row = (long long)pool.hkv * pool.head_dim;
    if (p->q_stride < q_row || p->k_stride < kv_row || p->v_stride < kv_row) return SV_EINVAL;
    if (p->n_rows == 0) return SV_OK;
    if (p->q == nullptr || p->k_new == nullptr || p->v_new == nullptr || p->q_out == nullptr || p->slot_map == nullptr ||
        p->positions == nullptr || (p->rot_dim > 0 && p->inv_freq == nullptr))
        return SV_EINVAL;
    if (!aligned16(p->q) || !aligned16(p->k_new) || !aligned16(p->v_new) || !aligned16(p->q_out) || !aligned16(p->q_weight) ||
        !aligned16(p->k_weight) || p->q_stride % 8 != 0 || p->k_stride % 8 != 0 || p->v_stride % 8 != 0)
        return SV_EALIGN;
    const long long out_bytes = p->n_rows * q_row * 2;
    const bool in_place = p->q_out == p->q && p->q_stride == q_row;
    // a view's last row ends with its heads, not with the stride
    auto bytes = [&](long long stride, long long width) { return ((p->n_rows - 1) * stride + width) * 2; };
    if ((!in_place && overlap(p->q_out, out_bytes, p->q, bytes(p->q_stride, q_row))) ||
        overlap(p->q_out, out_bytes, p->k_new, bytes(p->k_stride, kv_row)) ||
        overlap(p->q_out, out_bytes, p->v_new, bytes(p->v_stride, kv_row)))
        return SV_EINVAL;
    RopeAppendLaunch a;
    a.p = *p;
    // the pool was registered through const pointers for the readers; this call is its writer
    a.k_pool = static_cast<uint4 *>(const_cast<void *>(pool.k));
    a.v_pool = static_cast<uint4 *>(const_cast<void *>(pool.v));
    a.n_slots = (long long)pool.n_pages * RA_PAGE;
    a.stride_page = pool.strides[0] / 8;
    a.stride_head = pool.strides[1] / 8;
    a.stride_slot = pool.strides[2] / 8;
    a.hkv = pool.hkv;
    a.lanes = pool.head_dim / 16;
    const dim3 grid((unsigned)p->n_rows);
    cudaStream_t s = (cudaStream_t)stream;
    if (a.lanes <= 4) return launch_kernel(true, rope_append_kernel<4>, grid, RA_THREADS, 0, s, a);
    return launch_kernel(true, rope_append_kernel<8>, grid, RA_THREADS, 0, s, a);
}
