// Penalties, biases and grammar masks on logit rows in one pass (paper Section 3: target and draft sample from these rows).
//
// A block takes a slice of the vocabulary and the rows of one sequence's block.  What the counts and the bias list do to
// an element is the same for all of these rows, x * factor + add, except where a draft token falls on it: the counts and the
// list are read once, the two numbers stay in registers, and row i + 1 only updates the element that draft i names.
// HBM bounds it: the logits in and out, and 2 bytes of counts per 17 rows.
#include "common.cuh"
#include "row_stream.cuh"

namespace sv {

constexpr int LA_THREADS = 256;
constexpr int LA_UNITS = 2;                // 16-byte units of a row that a thread has
constexpr int LA_AHEAD = 2;                // rows under way
constexpr int LA_MAX_GAMMA = 64;

struct LogitsAdjustLaunch {
    sv_logits_adjust_params p;
    int slices;                            // blocks along the vocabulary
    int rows_per_block, chunks;            // rows of a block, blocks along a sequence's rows
    int in_place, vec;
    int penalties;
};

// streamed once; not the read-only path, since the call may work in place
__device__ __forceinline__ uint4 ld_once(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <bool BF16>
struct Unit {
    static constexpr int N = BF16 ? 8 : 4;                      // elements of a unit
    static constexpr int SLICE = LA_THREADS * LA_UNITS * N;     // elements of a block
};

// unit at element k of a row; past the vocabulary -inf.  `vec`: whole units are one access
template <bool BF16>
__device__ __forceinline__ void unit_load(const void *row, int k, int V, bool vec, uint4 &raw)
{
    if (vec && k + Unit<BF16>::N <= V) {
        raw = BF16 ? ld_once(static_cast<const unsigned short *>(row) + k) : ld_once(static_cast<const float *>(row) + k);
        return;
    }
    uint32_t w[4] = {0, 0, 0, 0};
    if (BF16) {
        const unsigned short *s = static_cast<const unsigned short *>(row);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < V) w[e / 2] |= (uint32_t)s[k + e] << (16 * (e & 1));
    } else {
        const uint32_t *s = static_cast<const uint32_t *>(row);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < V) w[e] = s[k + e];
    }
    raw = make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool BF16>
__device__ __forceinline__ void unit_store(void *row, int k, int V, bool vec, const uint4 &raw)
{
    if (vec && k + Unit<BF16>::N <= V) {
        if (BF16) *reinterpret_cast<uint4 *>(static_cast<unsigned short *>(row) + k) = raw;
        else *reinterpret_cast<uint4 *>(static_cast<float *>(row) + k) = raw;
        return;
    }
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if (BF16) {
        unsigned short *s = static_cast<unsigned short *>(row);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < V) s[k + e] = (unsigned short)(w[e / 2] >> (16 * (e & 1)));
    } else {
        uint32_t *s = static_cast<uint32_t *>(row);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < V) s[k + e] = w[e];
    }
}

// ADD: penalties or biases; MASK: grammar masks
template <bool BF16, bool ADD, bool MASK>
__global__ void __launch_bounds__(LA_THREADS)
logits_adjust_kernel(const __grid_constant__ LogitsAdjustLaunch a)
{
    pdl_enter();
    constexpr int N = Unit<BF16>::N, SLICE = Unit<BF16>::SLICE;
    __shared__ int bias_at[ADD ? SLICE : 1];           // entry of the bias list that names the element, plus one
    __shared__ int tokens[LA_MAX_GAMMA];
    const sv_logits_adjust_params &p = a.p;
    const int tid = threadIdx.x, V = p.vocab;
    const int slice = blockIdx.x % a.slices, seq_chunk = blockIdx.x / a.slices;
    const int b = seq_chunk / a.chunks, chunk = seq_chunk - b * a.chunks;
    if (p.active != nullptr && p.active[b] == 0) return;
    uint32_t bad = 0;
    const bool draft = p.n_drafted != nullptr;
    int g = draft ? p.n_drafted[b] : p.gamma[b];
    if (g < 0 || g > p.gamma_max) {
        bad |= SV_DEV_BAD_GAMMA;
        g = min(max(g, 0), p.gamma_max);
    }
    // rows of this block, and drafts in front of its first row
    const int rows = draft ? 1 : g + 1, i_begin = chunk * a.rows_per_block, i_end = min(rows, i_begin + a.rows_per_block);
    const int before = draft ? g : i_begin;
    long long row0 = draft ? b : p.cu_q[b];
    if (i_begin >= i_end) {
        if (bad != 0 && tid == 0) set_status(p.device_status, bad);
        return;
    }
    if (row0 < 0 || row0 + rows > p.n_rows) {
        if (tid == 0) set_status(p.device_status, bad | SV_DEV_BAD_LEN);
        return;
    }
    const int base = slice * SLICE;
    int k0[LA_UNITS];
#pragma unroll
    for (int u = 0; u < LA_UNITS; ++u) k0[u] = base + (u * LA_THREADS + tid) * N;

    // ---- what counts and biases do to this thread's elements
    float add[LA_UNITS][N];
    uint32_t seen = 0;                                 // bit u * N + e: the element is in the history or the prompt
    float rep = 1.f, rep_inv = 1.f, freq = 0.f, pres = 0.f;
    const int16_t *counts = nullptr;
    const float *bias = nullptr;
    if (ADD) {
        if (a.penalties) {
            counts = p.token_counts + b * p.count_stride;
            if (p.repetition != nullptr) rep = p.repetition[b];
            rep_inv = 1.f / rep;
            if (p.frequency != nullptr) freq = p.frequency[b];
            if (p.presence != nullptr) pres = p.presence[b];
            const int n = draft ? g : i_end - 1;       // drafts that some row of this block has in its history
            const long long first = n > 0 ? p.cu_d[b] : 0;
            for (int j = tid; j < n; j += LA_THREADS) {
                int t = -1;
                if (first < 0 || first + j >= p.n_d_rows) {
                    bad |= SV_DEV_BAD_LEN;
                } else {
                    t = p.draft_tokens[first + j];
                    if (t < 0 || t >= V) {
                        bad |= SV_DEV_BAD_TOKEN;
                        t = -1;
                    }
                }
                tokens[j] = t;
            }
        }
        if (p.n_bias != nullptr) {
            bias = p.bias_values + (long long)b * p.bias_stride;
            for (int i = tid; i < SLICE; i += LA_THREADS) bias_at[i] = 0;
            __syncthreads();
            int n = p.n_bias[b];
            if (n < 0 || n > p.bias_stride) {
                bad |= SV_DEV_BAD_LEN;
                n = min(max(n, 0), p.bias_stride);
            }
            for (int i = tid; i < n; i += LA_THREADS) {
                const int t = p.bias_tokens[(long long)b * p.bias_stride + i];
                if (t < 0 || t >= V) bad |= SV_DEV_BAD_TOKEN;
                else if (t >= base && t < base + SLICE) atomicMax(&bias_at[t - base], i + 1);      // the later entry counts
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            uint32_t w[4] = {0, 0, 0, 0};
            if (counts != nullptr && k0[u] < V) {      // rows of counts are padded to whole units
                if (BF16) {
                    const uint4 c = *reinterpret_cast<const uint4 *>(counts + k0[u]);
                    w[0] = c.x; w[1] = c.y; w[2] = c.z; w[3] = c.w;
                } else {
                    const uint2 c = *reinterpret_cast<const uint2 *>(counts + k0[u]);
                    w[0] = c.x; w[1] = c.y;
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t h = (w[e / 2] >> (16 * (e & 1))) & 0xffffu, c = h & 0x7fffu;
                seen |= (h != 0 ? 1u : 0u) << (u * N + e);
                add[u][e] = -(freq * (float)c + (c > 0 ? pres : 0.f));
                if (bias != nullptr) {
                    const int i = bias_at[k0[u] - base + e];
                    if (i > 0) add[u][e] += bias[i - 1];
                }
            }
        }
    }
    // draft j of the sequence joins the history of the rows from here on
    auto take = [&](int j) {
        const int t = tokens[j];
        if (t < base || t >= base + SLICE) return;
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            if (t < k0[u] || t >= k0[u] + N) continue;
            int c = (counts[t] & 0x7fff) + 1;          // times in the counts and among drafts 0 .. j
            for (int i = 0; i < j; ++i) c += tokens[i] == t ? 1 : 0;
            float v = -(freq * (float)c + pres);
            const int i = bias != nullptr ? bias_at[t - base] : 0;
            if (i > 0) v += bias[i - 1];
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (t == k0[u] + e) add[u][e] = v;
            seen |= 1u << (u * N + t - k0[u]);
        }
    };
    if (ADD && a.penalties)
        for (int j = 0; j < before; ++j) take(j);

    // ---- rows
    for (int i0 = i_begin; i0 < i_end; i0 += LA_AHEAD) {
        uint4 raw[LA_AHEAD][LA_UNITS];
        uint32_t allowed[LA_AHEAD][LA_UNITS];
#pragma unroll
        for (int r = 0; r < LA_AHEAD; ++r) {
            const long long row = row0 + i0 + r;
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                allowed[r][u] = (1u << N) - 1;
                if (MASK && i0 + r < i_end && k0[u] < V)
                    allowed[r][u] &= __ldg(reinterpret_cast<const unsigned char *>(p.mask + row * p.mask_stride) + k0[u] / 8) >> (k0[u] & 7);
            }
        }
#pragma unroll
        for (int r = 0; r < LA_AHEAD; ++r) {
            const void *src = logit_row<BF16>(p.logits, row0 + i0 + r, p.row_stride);
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                raw[r][u] = make_uint4(0, 0, 0, 0);
                if (i0 + r < i_end && k0[u] < V && (!MASK || allowed[r][u] != 0)) unit_load<BF16>(src, k0[u], V, a.vec != 0, raw[r][u]);
            }
        }
#pragma unroll
        for (int r = 0; r < LA_AHEAD; ++r) {
            if (i0 + r >= i_end) break;
            if (ADD && a.penalties && i0 + r > i_begin) take(i0 + r - 1);
            void *dst = const_cast<void *>(logit_row<BF16>(p.out, row0 + i0 + r, p.out_stride));
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                if (k0[u] >= V) continue;
                uint32_t w[4] = {raw[r][u].x, raw[r][u].y, raw[r][u].z, raw[r][u].w};
                float x[N];
#pragma unroll
                for (int e = 0; e < N; ++e)
                    x[e] = BF16 ? __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16) : __uint_as_float(w[e]);
                if (ADD) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float f = (seen >> (u * N + e)) & 1u ? (x[e] > 0.f ? rep_inv : rep) : 1.f;
                        x[e] = x[e] * f + add[u][e];
                    }
                }
                if (MASK) {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (!((allowed[r][u] >> e) & 1u)) x[e] = -CUDART_INF_F;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (BF16) {
                        if (e & 1) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(x[e - 1], x[e]);        // the one rounding
                            w[e / 2] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                    } else {
                        w[e] = __float_as_uint(x[e]);
                    }
                }
                unit_store<BF16>(dst, k0[u], V, a.vec != 0, make_uint4(w[0], w[1], w[2], w[3]));
            }
        }
    }
    if (bad != 0) set_status(p.device_status, bad);
}

template <bool BF16>
static sv_status launch_adjust(LogitsAdjustLaunch &a, cudaStream_t stream)
{
    const sv_logits_adjust_params &p = a.p;
    a.slices = (p.vocab + Unit<BF16>::SLICE - 1) / Unit<BF16>::SLICE;
    const int rows = p.n_drafted != nullptr ? 1 : p.gamma_max + 1;
    a.rows_per_block = rows;
    a.chunks = (rows + a.rows_per_block - 1) / a.rows_per_block;
    const long long blocks = (long long)p.batch * a.chunks * a.slices;
    if (blocks > 0x7fffffffLL) return SV_EUNSUPPORTED;
    const dim3 grid((unsigned)blocks);
    const bool add = a.penalties || p.n_bias != nullptr, mask = p.mask != nullptr;
    if (add && mask) return launch_kernel(true, logits_adjust_kernel<BF16, true, true>, grid, LA_THREADS, 0, stream, a);
    if (add) return launch_kernel(true, logits_adjust_kernel<BF16, true, false>, grid, LA_THREADS, 0, stream, a);
    if (mask) return launch_kernel(true, logits_adjust_kernel<BF16, false, true>, grid, LA_THREADS, 0, stream, a);
    return launch_kernel(true, logits_adjust_kernel<BF16, false, false>, grid, LA_THREADS, 0, stream, a);
}

}  // namespace sv

extern "C" sv_status spec_logits_adjust(const sv_logits_adjust_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr || p->logits == nullptr || p->out == nullptr) return SV_EINVAL;
    if (p->batch <= 0 || p->vocab <= 0 || p->n_rows <= 0 || p->gamma_max < 0) return SV_EINVAL;
    if (p->row_stride < p->vocab || p->out_stride < p->vocab) return SV_EINVAL;
    if (p->gamma_max > LA_MAX_GAMMA || p->vocab > 1 << 30) return SV_EUNSUPPORTED;
    if (p->n_drafted == nullptr ? p->gamma == nullptr || p->cu_q == nullptr : p->n_rows < p->batch) return SV_EINVAL;
    const bool penalties = p->repetition != nullptr || p->frequency != nullptr || p->presence != nullptr;
    if (penalties) {
        if (p->token_counts == nullptr || p->count_stride < p->vocab || p->n_d_rows < 0) return SV_EINVAL;
        if (p->gamma_max > 0 && (p->draft_tokens == nullptr || p->cu_d == nullptr)) return SV_EINVAL;
        if (!aligned16(p->token_counts) || p->count_stride % 8 != 0) return SV_EALIGN;
    }
    if (p->n_bias != nullptr && (p->bias_tokens == nullptr || p->bias_values == nullptr || p->bias_stride <= 0)) return SV_EINVAL;
    if (p->n_bias == nullptr && (p->bias_tokens != nullptr || p->bias_values != nullptr)) return SV_EINVAL;
    if (p->mask != nullptr && p->mask_stride < ((int64_t)p->vocab + 31) / 32) return SV_EINVAL;
    const int size = p->logits_bf16 != 0 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(p->logits) % size != 0 || reinterpret_cast<uintptr_t>(p->out) % size != 0) return SV_EALIGN;
    const bool in_place = p->out == p->logits && p->out_stride == p->row_stride;
    const uintptr_t x = reinterpret_cast<uintptr_t>(p->logits), y = reinterpret_cast<uintptr_t>(p->out);
    const uintptr_t nx = (uintptr_t)((p->n_rows - 1) * p->row_stride + p->vocab) * size;
    const uintptr_t ny = (uintptr_t)((p->n_rows - 1) * p->out_stride + p->vocab) * size;
    if (!in_place && x < y + ny && y < x + nx) return SV_EINVAL;
    if (in_place && !penalties && p->n_bias == nullptr && p->mask == nullptr) return SV_OK;        // nothing to change
    LogitsAdjustLaunch a;
    a.p = *p;
    a.in_place = in_place;
    a.penalties = penalties;
    a.vec = logits_vec_ok(p->logits, p->row_stride, p->logits_bf16 != 0) && logits_vec_ok(p->out, p->out_stride, p->logits_bf16 != 0);
    return p->logits_bf16 != 0 ? launch_adjust<true>(a, (cudaStream_t)stream) : launch_adjust<false>(a, (cudaStream_t)stream);
}
