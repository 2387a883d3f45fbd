// Token counts behind the penalties of spec_logits_adjust: 15 bits of count and one of "in the prompt" per
// (sequence, vocabulary entry).
//
// Counting touches a word per token: a warp joins equal tokens first and adds what is left with compare-and-swap, which
// saturates, so the sum is the same in any order.  An admission writes whole rows: a block takes a slice of the vocabulary,
// collects the prompt's marks in shared memory (a byte each: no atomics, whose conflicts on frequent tokens cost more) and
// writes the slice once, cleared and marked together.  Measured for 128 prompts of 4096 to 8192 tokens at a vocabulary of 128256
// (36 MB, 5.6 us at the copy rate): 9.5 us, of which about 2 are the launch and 2 the prompts, which every slice's block reads
// for itself (slices of 16384 entries: 11 us; blocks of 256 or 1024 threads: 13 and 12 us; tokens one by one: 9.9 us;
// the slices as a cluster that shares the prompt and marks in one another's shared memory: 16.5 us).  Marks as
// bits 11.7 to 12.7 us; slices cleared first and marked in global memory 18 to 23 us (scattered two-byte stores).
#include "common.cuh"

namespace sv {

constexpr int TC_THREADS = 256;
constexpr int TC_RESET_THREADS = 512;
constexpr int TC_SLICE = 32768;            // vocabulary entries of a block that clears

struct TokenCountsLaunch {
    sv_token_counts_params p;
    int parts;                             // blocks per sequence
};

// tokens of sequence b: how many, and the first
__device__ __forceinline__ int tc_range(const sv_token_counts_params &p, int b, const int32_t *&first, uint32_t &bad)
{
    if (p.cu_tokens == nullptr) {
        first = p.tokens + b * p.token_stride;
        return p.max_tokens;
    }
    const long long lo = p.cu_tokens[b], hi = p.cu_tokens[b + 1];
    if (lo < 0 || hi < lo || hi > p.n_tokens || hi - lo > p.max_tokens) {
        bad |= SV_DEV_BAD_LEN;
        return 0;
    }
    first = p.tokens + lo;
    return (int)(hi - lo);
}

// n more of token k, or its prompt mark; half a 32-bit word (rows start at even elements)
__device__ __forceinline__ void tc_add(int16_t *row, int k, int n, bool prompt)
{
    unsigned int *word = reinterpret_cast<unsigned int *>(row + (k & ~1));
    const int shift = (k & 1) * 16;
    if (prompt) {
        atomicOr(word, 0x8000u << shift);
        return;
    }
    unsigned int old = __ldcg(word);
    for (;;) {                                                  // another thread's success is what makes this one try again
        const unsigned int half = (old >> shift) & 0xffffu;
        const unsigned int count = min((half & 0x7fffu) + (unsigned int)n, 0x7fffu) | (half & 0x8000u);
        const unsigned int was = atomicCAS(word, old, (old & ~(0xffffu << shift)) | (count << shift));
        if (was == old) return;
        old = was;
    }
}

// counts `token` (every lane of the warp calls; lanes that have none pass `has` = false)
__device__ __forceinline__ void tc_add_warp(int16_t *row, int token, bool has, bool prompt, int lane)
{
    const unsigned int all = __ballot_sync(0xffffffffu, has);
    if (!has) return;
    const unsigned int same = __match_any_sync(all, token);
    if (lane == __ffs(same) - 1) tc_add(row, token, __popc(same), prompt);
}

// nothing is cleared: a warp per 32 tokens
__global__ void __launch_bounds__(TC_THREADS)
token_counts_kernel(const __grid_constant__ TokenCountsLaunch a)
{
    pdl_enter();
    const sv_token_counts_params &p = a.p;
    const long long warp = (long long)blockIdx.x * (TC_THREADS / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, b = (int)(warp / a.parts), part = (int)(warp - (long long)b * a.parts);
    if (b >= p.batch) return;
    uint32_t bad = 0;
    const int32_t *first = nullptr;
    const int n = tc_range(p, b, first, bad);
    int token = -1;
    if (part * 32 + lane < n) {
        token = first[part * 32 + lane];
        if (token < -1 || token >= p.vocab) {
            bad |= SV_DEV_BAD_TOKEN;
            token = -1;
        }
    }
    tc_add_warp(p.token_counts + b * p.count_stride, token, token >= 0, p.prompt != 0, lane);
    if (bad != 0) set_status(p.device_status, bad);
}

// rows may be cleared: a block per slice of a sequence's vocabulary
__global__ void __launch_bounds__(TC_RESET_THREADS, 2048 / TC_RESET_THREADS)      // as many as an SM takes: with more registers 13 us
token_counts_reset_kernel(const __grid_constant__ TokenCountsLaunch a)
{
    pdl_enter();
    extern __shared__ __align__(16) uint8_t marks[];   // per entry of the slice: 0x80 if the prompt has it
    const sv_token_counts_params &p = a.p;
    const int b = blockIdx.x / a.parts, lo = (blockIdx.x - b * a.parts) * TC_SLICE, tid = threadIdx.x;
    const int hi = min(p.vocab - lo, TC_SLICE) + lo;
    const bool clear = p.reset[b] != 0, marking = clear && p.prompt != 0;
    int16_t *row = p.token_counts + b * p.count_stride;
    uint32_t bad = 0;
    const int32_t *first = nullptr;
    const int n = tc_range(p, b, first, bad);
    // of a token: its entry of the slice; at least hi - lo if it is none of them
    auto entry_of = [&](int token) {
        const unsigned int at = (unsigned int)token - lo;
        if (at >= (unsigned int)(hi - lo) && (unsigned int)token + 1 > (unsigned int)p.vocab) bad = SV_DEV_BAD_TOKEN;
        return at;
    };
    if (marking) {
        auto mark = [&](int token) {
            const unsigned int at = entry_of(token);
            if (at < (unsigned int)(hi - lo)) marks[at] = 0x80;        // whoever else marks it stores the same
        };
        // four tokens a load, the next on its way: up to three in front of the first 16-byte boundary and behind the last go one by one
        const int head = min(n, (int)(-(reinterpret_cast<uintptr_t>(first) >> 2) & 3)), vectors = (n - head) / 4, behind = head + 4 * vectors;
        const int4 *four = reinterpret_cast<const int4 *>(first + head);
        int4 next = tid < vectors ? four[tid] : make_int4(-1, -1, -1, -1);
        const int single = tid < head ? first[tid] : tid - head < n - behind ? first[behind + tid - head] : -1;
        for (int i = tid; i < TC_SLICE / 16; i += TC_RESET_THREADS) reinterpret_cast<uint4 *>(marks)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll 1                                       // unrolled it takes registers and time
        for (int i = tid; i < vectors; i += TC_RESET_THREADS) {
            const int4 t = next;
            if (i + TC_RESET_THREADS < vectors) next = four[i + TC_RESET_THREADS];
            mark(t.x);
            mark(t.y);
            mark(t.z);
            mark(t.w);
        }
        mark(single);
    } else {
        if (clear) {
            for (int k = lo + 8 * tid; k + 8 <= hi; k += 8 * TC_RESET_THREADS) *reinterpret_cast<uint4 *>(row + k) = make_uint4(0, 0, 0, 0);
            for (int k = lo + (hi - lo) / 8 * 8 + tid; k < hi; k += TC_RESET_THREADS) row[k] = 0;
        }
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += TC_RESET_THREADS) {
            const int token = i0 + tid < n ? first[i0 + tid] : -1;
            tc_add_warp(row, token, entry_of(token) < (unsigned int)(hi - lo), p.prompt != 0, tid & 31);
        }
    }
    if (marking) {
        __syncthreads();
        for (int k = lo + 8 * tid; k < hi; k += 8 * TC_RESET_THREADS) {
            const uint2 m = *reinterpret_cast<const uint2 *>(marks + k - lo);
            // a mark's byte becomes the upper one of its 16-bit entry
            const uint32_t w[4] = {__byte_perm(m.x, 0, 0x1404), __byte_perm(m.x, 0, 0x3424), __byte_perm(m.y, 0, 0x1404), __byte_perm(m.y, 0, 0x3424)};
            if (k + 8 <= hi) {
                *reinterpret_cast<uint4 *>(row + k) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                for (int i = 0; k + i < hi; ++i) row[k + i] = (int16_t)(marks[k - lo + i] << 8);
            }
        }
    }
    if (bad != 0) set_status(p.device_status, bad);
}

}  // namespace sv

extern "C" sv_status spec_token_counts_update(const sv_token_counts_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr || p->token_counts == nullptr) return SV_EINVAL;
    if (p->batch <= 0 || p->vocab <= 0 || p->max_tokens < 0 || p->count_stride < p->vocab) return SV_EINVAL;
    if (p->max_tokens > 0 && p->tokens == nullptr) return SV_EINVAL;
    if (p->cu_tokens == nullptr && p->token_stride < p->max_tokens) return SV_EINVAL;
    if (p->cu_tokens != nullptr && p->n_tokens < 0) return SV_EINVAL;
    if (!aligned16(p->token_counts) || p->count_stride % 8 != 0) return SV_EALIGN;
    if (p->reset == nullptr && p->max_tokens == 0) return SV_OK;
    TokenCountsLaunch a;
    a.p = *p;
    cudaStream_t s = (cudaStream_t)stream;
    // room for the loops' last steps in 32 bits
    if (p->max_tokens > 1 << 30 || p->vocab > 1 << 30) return SV_EUNSUPPORTED;
    a.parts = p->reset != nullptr ? (p->vocab + TC_SLICE - 1) / TC_SLICE : (p->max_tokens + 31) / 32;
    const long long items = (long long)p->batch * a.parts;
    const long long blocks = p->reset != nullptr ? items : (items + TC_THREADS / 32 - 1) / (TC_THREADS / 32);
    if (blocks > 0x7fffffffLL) return SV_EUNSUPPORTED;
    return p->reset != nullptr ? launch_kernel(true, token_counts_reset_kernel, dim3((unsigned)blocks), TC_RESET_THREADS, p->prompt != 0 ? TC_SLICE : 0, s, a)
                               : launch_kernel(true, token_counts_kernel, dim3((unsigned)blocks), TC_THREADS, 0, s, a);
}
