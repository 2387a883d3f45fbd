// Penalties, biases and grammar masks on logit rows in one pass (paper Section 3: target and draft sample from these rows).
//
// A block takes a slice of the vocabulary and the rows of one sequence's block.  What the counts and the bias list do to
// an element is the same for all of these rows, x * factor + add, except where a draft token falls on it: the counts and the
// list are read once, the two numbers stay in registers, and row i + 1 only updates the element that draft i names.  Rows and
// masks stream through a ring in shared memory.  HBM bounds it: the logits in and out, a bit of mask per element, and 2 bytes
// of counts per block of rows.
//
// Measured: 2176 float32 rows of 128256 with penalties, masks and 300 biases each 343 us (2.3 GB, 6.7 TB/s); bf16 rows of 128256
// (64 sequences of 5 to 9) 41 us with penalties, 50 us with masks and 300 biases too (38 and 39 us at the copy rate):
// instructions bound the latter.  Work in place (no ring: what the counts and the mask say comes before the loads) 236 us for the
// float32 rows with penalties, which leave most units alone, but 378 us with masks too and 391 us with all rules: a mask that clears
// some bits of most units spares no load, and rows are loaded when they are needed.  One draft row each of 64 sequences, with
// penalties: float32 24 us (13 at the copy rate, 4032 blocks on 592 places), bf16 17 us (8; 2048 blocks); every block makes its
// way through counts and drafts for a single row.  Steps that led here: rows loaded to registers two ahead
// 651 us; the effect of each draft prepared once per block and rows one at a time at a higher occupancy 379 us; the ring 353 us;
// masks through the ring 343 us.  A correction of the touched elements alone, in the ring, needs fewer instructions where they
// are few, but the slices that hold most of a history (frequent tokens have neighbouring ids) then keep the others waiting: 4
// sequences at a vocabulary of 32000 took 8.5 us instead of 3.8, the bf16 rows 49 us instead of 41.
#include <type_traits>

#include "common.cuh"
#include "row_stream.cuh"

namespace sv {

constexpr int LA_THREADS = 256;
constexpr int LA_UNITS = 2;                // 16-byte units of a row that a thread has
constexpr int LA_BLOCKS = 4;               // blocks of an SM, with penalties or biases
constexpr int LA_BLOCKS_MASK = 6;          // and with masks alone
constexpr int LA_BLOCKS_DIRECT = 8;        // or in place
constexpr int LA_MAX_GAMMA = 64;
constexpr int LA_STAGES = 4;               // rows of the ring
constexpr int LA_PART = 1 + LA_UNITS * 32; // vectors of a row's part in the ring that a warp has
constexpr int LA_RING = LA_THREADS / 32 * LA_PART;
enum { LA_RING_PATH, LA_DIRECT, LA_SHIFT };
constexpr int LA_BIASES = 1024;            // entries of the bias list at a time

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

// 16 bytes from global to shared memory, asynchronously; a group is the copies between two commits of a thread
__device__ __forceinline__ void cp_chunk(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// its first `bytes` bytes, zeros behind them; no more is read
__device__ __forceinline__ void cp_part(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_word(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Elements of a slice: a warp has LA_UNITS * 32 neighbouring units of 16 bytes, a thread unit u * 32 + lane of them.
template <bool BF16>
struct Layout {
    static constexpr int N = BF16 ? 8 : 4;                      // elements of a unit
    static constexpr int PART = 32 * LA_UNITS * N;              // elements of a warp
    static constexpr int SLICE = LA_THREADS / 32 * PART;        // elements of a block
    static_assert(SLICE <= 1 << 16, "an element of a slice fits 16 bits");
    static __device__ __forceinline__ int at(int u, int e, int tid) { return (((tid >> 5) * LA_UNITS + u) * 32 + (tid & 31)) * N + e; }
    static __device__ __forceinline__ int owner(int at) { return at / (32 * LA_UNITS * N) * 32 + at / N % 32; }
    static __device__ __forceinline__ int unit(int at) { return at / (32 * N) % LA_UNITS; }
};

// A thread's units of a row that lies across vectors of shared memory: unit u starts at element s (the same for all lanes) of
// vector v[32 * u].  Vectors at and behind v_end are not read.  Two 16-byte reads a unit and words picked by a branch: single
// words, 16 bytes apart from lane to lane, meet in every fourth bank.
template <bool BF16>
__device__ __forceinline__ void read_units(const uint4 *v, const uint4 *v_end, int s, uint32_t (&w)[LA_UNITS][4])
{
    uint32_t x[LA_UNITS][8];
#pragma unroll
    for (int u = 0; u < LA_UNITS; ++u) {
        const uint4 a = v[32 * u];
        x[u][0] = a.x; x[u][1] = a.y; x[u][2] = a.z; x[u][3] = a.w;
        x[u][4] = x[u][5] = x[u][6] = x[u][7] = 0;
        if (s > 0 && v + 32 * u + 1 < v_end) {
            const uint4 b = v[32 * u + 1];
            x[u][4] = b.x; x[u][5] = b.y; x[u][6] = b.z; x[u][7] = b.w;
        }
    }
    auto take = [&](auto first) {                      // words first .. first + 3, half a word further on for odd elements
        constexpr int F = decltype(first)::value;
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[u][i] = BF16 ? __funnelshift_r(x[u][F + i], x[u][F + i + 1 < 8 ? F + i + 1 : 7], 16 * (s & 1)) : x[u][F + i];
    };
    switch (BF16 ? s >> 1 : s) {
        case 0: return take(std::integral_constant<int, 0>());
        case 1: return take(std::integral_constant<int, 1>());
        case 2: return take(std::integral_constant<int, 2>());
        default: return take(std::integral_constant<int, 3>());
    }
}

// ADD: penalties or biases; MASK: grammar masks.
// PATH: LA_RING_PATH where every unit of every row starts on a 16-byte boundary and ends inside the vocabulary; LA_DIRECT where
// that is so and the call works in place: units that do not change are not loaded, so what the mask and the counts say comes
// before the loads.  Elsewhere LA_SHIFT: a row's 16-byte boundaries lie d elements behind the units' (a vocabulary of odd size,
// say), d differing from row to row: global accesses keep to the boundaries, and a warp moves its units to and from them in
// shared memory.  (By shuffles and selects instead this took 340 warp instructions per 32 units, and 44 us for bf16 rows of
// 50257 where this takes 30.6; by single elements 66; with vectors on the boundaries and what is added to their elements
// looked up in shared memory 32.7.)
template <bool BF16, bool ADD, bool MASK, int PATH>
__global__ void __launch_bounds__(LA_THREADS, ADD ? LA_BLOCKS : PATH == LA_DIRECT ? LA_BLOCKS_DIRECT : LA_BLOCKS_MASK)
logits_adjust_kernel(const __grid_constant__ LogitsAdjustLaunch a)
{
    pdl_enter();
    using L = Layout<BF16>;
    constexpr bool VEC = PATH != LA_SHIFT, ahead = PATH != LA_DIRECT;
    constexpr int N = L::N, SLICE = L::SLICE, ES = 16 / N;
    __shared__ int draft_at[LA_MAX_GAMMA];             // element of the slice that draft j names, or -1
    __shared__ float draft_add[LA_MAX_GAMMA];          // what is added to it once the draft is in the history
    __shared__ int bias_head[ADD ? LA_THREADS : 1];    // entries of the bias list that name an element of thread t: a linked list, -1 its end
    __shared__ int bias_node[ADD ? LA_BIASES : 1];     // per entry: its element of the slice, and the next entry of the thread's list << 16
    __shared__ uint32_t mask_ring[MASK && ahead ? LA_STAGES : 1][LA_THREADS / 32][L::PART / 32];      // the rows' masks
    __shared__ uint2 keep[MASK && BF16 && ahead ? 16 : 1];      // what four allowed bits keep of four bf16 elements
    const sv_logits_adjust_params &p = a.p;
    const int tid = threadIdx.x, lane = tid & 31, V = p.vocab;
    const int slice = blockIdx.x % a.slices, seq_chunk = blockIdx.x / a.slices;
    const int b = seq_chunk / a.chunks, chunk = seq_chunk - b * a.chunks;
    uint32_t bad = 0;
    const bool draft = p.n_drafted != nullptr;
    // what the sequence says, loaded together
    const int active = p.active != nullptr ? p.active[b] : 1;
    const long long row0 = draft ? b : p.cu_q[b];
    const long long first_draft = ADD && a.penalties && p.gamma_max > 0 ? p.cu_d[b] : 0;
    int g = draft ? ADD && a.penalties ? p.n_drafted[b] : 0 : p.gamma[b];
    if (active == 0) return;
    if (g < 0 || g > p.gamma_max) {
        bad |= SV_DEV_BAD_GAMMA;
        g = min(max(g, 0), p.gamma_max);
    }
    const int rows = draft ? 1 : g + 1, i_begin = chunk * a.rows_per_block, i_end = min(rows, i_begin + a.rows_per_block);
    // of thread j: draft j of the sequence, whether or not this step has so many
    int my_token = 0;
    bool my_token_there = false;
    if (ADD && a.penalties && tid < p.gamma_max) {     // at most LA_MAX_GAMMA
        const long long at = first_draft + tid;
        my_token_there = at >= tid && at < p.n_d_rows;
        if (my_token_there) my_token = p.draft_tokens[at];
    }
    if (i_begin >= i_end) {
        if (bad != 0 && tid == 0) set_status(p.device_status, bad);
        return;
    }
    if (row0 < 0 || row0 + rows > p.n_rows) {
        if (tid == 0) set_status(p.device_status, bad | SV_DEV_BAD_LEN);
        return;
    }
    const int base = slice * SLICE;

    // ---- loads that nothing waits for come first: the first row, unless the counts and the mask may spare it, and the counts
    const unsigned char *mask = MASK ? reinterpret_cast<const unsigned char *>(p.mask + (row0 + i_begin) * p.mask_stride) : nullptr;
    const char *src = static_cast<const char *>(p.logits) + (row0 + i_begin) * p.row_stride * ES;
    char *dst = static_cast<char *>(p.out) + (row0 + i_begin) * p.out_stride * ES;
    uint32_t w[LA_UNITS][4];
    // Rows come through a ring in shared memory, LA_STAGES - 1 ahead.
    // A warp's part of a row: the vector in front of its first unit (used where boundaries and units differ), then its vectors.
    extern __shared__ __align__(16) uint4 la_ring[];   // [LA_STAGES][warps][LA_PART]
    const uint4 *part = la_ring + (tid >> 5) * LA_PART;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(part);
    int p_row = i_begin, p_stage = 0;
    const char *p_src = src;
    const unsigned char *p_mask = mask;
    const uint32_t mask_to = (uint32_t)__cvta_generic_to_shared(&mask_ring[0][MASK ? tid >> 5 : 0][MASK ? lane % (L::PART / 32) : 0]);
    if (MASK && BF16 && ahead && tid < 16)
        keep[tid] = make_uint2((tid & 1 ? 0xffffu : 0u) | (tid & 2 ? 0xffff0000u : 0u), (tid & 4 ? 0xffffu : 0u) | (tid & 8 ? 0xffff0000u : 0u));
    if (MASK && BF16 && ahead) __syncthreads();
    auto shift_of = [&](const void *row) { return VEC ? 0 : (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / ES; };
    auto issue = [&]() {
        if (p_row < i_end) {
            const int d = shift_of(p_src);
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                const int k = base + L::at(u, 0, tid) + d;
                const uint32_t to = ring + (p_stage * LA_RING + 1 + u * 32 + lane) * 16;
                if (VEC) {
                    if (k < V) cp_chunk(to, p_src + (long long)k * ES);
                } else {
                    if (k < V) cp_part(to, p_src + (long long)k * ES, min(V - k, N) * ES);
                    const char *front = p_src + (long long)(k - N) * ES;
                    if (u == 0 && lane == 0 && d > 0 && k - N < V && front >= p.logits) cp_part(ring + p_stage * LA_RING * 16, front, min(V - k + N, N) * ES);
                }
            }
            if (MASK) {
                const int k = base + (tid >> 5) * L::PART + 32 * lane;
                if (lane < L::PART / 32 && k < V) cp_word(mask_to + p_stage * sizeof(mask_ring[0]), p_mask + k / 8);
                p_mask += p.mask_stride * 4;
            }
            ++p_row;
            p_src += p.row_stride * ES;
        }
        p_stage = p_stage + 1 == LA_STAGES ? 0 : p_stage + 1;
        cp_commit();                                   // an empty group where nothing is left
    };
    if (ahead) {
#pragma unroll
        for (int s = 0; s < LA_STAGES - 1; ++s) issue();
    }
    const int16_t *counts = ADD && a.penalties ? p.token_counts + b * p.count_stride + base : nullptr;
    uint32_t held[LA_UNITS][N / 2];                    // counts of this thread's units
    if (ADD) {
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            const int k = L::at(u, 0, tid);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) held[u][i] = 0;
            if (counts == nullptr) continue;
            if (base + k >= V) continue;               // rows of counts are padded to whole units
            if (BF16) {
                const uint4 c = *reinterpret_cast<const uint4 *>(counts + k);
                held[u][0] = c.x; held[u][1] = c.y; held[u][N / 2 - 2] = c.z; held[u][N / 2 - 1] = c.w;
            } else {
                const uint2 c = *reinterpret_cast<const uint2 *>(counts + k);
                held[u][0] = c.x; held[u][1] = c.y;
            }
        }
    }
    int bias_token[LA_BIASES / LA_THREADS];            // entries tid, tid + LA_THREADS, .. of the bias list
    if (ADD && p.n_bias != nullptr) {
#pragma unroll
        for (int c = 0; c < LA_BIASES / LA_THREADS; ++c) {
            const int i = c * LA_THREADS + tid;
            bias_token[c] = i < p.bias_stride ? p.bias_tokens[(long long)b * p.bias_stride + i] : 0;
        }
    }
    // ---- what counts and biases do to this thread's elements
    float add[LA_UNITS][N];
    uint32_t seen = 0;                                 // bit u * N + e: the element is in the history or the prompt
    float rep = 1.f, rep_inv = 1.f;
    const int before = draft ? g : i_begin;            // drafts in front of the block's first row
    const int n_drafts = ADD && a.penalties ? draft ? g : i_end - 1 : 0;       // drafts that some row of this block has in its history
    if (ADD) {
        float freq = 0.f, pres = 0.f;
        auto penalty = [&](int c) { return -(freq * (float)c + (c > 0 ? pres : 0.f)); };
        int my_at = -1;                                // of thread j: the element that draft j names,
        float my_add = 0.f, my_bias = 0.f;             // its penalty with drafts 0 .. j in the history, its bias
        if (a.penalties) {
            if (p.repetition != nullptr) rep = p.repetition[b];
            rep_inv = 1.f / rep;
            if (p.frequency != nullptr) freq = p.frequency[b];
            if (p.presence != nullptr) pres = p.presence[b];
            if (tid < n_drafts) {
                if (!my_token_there) bad |= SV_DEV_BAD_LEN;
                else if (my_token < 0 || my_token >= V) bad |= SV_DEV_BAD_TOKEN;
                else if (my_token >= base && my_token < base + SLICE) my_at = my_token - base;
                draft_at[tid] = my_at;
            }
            if (n_drafts > 0) __syncthreads();
            if (my_at >= 0) {
                int c = (counts[my_at] & 0x7fff) + 1;
                for (int i = 0; i < tid; ++i) c += draft_at[i] == my_at ? 1 : 0;
                my_add = penalty(c);
            }
        }
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t h = (held[u][e / 2] >> (16 * (e & 1))) & 0xffffu;
                seen |= (h != 0 ? 1u : 0u) << (u * N + e);
                add[u][e] = penalty(h & 0x7fff);
            }
        if (p.n_bias != nullptr) {
            int n = p.n_bias[b];
            if (n < 0 || n > p.bias_stride) {
                bad |= SV_DEV_BAD_LEN;
                n = min(max(n, 0), p.bias_stride);
            }
            const int32_t *bias_tokens = p.bias_tokens + (long long)b * p.bias_stride;
            const float *bias_values = p.bias_values + (long long)b * p.bias_stride;
            for (int i0 = 0; i0 < n; i0 += LA_BIASES) {
                if (i0 > 0) __syncthreads();
                bias_head[tid] = -1;
                __syncthreads();
#pragma unroll
                for (int c = 0; c < LA_BIASES / LA_THREADS; ++c) {
                    const int i = c * LA_THREADS + tid, t = i0 == 0 ? bias_token[c] : i0 + i < n ? bias_tokens[i0 + i] : 0;
                    if (i0 + i >= n) break;
                    if (t < 0 || t >= V) bad |= SV_DEV_BAD_TOKEN;
                    else if (t >= base && t < base + SLICE)
                        bias_node[i] = (t - base) | atomicExch(&bias_head[L::owner(t - base)], i) << 16;
                }
                __syncthreads();
                // entry that decides about element `at` in this part of the list, or -1: the last that names it
                auto look_up = [&](int at) {
                    int found = -1;
                    for (int i = bias_head[L::owner(at)]; i >= 0; i = bias_node[i] >> 16)
                        if ((bias_node[i] & 0xffff) == at) found = max(found, i);
                    return found;
                };
                for (int i = bias_head[tid]; i >= 0; i = bias_node[i] >> 16) {
                    const int at = bias_node[i] & 0xffff;
                    if (look_up(at) != i) continue;
                    const float v = bias_values[i0 + i] + penalty(counts != nullptr ? counts[at] & 0x7fff : 0);
#pragma unroll
                    for (int u = 0; u < LA_UNITS; ++u)
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (at == L::at(u, e, tid)) add[u][e] = v;
                }
                if (my_at >= 0) {
                    const int i = look_up(my_at);
                    if (i >= 0) my_bias = bias_values[i0 + i];
                }
            }
        }
        if (n_drafts > 0) {
            if (my_at >= 0) draft_add[tid] = my_add + my_bias;
            __syncthreads();
        }
    }
    // draft j of the sequence joins the history of the rows from here on
    auto take = [&](int j) {
        const int at = draft_at[j];
        const float v = draft_add[j];
        if (at < 0 || L::owner(at) != tid) return;
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at == L::at(u, e, tid)) {
                    add[u][e] = v;
                    seen |= 1u << (u * N + e);
                }
    };
    for (int j = 0; j < min(before, n_drafts); ++j) take(j);
    // In place, a unit that nothing is added to in any of the rows is left alone where the mask allows all of it.
    uint32_t still = 0;                                // bit u
    if (!ahead) {
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            bool moves = false;
            if (ADD) {
                moves = ((seen >> (u * N)) & ((1u << N) - 1)) != 0;
#pragma unroll
                for (int e = 0; e < N; ++e) moves = moves || add[u][e] != 0.f;
            }
            still |= (moves ? 0u : 1u) << u;
        }
        for (int j = before; j < n_drafts; ++j) {
            const int at = draft_at[j];
            if (at < 0 || L::owner(at) != tid) continue;
            still &= ~(1u << L::unit(at));
        }
    }

    // ---- rows
    auto mask_row = [&]() {                            // what `mask` points to allows of this thread's elements, bit u * N + e
        uint32_t allowed = 0;
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            const int k = base + L::at(u, 0, tid);
            if (k < V) allowed |= ((mask[k / 8] >> (k & 7)) & ((1u << N) - 1)) << (u * N);
        }
        return allowed;
    };
    int stage = 0;
    uint32_t next = MASK && !ahead ? mask_row() : 0xffffffffu;
    for (int i = i_begin; i < i_end; ++i) {
        uint32_t allowed = next;
        if (MASK && !ahead && i + 1 < i_end) {         // a row ahead: it decides what is loaded
            mask += p.mask_stride * 4;
            next = mask_row();
        }
        uint4 *out_slot = nullptr;                     // where the row's results meet
        if (ahead) {
            cp_wait<LA_STAGES - 2>();
            const uint4 *slot = part + stage * LA_RING;
            if (MASK || !VEC) __syncwarp();            // every lane's copies of this row are there
            if (MASK) {
                const unsigned char *bits = reinterpret_cast<const unsigned char *>(mask_ring[stage][tid >> 5]);
                allowed = 0;
#pragma unroll
                for (int u = 0; u < LA_UNITS; ++u) {
                    const int e = (u * 32 + lane) * N;
                    allowed |= (bits[e / 8] >> (e & 7) & ((1u << N) - 1)) << (u * N);
                }
            }
            if (VEC) {
#pragma unroll
                for (int u = 0; u < LA_UNITS; ++u) {
                    const uint4 v = slot[1 + u * 32 + lane];
                    w[u][0] = v.x; w[u][1] = v.y; w[u][2] = v.z; w[u][3] = v.w;
                }
            } else {
                const int d = shift_of(src);
                if (d > 0 && base + tid == 0 && src - (N - d) * ES < p.logits) {       // nothing lies before the first row
                    for (int e = 0; e < min(d, V); ++e) {
                        char *to = reinterpret_cast<char *>(const_cast<uint4 *>(slot)) + 16 - (d - e) * ES;
                        if (BF16) *reinterpret_cast<unsigned short *>(to) = reinterpret_cast<const unsigned short *>(src)[e];
                        else *reinterpret_cast<uint32_t *>(to) = reinterpret_cast<const uint32_t *>(src)[e];
                    }
                }
                read_units<BF16>(slot + (d > 0 ? 0 : 1) + lane, slot + LA_PART, d > 0 ? N - d : 0, w);
                __syncwarp();                          // and are read
                out_slot = const_cast<uint4 *>(slot) + 1;
            }
            stage = stage + 1 == LA_STAGES ? 0 : stage + 1;
            issue();
        } else {
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                w[u][0] = w[u][1] = w[u][2] = w[u][3] = 0;
                const int k = base + L::at(u, 0, tid);
                const uint32_t own = allowed >> (u * N) & ((1u << N) - 1);
                if (k < V && own != 0 && !((still >> u) & 1u && own == (1u << N) - 1)) {
                    const uint4 v = ld_once(src + (long long)k * ES);
                    w[u][0] = v.x; w[u][1] = v.y; w[u][2] = v.z; w[u][3] = v.w;
                }
            }
        }
        src += p.row_stride * ES;
        if (i > i_begin && i <= n_drafts) take(i - 1);
#pragma unroll
        for (int u = 0; u < LA_UNITS; ++u) {
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = BF16 ? __uint_as_float(e & 1 ? w[u][e / 2] & 0xffff0000u : w[u][e / 2] << 16) : __uint_as_float(w[u][e & 3]);
                if (ADD) x[e] = x[e] * ((seen >> (u * N + e)) & 1u ? (x[e] > 0.f ? rep_inv : rep) : 1.f) + add[u][e];
                if (MASK && !BF16 && !((allowed >> (u * N + e)) & 1u)) x[e] = -CUDART_INF_F;
                if (!BF16) w[u][e & 3] = __float_as_uint(x[e]);
                else if (e & 1) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(x[e - 1], x[e]);                // the one rounding
                    w[u][e / 2] = *reinterpret_cast<const uint32_t *>(&h);
                }
            }
        }
        if (MASK && BF16) {                            // -inf in what is not allowed
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                uint32_t stay[4];
                if (ahead) {
                    const uint2 lo = keep[allowed >> (u * N) & 15], hi = keep[allowed >> (u * N + 4) & 15];
                    stay[0] = lo.x; stay[1] = lo.y; stay[2] = hi.x; stay[3] = hi.y;
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        stay[c] = (allowed >> (u * N + 2 * c) & 1u ? 0xffffu : 0u) | (allowed >> (u * N + 2 * c + 1) & 1u ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) w[u][c] = (w[u][c] & stay[c]) | (0xff80ff80u & ~stay[c]);
            }
        }
        if (VEC) {
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                const int k = base + L::at(u, 0, tid);
                const uint32_t own = allowed >> (u * N) & ((1u << N) - 1);
                if (k < V && !((still >> u) & 1u && own == (1u << N) - 1))
                    *reinterpret_cast<uint4 *>(dst + (long long)k * ES) = make_uint4(w[u][0], w[u][1], w[u][2], w[u][3]);
            }
        } else {
            const int d = shift_of(dst);
            const int first = base + L::at(0, 0, tid & ~31), end = min(first + 32 * LA_UNITS * N, V);      // elements of the warp
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) out_slot[u * 32 + lane] = make_uint4(w[u][0], w[u][1], w[u][2], w[u][3]);
            __syncwarp();
            read_units<BF16>(out_slot + lane, out_slot + LA_UNITS * 32, d, w);
#pragma unroll
            for (int u = 0; u < LA_UNITS; ++u) {
                const int k = first + d + (u * 32 + lane) * N;
                if (k + N <= end) *reinterpret_cast<uint4 *>(dst + (long long)k * ES) = make_uint4(w[u][0], w[u][1], w[u][2], w[u][3]);
            }
            // the elements in front of the first boundary, and behind the last vector: fewer than N each
            const int behind = end - first <= d ? end : end - (end - first - d) % N;
            const int k = lane < N ? (first + lane < min(first + d, end) ? first + lane : -1)
                                   : (lane < 2 * N && behind + lane - N < end ? behind + lane - N : -1);
            if (k >= 0) {
                if (BF16) reinterpret_cast<unsigned short *>(dst)[k] = reinterpret_cast<const unsigned short *>(out_slot)[k - first];
                else reinterpret_cast<uint32_t *>(dst)[k] = reinterpret_cast<const uint32_t *>(out_slot)[k - first];
            }
        }
        dst += p.out_stride * ES;
    }
    if (bad != 0) set_status(p.device_status, bad);
}

template <bool BF16, bool ADD, bool MASK, int PATH>
static sv_status launch_one(const LogitsAdjustLaunch &a, dim3 grid, cudaStream_t stream)
{
    return launch_kernel(true, logits_adjust_kernel<BF16, ADD, MASK, PATH>, grid, LA_THREADS, PATH != LA_DIRECT ? (size_t)LA_STAGES * LA_RING * 16 : 0, stream, a);
}
template <bool BF16, int PATH>
static sv_status launch_kinds(const LogitsAdjustLaunch &a, bool add, bool mask, dim3 grid, cudaStream_t stream)
{
    if (add && mask) return launch_one<BF16, true, true, PATH>(a, grid, stream);
    if (add) return launch_one<BF16, true, false, PATH>(a, grid, stream);
    if (mask || PATH == LA_DIRECT) return launch_one<BF16, false, true, PATH>(a, grid, stream);
    return launch_one<BF16, false, PATH == LA_DIRECT, PATH>(a, grid, stream);      // a copy; in place it has returned already
}

template <bool BF16>
static sv_status launch_adjust(LogitsAdjustLaunch &a, cudaStream_t stream)
{
    const sv_logits_adjust_params &p = a.p;
    constexpr int slice = Layout<BF16>::SLICE;
    a.slices = (p.vocab + slice - 1) / slice;
    const int rows = p.n_drafted != nullptr ? 1 : p.gamma_max + 1;
    // Few blocks: a sequence's rows are dealt out as well.
    const long long whole = (long long)p.batch * a.slices, resident = (long long)sm_count() * LA_BLOCKS;
    const long long split = resident / whole < 1 ? 1 : resident / whole < rows ? resident / whole : rows;
    a.rows_per_block = (int)((rows + split - 1) / split);
    a.chunks = (rows + a.rows_per_block - 1) / a.rows_per_block;
    const long long blocks = (long long)p.batch * a.chunks * a.slices;
    if (blocks > 0x7fffffffLL) return SV_EUNSUPPORTED;
    const dim3 grid((unsigned)blocks);
    const bool add = a.penalties || p.n_bias != nullptr, mask = p.mask != nullptr;
    if (!a.vec) return launch_kinds<BF16, LA_SHIFT>(a, add, mask, grid, stream);
    return a.in_place ? launch_kinds<BF16, LA_DIRECT>(a, add, mask, grid, stream) : launch_kinds<BF16, LA_RING_PATH>(a, add, mask, grid, stream);
}

}  // namespace sv

extern "C" sv_status spec_logits_adjust(const sv_logits_adjust_params *p, void *stream)
{
    using namespace sv;
    if (p == nullptr || p->logits == nullptr || p->out == nullptr) return SV_EINVAL;
    if (p->batch <= 0 || p->vocab <= 0 || p->n_rows <= 0 || p->gamma_max < 0) return SV_EINVAL;
    if (p->row_stride < p->vocab || p->out_stride < p->vocab) return SV_EINVAL;
    if (p->gamma_max > LA_MAX_GAMMA || p->vocab > 1 << 30 || p->bias_stride > 1 << 30) return SV_EUNSUPPORTED;
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
    if (reinterpret_cast<uintptr_t>(p->mask) % 4 != 0) return SV_EALIGN;
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
    // whole units, all of them: the vocabulary ends with a unit
    a.vec = p->vocab % (p->logits_bf16 != 0 ? 8 : 4) == 0 && logits_vec_ok(p->logits, p->row_stride, p->logits_bf16 != 0) && logits_vec_ok(p->out, p->out_stride, p->logits_bf16 != 0);
    return p->logits_bf16 != 0 ? launch_adjust<true>(a, (cudaStream_t)stream) : launch_adjust<false>(a, (cudaStream_t)stream);
}
