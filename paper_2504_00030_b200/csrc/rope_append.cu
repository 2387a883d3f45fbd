// Per-head norm of queries and keys, position rotation and cache append in one pass (KV caching, paper Section 5).
//
// y = x * w * rsqrt(mean(x^2) + eps), then z = y rotated by the row's angles; queries to the attention's input, keys and
// values to the row's slot of the paged cache.  Every element is read once and written once, so HBM bounds large
// calls and the latency of one pass through the chain small ones.
//
// A lane holds two 16-byte chunks (16 dims) of a head and head_dim / 16 lanes hold the head.  Which two is chosen so
// that a rotated pair never leaves its lane: the norm's sum alone crosses lanes (two or three shuffles).
//
// One warp takes one row, or a part of its heads when there are few rows; its heads arrive through a ring of asynchronous
// copies in shared memory, up to RA_STAGES - 1 KB ahead, while the angles are formed and earlier heads are finished.  Measured
// for 16381 rows of 32 + 8 + 8 heads of 128 dims (402 MB, 62 us at the copy rate): 157 us with a block per row and the
// angles shared through its barrier, 81 us with loads held in registers two rounds ahead, 66 us with the ring, 64.5 us (6.2 TB/s)
// with the first copies under way before the row's slot is known.  Half of that way is instructions: scalar float32 arithmetic
// took 64 million warp instructions (72 % of the issue slots), the packed form below 42 million.  Warps that loop over rows
// and fetch the next row's slot early run in step with one another and reach 5.2 TB/s only.  Rows of few heads are bound by what
// a row costs before its first head (angles, factors), and their rounds of keys and values leave lanes idle.  Where there are many
// such rows, a warp takes several, a head of each in a round, and forms the factors' weights once: one row a warp / several, by
// launch_rope's estimate: 16381 rows of 8 + 1 + 1 heads of 128 26.5 / 18.9 us (13 at the copy rate), of 4 + 1 + 1 heads of 64
// 21.5 / 7.6 (4), of 1 + 1 + 1 heads of 128 22.7 / 10.8; of 12 + 4 + 4 (10000 rows) 21.0 / 24.4, of 32 + 8 + 8 63.6 / 69.0.
// The turns' places in shared memory without bank conflicts are 5 us of the first.
#include "attn_common.cuh"
#include "common.cuh"

namespace sv {

constexpr int RA_THREADS = 256;
constexpr int RA_BLOCKS_PER_SM = 2;        // the factors take registers: three blocks spill, 97 us instead of 66
constexpr int RA_WARPS = RA_THREADS / 32;
constexpr int ra_stages(bool rows) { return rows ? 4 : 5; }      // rounds of a warp under way, in shared memory (1 KB each)
constexpr int RA_PAGE = 16;
// What a warp does before its first round (angles, factors, the pipeline's start), in rounds: with one row, and with several
// (each row's angles, the factors once).
constexpr int RA_BEFORE = 2, RA_BEFORE_ROWS = 5;
// Rows of more rounds than this are not taken several at a time: HBM bounds them, and is read better in whole rows.  One / several,
// us: 3000 rows of 32 + 32 + 32 heads of 128 25.3 / 27.9, 16381 of 48 + 12 + 12 of 64 51.8 / 58.5 (24 and 10 rounds); 3000 of
// 16 + 2 + 2 of 128 10.6 / 8.2, 8192 of 12 + 12 + 12 of 64 18.7 / 15.7 (6 rounds).
constexpr int RA_FEW_ROUNDS = 8;
constexpr int RA_MAX_FREQ = 64;            // rot_dim <= head_dim <= 128
constexpr int RA_MAX_HEADS = 1 << 20;      // a head's place in its row, in chunks, stays within 32 bits

struct RopeAppendLaunch {
    sv_rope_append_params p;
    uint4 *k_pool;
    uint4 *v_pool;
    long long n_slots;
    long long stride_page, stride_head, stride_slot;   // in 16-byte chunks, as the rows' strides
    long long q_stride, k_stride, v_stride;
    int q_chunks;                          // of a row of q_out
    int hkv, lanes;                        // lanes that hold a head (head_dim / 16)
    int q_rounds, k_rounds;                // rounds of a row's queries; of its keys, and of its values
    int rounds, segments;                  // rounds of a warp; warps that share a row
    float inv_dim;
};

// 16 bytes from global to shared memory, asynchronously; a group is the copies between two commits of a thread
__device__ __forceinline__ void cp_chunk(uint32_t dst, const uint4 *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Two float32 values in a register pair: one instruction does both (the kernel is bound by instructions issued before it is
// bound by HBM).
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ float2 split(f32x2 v)
{
    float2 x;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x.x), "=f"(x.y) : "l"(v));
    return x;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 unpack2(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(f32x2 v)                   // the one rounding
{
    const float2 x = split(v);
    const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Fraction of a turn that one position step adds at a frequency, in units of 2^-64.  pos * step in 64-bit integers then
// drops whole turns exactly, at any 32-bit position: the angle of a far position keeps its digits, and one product is
// all that is left to float64 arithmetic.
__device__ __forceinline__ unsigned long long turn_step(double inv_freq)
{
    const long long bits = __double_as_longlong(inv_freq * 0.15915494309189535);        // turns per position
    const int e = (int)(bits >> 52 & 0x7ff), s = e - 1011;                              // m * 2^(e - 1075) turns
    const unsigned long long m = (bits & 0xfffffffffffffLL) | (e != 0 ? 1LL << 52 : 0);
    const unsigned long long x = s >= 64 || s <= -64 ? 0 : s >= 0 ? m << s : m >> -s;
    return bits < 0 ? 0 - x : x;
}

template <bool ROWS>
struct RopeShared {
    uint4 ring[RA_WARPS][ra_stages(ROWS)][2][32];      // a round's chunks on their way: each lane reads back its own
    float2 turns[RA_WARPS][(ROWS ? 4 : 1) * RA_MAX_FREQ];      // (cos, sin) of the warp's row or rows
};

// GL: lanes given to a head (a power of two >= head_dim / 16).  PAIRED: pairs (2f, 2f + 1).  WF32: float32 weights.
// A round is 32 / GL heads of one kind (queries, keys, values); a warp has `rounds` consecutive rounds of a row.  ROWS: a warp
// takes 32 / GL rows, a round is one head of each.
template <int GL, bool PAIRED, bool WF32, bool ROWS>
__global__ void __launch_bounds__(RA_THREADS, RA_BLOCKS_PER_SM)
rope_append_kernel(const __grid_constant__ RopeAppendLaunch a)
{
    pdl_enter();
    constexpr int HEADS = ROWS ? 1 : 32 / GL, ROWS_WARP = ROWS ? 32 / GL : 1, TEAM = ROWS ? GL : 32;      // TEAM lanes share a row
    constexpr int RA_STAGES = ra_stages(ROWS);
    __shared__ RopeShared<ROWS> sh;
    const sv_rope_append_params &p = a.p;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = lane % GL, group = lane / GL, slot_h = ROWS ? 0 : group;
    const unsigned first_row = (blockIdx.x * RA_WARPS + warp) * ROWS_WARP;
    if (first_row >= (unsigned)p.n_rows) return;
    const unsigned row = ROWS ? min(first_row + group, (unsigned)p.n_rows - 1) : first_row;      // the last row again where there is none
    const int k_first = a.q_rounds, v_first = a.q_rounds + a.k_rounds;         // first rounds of keys and of values
    const int t_begin = blockIdx.y * a.rounds, t_end = min(t_begin + a.rounds, v_first + a.k_rounds);
    // Loads that nothing waits for come first: the slot, and what belongs to this lane's frequencies.
    const long long slot = p.slot_map[row];
    const bool turning = t_begin < v_first && p.rot_dim > 0;
    constexpr int FREQS = (ROWS ? 8 * GL : RA_MAX_FREQ) / TEAM;         // of a lane
    double freq[FREQS];
    int pos[FREQS];
#pragma unroll
    for (int i = 0; i < FREQS; ++i) {
        const int f = lane % TEAM + TEAM * i;
        freq[i] = 0.0;
        pos[i] = 0;
        if (!turning || f >= p.rot_dim / 2) continue;
        freq[i] = p.inv_freq[f];
        const int axis = p.freq_axis != nullptr ? min((int)p.freq_axis[f], p.n_axes - 1) : 0;
        pos[i] = p.positions[axis * p.n_rows + row];
    }
    // This lane's chunks, neighbouring lanes at neighbouring ones.  Where the pairs are (f, f + rot/2), the first rot/16 lanes
    // hold the turned dims; pairs (2f, 2f + 1) lie within a chunk.
    const int pair_lanes = PAIRED ? a.lanes : p.rot_dim / 16;
    bool live = j < a.lanes && (!ROWS || first_row + group < (unsigned)p.n_rows);
    const bool low = j < pair_lanes;
    const int c0 = low ? j : pair_lanes + j, c1 = low ? j + pair_lanes : a.lanes + j;
    const bool turn0 = c0 < p.rot_dim / 8, turn1 = c1 < p.rot_dim / 8;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(&sh.ring[warp][0][0][lane]);
    float2 *turns = sh.turns[warp] + (ROWS ? group * 8 * GL : 0);
    // where a frequency's turn lies: lanes read every fourth pair of them, which without the exclusive or would be in the same banks
    auto turn_at = [&](int f) { return f ^ (f >> 4 & 3) << 1 ^ (ROWS ? (group & 1) << 2 : 0); };
    // ---- producer: the rounds in order, RA_STAGES - 1 of them under way (from before the row's slot is known)
    int p_t = t_begin, p_stage = 0;
    auto issue = [&]() {
        if (p_t < t_end) {
            const bool q = p_t < k_first, v = p_t >= v_first;
            const int h = (p_t - (q ? 0 : v ? v_first : k_first)) * HEADS + slot_h;
            if (live && h < (q ? p.hq : a.hkv)) {
                const uint4 *src = static_cast<const uint4 *>(q ? p.q : v ? p.v_new : p.k_new) +
                                   (long long)row * (q ? a.q_stride : v ? a.v_stride : a.k_stride) + h * (2 * a.lanes);
                cp_chunk(ring + p_stage * 1024, src + c0);
                cp_chunk(ring + p_stage * 1024 + 512, src + c1);
            }
            ++p_t;
        }
        p_stage = p_stage + 1 == RA_STAGES ? 0 : p_stage + 1;
        cp_commit();                                   // an empty group where nothing is left
    };
#pragma unroll
    for (int s = 0; s < RA_STAGES - 1; ++s) issue();
    const bool placed = slot >= 0 && slot < a.n_slots;
    if (slot >= a.n_slots && lane % TEAM == 0) set_status(p.device_status, SV_DEV_BAD_PAGE);
    if (ROWS) live = live && placed;
    if (ROWS ? !__any_sync(0xffffffffu, placed) : !placed) {
        cp_wait<0>();
        return;
    }
    // ---- angles
    if (turning) {
#pragma unroll
        for (int i = 0; i < FREQS; ++i) {
            const int f = lane % TEAM + TEAM * i;
            if (f >= p.rot_dim / 2) continue;
            const int t = (int)(turn_step(freq[i]) * (unsigned long long)(long long)pos[i] >> 32);     // [-1/2, 1/2) turns, in units of 2^-32
            float s, c;
            sincospif((float)t * 4.656612873077393e-10f, &s, &c);                                      // 2^-31: half turns
            turns[turn_at(f)] = make_float2(c * p.rope_scale, s * p.rope_scale);
        }
        __syncwarp();
    }
    // ---- consumer
    int stage = 0;
    const long long cache = (long long)((unsigned long long)slot / RA_PAGE) * a.stride_page + (int)(slot & (RA_PAGE - 1)) * a.stride_slot;
    // queries, then keys
    for (int kind = 0; kind < 2; ++kind) {
        const int first_t = kind == 0 ? 0 : k_first, t0 = max(t_begin, first_t), t1 = min(t_end, kind == 0 ? k_first : v_first);
        if (t0 >= t1) continue;
        const int n_heads = kind == 0 ? p.hq : a.hkv;
        int h = (t0 - first_t) * HEADS + slot_h;
        const long long dst_head = kind == 0 ? 2 * a.lanes : a.stride_head;
        uint4 *dst = (kind == 0 ? static_cast<uint4 *>(p.q_out) + (long long)row * a.q_chunks : a.k_pool + cache) + h * dst_head;
        const void *weight = kind == 0 ? p.q_weight : p.k_weight;
        // Factors of the row, weight and angle in one: with the pairs (a, b) in the two chunks,
        // z_a = r (x_a (w_a cos) + x_b (-w_b sin)) and z_b = r (x_b (w_b cos) + x_a (w_a sin)); with the pairs in a chunk
        // the same for its even and odd elements.  direct[] multiplies an element itself, across[] its partner.
        f32x2 direct0[4], direct1[4], across0[4], across1[4];
        {
            uint4 w0 = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), w1 = w0;      // ones
            if (!WF32 && weight != nullptr) {
                w0 = static_cast<const uint4 *>(weight)[live ? c0 : 0];
                w1 = static_cast<const uint4 *>(weight)[live ? c1 : 0];
            }
            const uint32_t m0[4] = {w0.x, w0.y, w0.z, w0.w}, m1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 wa = unpack2(m0[i]), wb = unpack2(m1[i]);
                if (WF32 && weight != nullptr && live) {
                    const float2 fa = static_cast<const float2 *>(weight)[4 * c0 + i], fb = static_cast<const float2 *>(weight)[4 * c1 + i];
                    wa = pair(fa.x, fa.y);
                    wb = pair(fb.x, fb.y);
                }
                direct0[i] = wa;
                direct1[i] = wb;
                if (PAIRED) {
                    const float2 ta = turns[turn0 ? turn_at(4 * c0 + i) : 0], tb = turns[turn1 ? turn_at(4 * c1 + i) : 0];
                    const float2 xa = split(wa), xb = split(wb);
                    if (turn0) direct0[i] = mul2(wa, pair(ta.x, ta.x));
                    if (turn1) direct1[i] = mul2(wb, pair(tb.x, tb.x));
                    across0[i] = mul2(pair(xa.y, xa.x), pair(-ta.y, ta.y));
                    across1[i] = mul2(pair(xb.y, xb.x), pair(-tb.y, tb.y));
                } else {
                    const float4 cs = reinterpret_cast<const float4 *>(turns)[turn0 ? turn_at(8 * j + 2 * i) / 2 : 0];
                    if (turn0) {
                        direct0[i] = mul2(wa, pair(cs.x, cs.z));
                        direct1[i] = mul2(wb, pair(cs.x, cs.z));
                    }
                    across0[i] = mul2(wb, pair(-cs.y, -cs.w));
                    across1[i] = mul2(wa, pair(cs.y, cs.w));
                }
            }
        }
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            cp_wait<RA_STAGES - 2>();
            const uint4 v0 = sh.ring[warp][stage][0][lane], v1 = sh.ring[warp][stage][1][lane];
            stage = stage + 1 == RA_STAGES ? 0 : stage + 1;
            const uint32_t b0[4] = {v0.x, v0.y, v0.z, v0.w}, b1[4] = {v1.x, v1.y, v1.z, v1.w};
            f32x2 x0[4], x1[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x0[i] = unpack2(b0[i]);
                x1[i] = unpack2(b1[i]);
            }
            issue();
            const bool here = live && h < n_heads;
            float r = 1.f;
            if (weight != nullptr) {
                f32x2 s0 = mul2(x0[0], x0[0]), s1 = mul2(x1[0], x1[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) {
                    s0 = fma2(x0[i], x0[i], s0);
                    s1 = fma2(x1[i], x1[i], s1);
                }
                float ss = here ? (split(s0).x + split(s0).y) + (split(s1).x + split(s1).y) : 0.f;
#pragma unroll
                for (int m = GL / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                r = rsqrtf(ss * a.inv_dim + p.eps);
            }
            const f32x2 rr = pair(r, r);
            uint32_t z0[4], z1[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 y0 = mul2(x0[i], direct0[i]), y1 = mul2(x1[i], direct1[i]);
                if (PAIRED) {
                    if (turn0) y0 = fma2(pair(split(x0[i]).y, split(x0[i]).x), across0[i], y0);
                    if (turn1) y1 = fma2(pair(split(x1[i]).y, split(x1[i]).x), across1[i], y1);
                } else if (turn0) {                // both chunks or none
                    y0 = fma2(x1[i], across0[i], y0);
                    y1 = fma2(x0[i], across1[i], y1);
                }
                z0[i] = pack2(mul2(y0, rr));
                z1[i] = pack2(mul2(y1, rr));
            }
            if (here) {
                dst[c0] = make_uint4(z0[0], z0[1], z0[2], z0[3]);
                dst[c1] = make_uint4(z1[0], z1[1], z1[2], z1[3]);
            }
            h += HEADS;
            dst += HEADS * dst_head;
        }
    }
    // values
    for (int t = max(t_begin, v_first); t < t_end; ++t) {
        cp_wait<RA_STAGES - 2>();
        const uint4 v0 = sh.ring[warp][stage][0][lane], v1 = sh.ring[warp][stage][1][lane];
        stage = stage + 1 == RA_STAGES ? 0 : stage + 1;
        const int h = (t - v_first) * HEADS + slot_h;
        if (live && h < a.hkv) {
            uint4 *dst = a.v_pool + cache + h * a.stride_head;
            dst[c0] = v0;
            dst[c1] = v1;
        }
        issue();
    }
}

// How many warps share a row's rounds (or several rows'): the fewest waves of resident warps, each as long as a warp's rounds and
// the `before` rounds' worth of what precedes them.  warps: without sharing; heads: of a row in a round.
static long long best_split(RopeAppendLaunch &a, long long warps, int heads, int before)
{
    a.q_rounds = (a.p.hq + heads - 1) / heads;
    a.k_rounds = (a.hkv + heads - 1) / heads;
    const int all = a.q_rounds + 2 * a.k_rounds;
    const long long resident = (long long)sm_count() * RA_BLOCKS_PER_SM * RA_WARPS;
    long long best = -1;
    for (int segments = 1; segments <= all; ++segments) {
        const int rounds = (all + segments - 1) / segments;
        const long long cost = (warps * segments + resident - 1) / resident * (rounds + before);
        if (best >= 0 && cost >= best) continue;
        best = cost;
        a.rounds = rounds;
        a.segments = (all + rounds - 1) / rounds;
    }
    return best;
}

template <int GL, bool PAIRED, bool WF32>
static sv_status launch_rope(RopeAppendLaunch &a, cudaStream_t stream)
{
    constexpr int share = 32 / GL;
    const long long sets = (a.p.n_rows + share - 1) / share;
    RopeAppendLaunch rows = a;
    const long long one = best_split(a, a.p.n_rows, share, RA_BEFORE);
    // rows that do not fill the GPU by themselves are not put together either
    if (a.q_rounds + 2 * a.k_rounds <= RA_FEW_ROUNDS && a.p.n_rows > (long long)sm_count() * RA_BLOCKS_PER_SM * RA_WARPS &&
        best_split(rows, sets, 1, RA_BEFORE_ROWS) < one) {
        const dim3 grid((unsigned)((sets + RA_WARPS - 1) / RA_WARPS), (unsigned)rows.segments);
        return launch_kernel(true, rope_append_kernel<GL, PAIRED, WF32, true>, grid, RA_THREADS, 0, stream, rows);
    }
    const dim3 grid((unsigned)((a.p.n_rows + RA_WARPS - 1) / RA_WARPS), (unsigned)a.segments);
    return launch_kernel(true, rope_append_kernel<GL, PAIRED, WF32, false>, grid, RA_THREADS, 0, stream, a);
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
    if (p->n_rows > 1 << 30) return SV_EUNSUPPORTED;       // rows are counted in 32 bits, with room for a step
    if (p->hq > RA_MAX_HEADS || pool.hkv > RA_MAX_HEADS) return SV_EUNSUPPORTED;
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
    a.q_stride = p->q_stride / 8;
    a.k_stride = p->k_stride / 8;
    a.v_stride = p->v_stride / 8;
    a.q_chunks = p->hq * (pool.head_dim / 8);
    a.lanes = pool.head_dim / 16;
    a.inv_dim = 1.f / (float)pool.head_dim;
    cudaStream_t s = (cudaStream_t)stream;
    const int kind = (a.lanes <= 4 ? 0 : 4) + (p->interleaved != 0 ? 2 : 0) + (p->weights_f32 != 0 ? 1 : 0);
    switch (kind) {
        case 0: return launch_rope<4, false, false>(a, s);
        case 1: return launch_rope<4, false, true>(a, s);
        case 2: return launch_rope<4, true, false>(a, s);
        case 3: return launch_rope<4, true, true>(a, s);
        case 4: return launch_rope<8, false, false>(a, s);
        case 5: return launch_rope<8, false, true>(a, s);
        case 6: return launch_rope<8, true, false>(a, s);
        default: return launch_rope<8, true, true>(a, s);
    }
}
