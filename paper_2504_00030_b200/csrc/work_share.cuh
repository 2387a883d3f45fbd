// Shares of a list of tiles for the blocks of a persistent kernel whose work is only known on the device.
//
// An owner has n_sub pairs of n_tiles tiles each; all tiles form one list, owner by owner and pair by pair.  Every block takes
// a contiguous part of it, equal in cost: a pair costs its tiles and pair_cost more (its own operands, its start and end).
// Every block finds its part by itself, from one look at each owner (two where there are more owners than threads).
#pragma once

#include "common.cuh"

namespace sv {

struct OwnerWork {
    int n_sub, n_tiles;
};

struct WorkShare {
    long long t_begin, t_end;    // the block's tiles
    long long total;             // tiles of the list
    int o, s, t;                 // owner, pair of the owner and tile of t_begin (t may be n_tiles: the next pair)
};

// a / b; nearly always in 32 bits (a 64-bit division is a hundred instructions, each fetched for this one use)
__device__ __forceinline__ long long share_div(long long a, int b)
{
    return (a >> 31) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// By the whole block of NT threads, with a barrier at the end.  owner(o, report): the work of owner o (report: first look);
// begins(): called by the thread whose last look was at the owner that t_begin lies in.
// red: two rows of shared scratch.  One scan over the owners where each thread has one of them; what it costs is paid by
// every launch: as a sum, a scan and 64-bit divisions, and a second look at the owner by every warp role, a token over 64 pages
// took 15.3 us in place of 14.6, a small prefix with its three launches 29.7 in place of 28.3.
template <int NT, typename Owner, typename Begins>
__device__ __forceinline__ void plan_work_share(int n_owners, int pair_cost, Owner &&owner, Begins &&begins, WorkShare *sh, long long (*red)[NT / 32])
{
    constexpr int NW = NT / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool one = n_owners <= NT;
    long long cost_all = 0, tiles_all = 0;
    if (!one) {
        long long cost = 0, tiles = 0;
        for (int o = tid; o < n_owners; o += NT) {
            const OwnerWork w = owner(o, true);
            tiles += (long long)w.n_sub * w.n_tiles;
            cost += w.n_tiles > 0 ? (long long)w.n_sub * (w.n_tiles + pair_cost) : 0;
        }
#pragma unroll 1
        for (int d = 16; d > 0; d >>= 1) {
            cost += __shfl_xor_sync(0xffffffffu, cost, d);
            tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
        }
        if (lane == 0) { red[0][warp] = cost; red[1][warp] = tiles; }
        __syncthreads();
        for (int i = 0; i < NW; ++i) { cost_all += red[0][i]; tiles_all += red[1][i]; }
        __syncthreads();
    }
    long long cost0 = 0, tiles0 = 0;           // of the owners in front of these NT
    for (int base = 0; base == 0 || base < n_owners; base += NT) {
        const int o = base + tid;
        OwnerWork w = {0, 0};
        if (o < n_owners) w = owner(o, one);
        const long long w_cost = w.n_tiles > 0 ? (long long)w.n_sub * (w.n_tiles + pair_cost) : 0;
        const long long w_tiles = (long long)w.n_sub * w.n_tiles;
        long long vc = w_cost, vt = w_tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, vc, d), y = __shfl_up_sync(0xffffffffu, vt, d);
            if (lane >= d) { vc += x; vt += y; }
        }
        if (lane == 31) { red[0][warp] = vc; red[1][warp] = vt; }
        __syncthreads();
        long long bc = cost0, bt = tiles0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const long long c = red[0][i], t = red[1][i];
            if (i < warp) { bc += c; bt += t; }
            cost0 += c; tiles0 += t;
        }
        if (one) { cost_all = cost0; tiles_all = tiles0; }
        // the block's part of the costs, [xb, xe); all owners' together are [0, cost_all)
        const long long xb = share_div(blockIdx.x * cost_all, (int)gridDim.x), xe = share_div((blockIdx.x + 1LL) * cost_all, (int)gridDim.x);
        if (tid == 0 && base == 0) {
            sh->total = tiles_all;
            if (cost_all == 0) { sh->t_begin = 0; sh->o = n_owners; sh->s = sh->t = 0; }
            if (xe == cost_all) sh->t_end = tiles_all;
        }
        const long long lo = bc + vc - w_cost, hi = bc + vc;
        const long long tile_lo = bt + vt - w_tiles;
        if (w_cost > 0) {
            const int per = w.n_tiles + pair_cost;
            if (lo <= xb && xb < hi) {
                const long long j = share_div(xb - lo, per), off = min(xb - lo - j * per, (long long)w.n_tiles);
                sh->t_begin = tile_lo + j * w.n_tiles + off;
                sh->o = o; sh->s = (int)j; sh->t = (int)off;
                begins();
            }
            if (lo <= xe && xe < hi) {
                const long long j = share_div(xe - lo, per), off = min(xe - lo - j * per, (long long)w.n_tiles);
                sh->t_end = tile_lo + j * w.n_tiles + off;
            }
        }
        __syncthreads();
    }
}

}  // namespace sv
