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

// By the whole block of NT threads, with a barrier at the end.  owner(o, report): the work of owner o (report: first look).
// red: two rows of shared scratch.
template <int NT, typename Owner>
__device__ __forceinline__ void plan_work_share(int n_owners, int pair_cost, Owner &&owner, WorkShare *sh, long long (*red)[NT / 32])
{
    constexpr int NW = NT / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    OwnerWork w = {0, 0};
    const bool one = n_owners <= NT;
    long long cost = 0, tiles = 0;
    for (int o = tid; o < n_owners; o += NT) {
        w = owner(o, true);
        tiles += (long long)w.n_sub * w.n_tiles;
        cost += w.n_tiles > 0 ? (long long)w.n_sub * (w.n_tiles + pair_cost) : 0;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        cost += __shfl_xor_sync(0xffffffffu, cost, d);
        tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
    }
    if (lane == 0) { red[0][warp] = cost; red[1][warp] = tiles; }
    __syncthreads();
    long long cost_all = 0, tiles_all = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) { cost_all += red[0][i]; tiles_all += red[1][i]; }
    const long long xb = blockIdx.x * cost_all / gridDim.x, xe = (blockIdx.x + 1LL) * cost_all / gridDim.x;
    if (tid == 0) {
        sh->t_begin = sh->t_end = sh->total = tiles_all;
        sh->o = n_owners; sh->s = sh->t = 0;
    }
    __syncthreads();
    long long cost0 = 0, tiles0 = 0;
    for (int base = 0; base < n_owners; base += NT) {
        const int o = base + tid;
        if (!one) {
            w.n_sub = w.n_tiles = 0;
            if (o < n_owners) w = owner(o, false);
        }
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
            if (i < warp) { bc += red[0][i]; bt += red[1][i]; }
            cost0 += red[0][i]; tiles0 += red[1][i];
        }
        const long long lo = bc + vc - w_cost, hi = bc + vc;
        const long long tile_lo = bt + vt - w_tiles;
        if (w_cost > 0) {
            const int per = w.n_tiles + pair_cost;
            if (lo <= xb && xb < hi) {
                const long long j = (xb - lo) / per, off = min(xb - lo - j * per, (long long)w.n_tiles);
                sh->t_begin = tile_lo + j * w.n_tiles + off;
                sh->o = o; sh->s = (int)j; sh->t = (int)off;
            }
            if (lo <= xe && xe < hi) {
                const long long j = (xe - lo) / per, off = min(xe - lo - j * per, (long long)w.n_tiles);
                sh->t_end = tile_lo + j * w.n_tiles + off;
            }
        }
        __syncthreads();
    }
}

}  // namespace sv
