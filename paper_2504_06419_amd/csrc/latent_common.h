// latent_common.h -- what the kernels of attention over a latent cache share.
//
// Rows of one sequence are its (k+1) * Hq queries.  They are cut into blocks of
// 16 that never mix query tokens (block rb: token rb / hb, heads 16 (rb % hb) ..),
// so a block's rows all see the same keys and a key hidden from the block is
// cleared as a whole: whatever it holds cannot reach them.  nb blocks make a
// unit, one workgroup's rows.
//
// Keys are cut into tiles and shared out in the stream-K manner of
// spire_internal.h with one segment per sequence: group g of `units` workgroups
// takes positions [g T / groups, (g+1) T / groups), every workgroup of a group the
// same keys for another unit of rows, so the rows of a tile are read from HBM
// once and then from the caches.  Segments that several groups share leave
// partials (normalised rows, base-2 log-sum-exp) that latent_combine merges.
#pragma once

#include "mfma_common.h"

namespace spire {

// Workgroup -> (group, unit).  Workgroups that follow each other go to different
// XCDs (blockIdx % 8), each with an L2 of its own; neighbours in `lin` share one,
// so a group's workgroups read their common keys through one L2.
__device__ __forceinline__ void latent_place(const Latent &a, int &g, int &u) {
    const int n = gridDim.x, x = blockIdx.x;
    const int lin = (n & 7) == 0 ? (x & 7) * (n >> 3) + (x >> 3) : x;
    g = lin / a.units;
    u = lin - g * a.units;
}

// Where group g starts and its positions: every workgroup forms the partition itself
// (a launch of its own took 7 us), in LDS that is free again afterwards; the merge
// finds the prefix sums and starts in the workspace.  False: nothing to do.
template <int THREADS>
__device__ __forceinline__ bool latent_start(const Latent &a, int g, int u, int32_t *lds, int &seg, int &tile,
                                             int64_t &pos, int64_t &end) {
    plan_in_kernel<THREADS>(a.p, a.pl, lds, lds + a.p.B + 1);
    bool some = false;
    if (g < a.pl.workers) {
        const int64_t T = __builtin_amdgcn_readfirstlane(lds[a.p.B]);
        pos = worker_begin(g, T, a.pl.workers);
        end = worker_begin(g + 1, T, a.pl.workers);
        some = pos < end;
        if (some) locate(lds, a.p.B, 1, pos, seg, tile);
        if (u == 0 && threadIdx.x == 0) {
            a.pl.wstart[2 * g] = some ? seg : -1;
            a.pl.wstart[2 * g + 1] = some ? tile : 0;
        }
    }
    seg = __builtin_amdgcn_readfirstlane(seg);
    tile = __builtin_amdgcn_readfirstlane(tile);
    __syncthreads();
    return some;
}

// Tiles of a sequence of n keys: without keys one, empty, so that its rows are written.
template <int TILE>
__device__ __forceinline__ int latent_tiles(int n) { return n > 0 ? (n + TILE - 1) / TILE : 1; }

}  // namespace spire
