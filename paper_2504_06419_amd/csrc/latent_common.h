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

#include "spire_internal.h"

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

}  // namespace spire
