// The ring of tiles that the copying warps of the chunk attention fill: which copies may still be on their way.
#pragma once

#ifdef __CUDACC__
#define LIBRA_HD __host__ __device__ __forceinline__
#else
#define LIBRA_HD inline
#endif

namespace libra {

constexpr int kChunkLoaders = 3;   // warps that take the ring's tiles by turns: tile i is warp i % kChunkLoaders'

// The newest tile of the warp whose next one would be `next`, and the one before a tile; negative: none.
LIBRA_HD int ring_newest(int next) { return next - kChunkLoaders; }
LIBRA_HD int ring_before(int tile) { return tile - kChunkLoaders; }
// Whether `tile` may be on its way yet.  The newest one was asked for after its place had been used before, that is after tile
// newest - n_stages and, tiles being used in order, every older one had arrived.
LIBRA_HD bool ring_may_fly(int tile, int next, int n_stages) { return tile >= 0 && tile > ring_newest(next) - n_stages; }

}  // namespace libra
