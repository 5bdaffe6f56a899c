// The tile kernel of chunk_tile.cuh over caches of 4-bit floats.  Chunks of 0 .. 500 tokens of
// 16 x 4 sets of 4451 .. 8900 slots, 28 heads of 128: 368 us (int4 356, int8 366), bound as
// over int8 by a key tile's way from copy over conversion to product.
#include "chunk_tile.cuh"

namespace tgvkv {

cudaError_t launch_tile_fp4(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream) {
    constexpr int F = TGVKV_CACHE_FP4;
    if (p.d == 64)
        return pair ? launch_tile<64, F, true>(p, pool, a, part, split, sync, status, stream)
                    : launch_tile<64, F, false>(p, pool, a, part, split, sync, status, stream);
    return pair ? launch_tile<128, F, true>(p, pool, a, part, split, sync, status, stream)
                : launch_tile<128, F, false>(p, pool, a, part, split, sync, status, stream);
}

}  // namespace tgvkv
