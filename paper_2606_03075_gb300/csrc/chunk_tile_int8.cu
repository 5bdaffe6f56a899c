// The tile kernel of chunk_tile.cuh over int8 caches.
#include "chunk_tile.cuh"

namespace tgvkv {

cudaError_t launch_tile_int8(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream) {
    constexpr int F = TGVKV_CACHE_INT8;
    if (p.d == 64)
        return pair ? launch_tile<64, F, true>(p, pool, a, part, split, sync, status, stream)
                    : launch_tile<64, F, false>(p, pool, a, part, split, sync, status, stream);
    return pair ? launch_tile<128, F, true>(p, pool, a, part, split, sync, status, stream)
                : launch_tile<128, F, false>(p, pool, a, part, split, sync, status, stream);
}

}  // namespace tgvkv
