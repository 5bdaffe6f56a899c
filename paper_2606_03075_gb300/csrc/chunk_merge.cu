// Joins the partial results that the tile kernel (chunk_tile.cuh) leaves for items
// that span many CTAs, in CTA order (so results do not depend on timing).  The CTA
// of that kernel in which such an item begins names it; the merge's CTA (x, y)
// takes `rows` rows from rows * x on of the y-th item named, a warp each, or all 8
// warps row after row when it has many records.  A programmatic dependent of the tile
// kernel; latency-bound (three dependent reads of L2), a few microseconds.
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

constexpr int kManyRecords = 32;       // from here on, 8 warps a row

template <int D>
__global__ void __launch_bounds__(256)
chunk_tile_merge(const CacheProblem p, const ChunkArgs a, const TilePlan pl, int ctas, int per_cta,
                 const float* __restrict__ part, const SplitItem* __restrict__ split) {
    constexpr int DPL = D / 32;
    __shared__ float shared[8 * (D + 2)];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ int found[4], count[8];
    griddep_launch_dependents();       // the next call's set-up may overlap
    griddep_wait();
    // the y-th of the items named: threads 0 .. ctas - 1 hold one CTA's word each
    int4 raw = make_int4(-1, 0, 0, 0);
    if (threadIdx.x < ctas) raw = __ldcg(reinterpret_cast<const int4*>(split) + threadIdx.x);
    // a CTA without a share leaves its word as it was: nothing out of range is taken
    if (raw.x >= p.S || raw.y < 0 || (long long)raw.y * pl.tpi > a.max_q || raw.z < 1 ||
        raw.z > ctas - (int)threadIdx.x || (raw.w & ~1))
        raw.x = -1;
    const uint32_t named = __ballot_sync(~0u, raw.x >= 0);
    if (lane == 0) count[warp] = __popc(named);
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    int rank = __popc(named & ((1u << lane) - 1u));
    for (int x = 0; x < warp; ++x) rank += count[x];
    if (raw.x >= 0 && rank == blockIdx.y)
        found[0] = threadIdx.x, found[1] = raw.x, found[2] = raw.y, found[3] = raw.z | (raw.w << 16);
    __syncthreads();
    const int start = found[0];        // the CTA in which it begins
    if (start < 0) return;
    const SplitItem it{found[1], found[2], found[3] & 0xFFFF, found[3] >> 16};
    const SetSpan sp = set_span(p, a, it.s);
    const int tok0 = it.u * pl.tpi;    // the item's first token within its chunk
    const int rows = min(pl.tpi, sp.n - tok0) * p.G;
    const int tiles = pl.tpi / pl.tpt;
    const size_t rec = chunk_record_floats(pl.rows, D);
    const bool many = it.ctas >= kManyRecords;
    for (int k = many ? 0 : warp; k < per_cta; k += many ? 1 : 8) {
        const int row = blockIdx.x * per_cta + k;         // row of the item
        if (row >= rows) break;
        const int w = row / pl.rows, r = row - w * pl.rows;  // its tile, and row there
        const int t = tok0 + row / p.G, head = (it.s % p.H_kv) * p.G + row % p.G;
        float acc[DPL];
        auto record = [&](int x) {
            return part + (((size_t)start + x) * 2 * tiles + (x == 0 ? it.slot : 0) * tiles + w) * rec;
        };
        if (many) {
            merge_records<D, 8, true>(it.ctas, pl.rows, r, record, acc, shared, warp);
            __syncthreads();           // shared is free for the next row
            if (warp != 0) continue;
        } else {
            merge_records<D, 1, true>(it.ctas, pl.rows, r, record, acc, nullptr, 0);
        }
        uint16_t* out = a.out + ((size_t)(sp.tok0 + t) * p.H_q + head) * D + DPL * lane;
#pragma unroll
        for (int c = 0; c < DPL; c += 2)
            *reinterpret_cast<uint32_t*>(out + c) = pack_bf16x2(acc[c], acc[(c + 1) % DPL]);
    }
}

}  // namespace

cudaError_t launch_tile_merge(const CacheProblem& p, const ChunkArgs& a, const TilePlan& pl, int ctas,
                              const float* part, const SplitItem* split, cudaStream_t stream) {
    const int rows = (a.max_q < pl.tpi ? a.max_q : pl.tpi) * p.G;          // of an item, at most
    // such items begin at least kJoin + 1 CTAs apart
    const long long all = (long long)p.S * ((a.max_q + pl.tpi - 1) / pl.tpi);
    const int items = (int)(all < ctas / (kJoin + 1) + 1 ? all : ctas / (kJoin + 1) + 1);
    // A row a CTA while one wave holds them, 8 at most: 2 sets of 33 rows, each over half
    // the GPU, take 27 us instead of 66 with 8.
    int per_cta = (items * rows + 8 * ctas - 1) / (8 * ctas);
    if (per_cta > 8) per_cta = 8;
    const dim3 grid((unsigned)((rows + per_cta - 1) / per_cta), (unsigned)items);
    if (p.d == 64)
        return launch_dependent(chunk_tile_merge<64>, grid, dim3(256), 0, stream, p, a, pl, ctas,
                                per_cta, part, split);
    return launch_dependent(chunk_tile_merge<128>, grid, dim3(256), 0, stream, p, a, pl, ctas,
                                per_cta, part, split);
}

}  // namespace tgvkv
