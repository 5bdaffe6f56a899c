// Joins the partial results that the tile kernel (chunk_tile.cuh) leaves for items
// that span several CTAs, in CTA order (so results do not depend on timing),
// and writes 0 for the rows that see no slot.  One warp per output row; most
// rows of a large call were written by the tile kernel and return at once.  A
// programmatic dependent of that kernel: the search for a row's item reads
// inputs only and overlaps it.
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

template <int D>
__global__ void __launch_bounds__(128)
chunk_tile_merge(const CacheProblem p, const ChunkArgs a, const TilePlan pl, int ctas,
                 const float* __restrict__ part, const long long* __restrict__ plan) {
    constexpr int DPL = D / 32;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int t = (int)(row / p.H_q), head = (int)(row - (long long)t * p.H_q);
    int lo = 0, hi = p.B - 1;          // the last sequence that starts at or before t
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(a.tok_offsets + mid) <= t) lo = mid;
        else hi = mid - 1;
    }
    const int s = lo * p.H_kv + head / p.G;
    const SetSpan sp = set_span(p, a, s);
    const int i = t - sp.tok0;
    const bool mine = t < a.T && i >= 0 && i < sp.n;
    const int u = mine ? i / pl.tpi : 0;
    const int nk = mine ? tiles_seen(sp, (u + 1) * pl.tpi) : 0;
    long long before = 0;              // units of the set's earlier items
    for (int x = lane; x < u; x += 32) before += tiles_seen(sp, (x + 1) * pl.tpi);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) before += __shfl_xor_sync(~0u, before, k);
    griddep_wait();
    if (!mine) return;
    float acc[DPL];
#pragma unroll
    for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
    if (nk > 0) {
        const long long total = __ldcg(plan + p.S), c0 = __ldcg(plan + s) + before;
        const long long per = (total + ctas - 1) / ctas;
        const int w0 = (int)(c0 / per), w1 = (int)((c0 + nk - 1) / per);
        if (w0 == w1) return;          // inside one CTA: written by it
        const int first = c0 != w0 * per ? 1 : 0;
        const int tiles = pl.tpi / pl.tpt, w = (i - u * pl.tpi) / pl.tpt;
        const int r = (i - u * pl.tpi - w * pl.tpt) * p.G + head % p.G;
        const size_t rec = chunk_record_floats(pl.rows, D);
        merge_records<D, 1>(w1 - w0 + 1, pl.rows, r, [&](int x) {
            return part + ((size_t)((w0 + x) * 2 + (x == 0 ? first : 0)) * tiles + w) * rec;
        }, acc, nullptr, 0);
    }
    uint16_t* out = a.out + row * D + DPL * lane;
#pragma unroll
    for (int c = 0; c < DPL; c += 2)
        *reinterpret_cast<uint32_t*>(out + c) = pack_bf16x2(acc[c], acc[(c + 1) % DPL]);
}

}  // namespace

cudaError_t launch_tile_merge(const CacheProblem& p, const ChunkArgs& a, const TilePlan& pl, int ctas,
                              const float* part, const long long* plan, cudaStream_t stream) {
    const long long rows = (long long)a.T * p.H_q;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (p.d == 64)
        return launch_dependent(chunk_tile_merge<64>, grid, dim3(128), 0, stream, p, a, pl, ctas, part,
                                plan);
    return launch_dependent(chunk_tile_merge<128>, grid, dim3(128), 0, stream, p, a, pl, ctas, part,
                            plan);
}

}  // namespace tgvkv
