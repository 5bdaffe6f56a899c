// Host-side launchers of the paged cache's kernels.  All of them are asynchronous
// on `stream` and assume the arguments were validated by the C-ABI layer.
#pragma once

#include <algorithm>

#include "cache.cuh"
#include "chunk.cuh"
#include "rope.cuh"

namespace tgvkv {

// cache_rows.cu: quantising writes and reads of whole rows.
// Exactly one of row_offsets (CSR rows: [S + 1]) and tok_offsets (tokens x
// heads: [B + 1], element strides k token, k head, v token, v head) is given;
// rows: rows that k and v hold.
cudaError_t launch_cache_write(const CacheProblem& p, const CachePools& pool, const uint16_t* k,
                               const uint16_t* v, const long long (&strides)[4], long long rows,
                               const int64_t* row_offsets, const int32_t* tok_offsets,
                               const int32_t* page_table, const int32_t* lens, int32_t* lens_out,
                               uint32_t* status, cudaStream_t stream);
cudaError_t launch_cache_read(const CacheProblem& p, const CachePools& pool,
                              const int32_t* page_table, const int32_t* first,
                              const int64_t* offsets, uint16_t* k_out, uint16_t* v_out,
                              long long rows, uint32_t* status, cudaStream_t stream);

// pages.cu: a page list's takings and givings back (mode), with the slots of new tokens
// (kPagesAppend), and the slots alone.  ticket: zero at the start and left zero.
enum { kPagesGrow, kPagesShrink, kPagesAppend };
struct PagesArgs {
    int32_t *table, *free_pages, *n_free;
    const int32_t *lens, *lens_new, *tok_offsets;
    int T;
    int32_t *slots, *lens_out;
    int granule_shift;                 // set by the launcher
};
cudaError_t launch_pages(const CacheProblem& p, int mode, const PagesArgs& a, uint32_t* ticket,
                         uint32_t* status, cudaStream_t stream);
cudaError_t launch_page_slots(const CacheProblem& p, const PagesArgs& a, uint32_t* status,
                              cudaStream_t stream);
cudaError_t launch_pages_init(const CacheProblem& p, const PagesArgs& a, cudaStream_t stream);

// rope.cu: rows turned by their positions, and turned into the paged cache (strides: k
// token, k head, v token, v head).
cudaError_t launch_rope(const tgvkv_rope_plan& plan, int mode, const int32_t* positions,
                        long long pos_stride, int T, const RopeTensor& q, const RopeTensor& k,
                        cudaStream_t stream);
cudaError_t launch_rope_write(const CacheProblem& p, const CachePools& pool,
                              const tgvkv_rope_plan& plan, const int32_t* positions,
                              long long pos_stride, const int32_t* slots, int T, const RopeTensor& q,
                              const uint16_t* k, const uint16_t* v, const long long (&strides)[4],
                              uint32_t* status, cudaStream_t stream);

// Attention of a chunk of new tokens: the row-stream kernel, for sets of at most
// stream_rows() query rows (max_q * G; chunk_stream.cu), and the tile kernel for
// larger ones, `pair`: two row tiles an item (chunk_tile.cuh), with its merge
// (chunk_merge.cu).  plan: S + 1 entries; split: one per CTA; sync: kTileSync words,
// zero at the start and left zero; part: the split sets' records.
cudaError_t launch_chunk_stream(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                                float* part, long long* plan, uint32_t* status,
                                cudaStream_t stream);
cudaError_t launch_tile_bf16(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream);
cudaError_t launch_tile_int8(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream);
cudaError_t launch_tile_int4(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream);
cudaError_t launch_tile_fp4(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                             float* part, SplitItem* split, uint32_t* sync, bool pair,
                             uint32_t* status, cudaStream_t stream);
cudaError_t launch_tile_merge(const CacheProblem& p, const ChunkArgs& a, const TilePlan& pl, int ctas,
                              const float* part, const SplitItem* split, cudaStream_t stream);

}  // namespace tgvkv
