// What the two chunk-attention kernels share: a call's arguments, the spans of
// its sets, and the records of split results that chunk_merge.cu joins.
#pragma once

#include <cuda.h>

#include "cache.cuh"

namespace tgvkv {

struct ChunkArgs {
    const uint16_t* q;           // [T][H_q][d] with strides
    long long q_tok, q_head;     // element strides
    const int32_t* tok_offsets;  // [B + 1]
    int T;                       // tokens q and out hold
    int max_q;                   // most new tokens of a sequence
    const int32_t* page_table;   // [S][max_pages]
    const int32_t* lens;         // [S], the new tokens included
    uint16_t* out;               // [T][H_q][d]
};

// Set s: its slots, its sequence's new tokens and the first of them.
struct SetSpan {
    int len, n, tok0;
};

__device__ __forceinline__ SetSpan set_span(const CacheProblem& p, const ChunkArgs& a, int s) {
    SetSpan r;
    const int b = s / p.H_kv;
    const int lo = __ldg(a.tok_offsets + b), hi = __ldg(a.tok_offsets + b + 1);
    r.len = clamp_len(__ldg(a.lens + s), p.cap);
    r.tok0 = min(max(lo, 0), a.T);
    r.n = min(min(max(hi, r.tok0), a.T) - r.tok0, a.max_q);
    return r;
}

// The caller's lengths and offsets, checked once (by one CTA): what set_span
// clips is reported here.
__device__ __forceinline__ void check_spans(const CacheProblem& p, const ChunkArgs& a, int tid,
                                            int threads, uint32_t* status) {
    for (int s = tid; s < p.S; s += threads) {
        const int b = s / p.H_kv;
        const int lo = a.tok_offsets[b], hi = a.tok_offsets[b + 1], len = a.lens[s];
        if (lo < 0 || hi < lo || hi > a.T || hi - lo > a.max_q || len < 0 || len > p.cap)
            raise_status(status, TGVKV_STATUS_INDEX);
    }
}

// Split results: every stream of work leaves at most two (the segment that
// starts its share and the one that ends it).  A record holds O [rows][d],
// then m [rows] and l [rows].
__host__ __device__ inline int chunk_record_floats(int rows, int d) {
    return rows * d + ((2 * rows + 3) & ~3);
}

constexpr int kStreamMax = 2048;       // streams of the row-stream kernel
constexpr int kStreamRows = 16;        // query rows it takes a set

// Two floats as bf16x2, `lo` in the low half.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// Host: a map of the pool's rows (row_bytes each) in boxes of box_rows rows of
// box_bytes bytes, swizzled over the box's rows; and of the queries,
// [token][head][d] with strides, in boxes of 64 dims x heads x tokens.
bool make_pool_map(CUtensorMap* map, const void* base, uint64_t rows, int row_bytes, int box_bytes,
                   uint32_t box_rows);
bool make_query_map(CUtensorMap* map, const CacheProblem& p, const ChunkArgs& a,
                    uint32_t box_heads, uint32_t box_tokens);

}  // namespace tgvkv
