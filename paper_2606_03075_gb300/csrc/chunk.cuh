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

// Set s: its sequence's new tokens and the first of them, and the slots up to the
// last of them.  Tokens past max_q or past q's end are left out, with the slots they
// stand for, so that the others see what they would have seen.
struct SetSpan {
    int len, n, tok0;
};

__device__ __forceinline__ SetSpan set_span(const CacheProblem& p, const ChunkArgs& a, int s) {
    SetSpan r;
    const int b = s / p.H_kv;
    const int lo = a.tok_offsets[b], hi = a.tok_offsets[b + 1];
    r.tok0 = min(max(lo, 0), a.T);
    const int all = max(hi, r.tok0) - r.tok0;
    r.n = min(min(all, a.T - r.tok0), a.max_q);
    r.len = max(clamp_len(a.lens[s], p.cap) - (all - r.n), 0);
    return r;
}

// The caller's lengths and offsets, checked once (by one CTA): what set_span
// clips is reported here.
__device__ __forceinline__ void check_spans(const CacheProblem& p, const ChunkArgs& a, int tid,
                                            int threads, uint32_t* status) {
    for (int s = tid; s < p.S; s += threads) {
        const int b = s / p.H_kv;
        const int lo = a.tok_offsets[b], hi = a.tok_offsets[b + 1], len = a.lens[s];
        if ((s == 0 && lo != 0) || lo < 0 || hi < lo || hi > a.T || hi - lo > a.max_q || len < 0 ||
            len > p.cap)
            raise_status(status, TGVKV_STATUS_INDEX);
    }
}

// Split results: every stream of work leaves at most two (the segment that
// starts its share and the one that ends it).  A record holds O [rows][d],
// then m [rows] and l [rows].
__host__ __device__ inline int chunk_record_floats(int rows, int d) {
    return rows * d + ((2 * rows + 3) & ~3);
}

constexpr int kStreamMaxCtas = 160;    // CTAs of the row-stream kernel
constexpr int kStreamRows = 32;        // query rows a set that it takes at most

// Query rows a set up to which the row-stream kernel takes a call.  Where it still has
// the registers it does without the tile kernel's 128-row tiles and the bf16 copy of
// integer codes: 256 sets of 20 rows over 2051 .. 4101 slots, tile kernel against it
// (us): d = 64 bf16 50 / 45, int8 62 / 45, int4 62 / 42 (32 rows 50 / 49, 62 / 54,
// 61 / 50); d = 128 bf16 75 / 78, int8 80 / 78, int4 82 / 60; 4-bit floats: d = 64 65 / 46
// (32 rows 64 / 55), d = 128 84 / 67.
__host__ __device__ constexpr int stream_rows(int d, int format) {
    return d == 64 ? kStreamRows : format == TGVKV_CACHE_BF16 ? 16 : 24;
}
constexpr int kTileMaxCtas = 160;      // CTAs of the tile kernel
constexpr int TM = 128;                // query rows of its row tiles
constexpr int TN = 128;                // slots of its key tiles

// The tile kernel's work.
struct TilePlan {
    int tpt;                           // tokens of a row tile
    int tpi;                           // tokens of an item: one row tile, or two
    int rows;                          // query rows of a record: tpt * G at most
};

// Later parts of an item that the CTA of its start joins; an item of more goes to the
// second kernel.  One sequence's 32 sets of 96 tokens over 8001 .. 16000 slots (int8): 52 us
// at 2, 59 at 3 (its warps read the parts one after another); 600 tokens of 28 heads
// over 20000 slots: 132 at 2, 141 at 1; 0 .. 500 tokens of 16 sequences 359 at 2, 397 at 0.
constexpr int kJoin = 2;
// words of the tile kernel's tickets and flags: two tickets, then 8 flags per CTA
constexpr int kTileFlags = 8;
constexpr int kTileSync = kTileFlags + 8 * kTileMaxCtas;

// The CTA's share of the work, the last for the first CTA that starts.  A workspace
// that was not at zero gives shares that do not exist: none is taken then.
__device__ __forceinline__ int take_share(uint32_t* ticket, uint32_t* status) {
    const uint32_t t = atomicAdd(ticket, 1u);
    if (t < gridDim.x) return (int)(gridDim.x - 1 - t);
    raise_status(status, TGVKV_STATUS_TIMEOUT);
    return (int)gridDim.x;
}

// What a CTA of the tile kernel leaves for the merge: the item that begins in it
// and spans more than kJoin + 1 CTAs (set -1: none), the CTAs it spans, and which
// of this CTA's two records is its first.
struct SplitItem {
    int s, u, ctas, slot;
};

// Key tiles that the tokens of set `sp` below `tok_end` see.
__device__ __forceinline__ int tiles_seen(const SetSpan& sp, int tok_end) {
    const int vis = min(sp.len - sp.n + min(sp.n, tok_end), sp.len);
    return vis <= 0 ? 0 : (vis + TN - 1) / TN;
}

// An item's units of work: its key tiles, and `start` for what its start and end cost.
__device__ __forceinline__ int item_units(int tiles, int start) {
    return tiles > 0 ? tiles + start : 0;
}

// Units of a set, of all its items.
__device__ __forceinline__ long long set_units(const SetSpan& sp, const TilePlan& pl, int start) {
    long long sum = 0;
    for (int t = 0; t < sp.n; t += pl.tpi) sum += item_units(tiles_seen(sp, t + pl.tpi), start);
    return sum;
}

// Joins the records of one query row (record i at rec(i), the row is row r of its
// rec_rows), by WPR warps: warp wr takes every WPR-th batch of 8 and the warps'
// sums are joined in warp order through `shared` (WPR > 1: floats [WPR][D + 2]).
// Which record goes where depends on the count alone, so the result does not
// depend on timing.  Lane t of warp 0 gets dims [t D / 32, (t + 1) D / 32) of the
// normalised result in acc.
// INTERLEAVED: a record's dims 4 k .. 4 k + 3 of row r are float4 k * rows + r (as the
// tile kernel, thread = row, writes them); else O is [rows][D].
template <int D, int WPR, bool INTERLEAVED, typename Rec>
__device__ __forceinline__ void merge_records(int count, int rec_rows, int r, Rec&& rec,
                                              float (&acc)[D / 32], float* shared, int wr) {
    constexpr int DPL = D / 32;
    const int lane = threadIdx.x & 31;
    const int at = INTERLEAVED ? ((DPL * lane / 4) * rec_rows + r) * 4 + DPL * lane % 4
                               : r * D + DPL * lane;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
    for (int b = 8 * wr; b < count; b += 8 * WPR) {
        const int cnt = min(count - b, 8);
        float mw = -INFINITY, lw = 0.f;
        if (lane < cnt) {
            const float* pp = rec(b + lane) + rec_rows * D + r;
            mw = __ldcg(pp);
            lw = __ldcg(pp + rec_rows);
        }
        float ov[8][DPL];                                    // 8 records' loads in flight
#pragma unroll
        for (int u = 0; u < 8; ++u) {
#pragma unroll
            for (int c = 0; c < DPL; ++c) ov[u][c] = 0.f;
            if (u < cnt) {
                const float* ow = rec(b + u) + at;
                if (DPL == 4) {
                    const float4 x = __ldcg(reinterpret_cast<const float4*>(ow));
                    ov[u][0] = x.x, ov[u][1 % DPL] = x.y, ov[u][2 % DPL] = x.z, ov[u][3 % DPL] = x.w;
                } else {
                    const float2 x = __ldcg(reinterpret_cast<const float2*>(ow));
                    ov[u][0] = x.x, ov[u][1 % DPL] = x.y;
                }
            }
        }
        float Mb = mw;
#pragma unroll
        for (int k = 4; k > 0; k >>= 1) Mb = fmaxf(Mb, __shfl_xor_sync(~0u, Mb, k));
        Mb = __shfl_sync(~0u, Mb, 0);
        const float Mn = fmaxf(M, Mb);
        const float ref = Mn == -INFINITY ? 0.f : Mn;        // no mass yet: all factors 0
        const float fa = fast_exp2(M - ref), f = fast_exp2(mw - ref);
        L *= fa;
#pragma unroll
        for (int c = 0; c < DPL; ++c) acc[c] *= fa;
        M = Mn;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float fj = __shfl_sync(~0u, f, u), lj = __shfl_sync(~0u, lw, u);
            if (u < cnt) {
                L += lj * fj;
#pragma unroll
                for (int c = 0; c < DPL; ++c) acc[c] += ov[u][c] * fj;
            }
        }
    }
    if (WPR > 1) {
        float* mine = shared + wr * (D + 2);
#pragma unroll
        for (int c = 0; c < DPL; ++c) mine[DPL * lane + c] = acc[c];
        if (lane == 0) mine[D] = M, mine[D + 1] = L;
        __syncthreads();
        if (wr != 0) return;
        M = -INFINITY;
#pragma unroll
        for (int x = 0; x < WPR; ++x) M = fmaxf(M, shared[x * (D + 2) + D]);
        const float ref = M == -INFINITY ? 0.f : M;
        L = 0.f;
#pragma unroll
        for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
#pragma unroll
        for (int x = 0; x < WPR; ++x) {
            const float* o = shared + x * (D + 2);
            const float f = fast_exp2(o[D] - ref);
            L += o[D + 1] * f;
#pragma unroll
            for (int c = 0; c < DPL; ++c) acc[c] += o[DPL * lane + c] * f;
        }
    }
    const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);
#pragma unroll
    for (int c = 0; c < DPL; ++c) acc[c] *= inv;
}

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
