// Attention of a few new tokens over the paged cache (a decode step, drafted
// tokens): up to 32 query rows a set, n tokens x G heads (stream_rows()).
//
//   o[t][h] = sum_{j <= len - n + i} softmax_j(scale <q[t][h], k_j>) v_j
//
// for token i of the n new tokens of its sequence (t = its row of q), over the
// slots j of set (b, h / G).  A row that sees no slot gives 0.
//
// Each slot's K and V row is read once for all query rows of its set (4 d * 32 flops
// against 4 d bytes at most, far below the 278 flops a byte where the tensor cores
// would bound): what counts is to keep the reads in flight.  The sets' slots form
// one sequence of chunks (CH slots, never across a set); each warp of a persistent
// CTA takes one contiguous share of it, so ragged lengths and long caches split
// evenly.  A chunk moves as whole page slices by TMA into the warp's own two-stage
// ring, with the scale bytes and, at a segment's start, the query rows; the next
// chunk's page numbers are fetched one chunk ahead.
//
// Arithmetic per chunk on the tensor cores (mma.sync m16n8k16: bf16 operands,
// fp32 accumulation), whose operands can be converted in registers, with the
// cache's rows on the long side so that 8 query rows fill an instruction:
//   S^T = K Q^T   16 slots x 8 rows; integer K: a lane holds D / 4 consecutive
//                 values of a slot (whole scale groups), Q follows that order;
//   O^T += V^T P^T  16 dims x 8 rows; P^T is S^T's fragment transposed
//                 (movmatrix); integer V: ldmatrix transposes pairs of slots,
//                 the 2 or 4 values of its 16-bit elements are rows apart.
// Online softmax in base 2 (fp32), lane-local: a row's reference maximum moves
// (and O is rescaled) only when some logit exceeds it by 2^8, which one vote per
// chunk finds.  P is rounded to bf16 for the product, the normaliser sums the
// unrounded P.  A set inside one stream is written out at once; a split one
// leaves a partial (m, l, O) per stream, merged by a second kernel in stream
// order, so results do not depend on timing.
//
// What bounds it.  bf16: HBM (64 x 4 sets of one token over 4353 .. 8705 slots: 136 us,
// 6.3 TB/s).  Integer caches (the same sets in int8 88 us, 5.0 TB/s, int4 64 us): the chain
// of one chunk, from conversion over S and its maximum to P V, with two warps a
// scheduler to hide it: the integer pipe, which does the conversion, is at 51 to 54%, half
// the cycles issue, and most stalls wait for the instruction before; and the start
// and the merge, about 10 us of each call.
//
// Measured and not kept: partials joined inside this kernel, by flags that a set's
// first stream awaits or by whichever stream comes last (the batch above 92 and 97 us
// against 88: a warp alone has too few loads in flight); scales applied to V instead
// of P (32 layers of int4 92 us against 86).
#include "cache_launch.h"
#include "launch.h"
#include "tc05.cuh"

namespace tgvkv {
namespace {

constexpr int kStages = 2;
constexpr float kStale = 8.f;          // a reference maximum may trail by 2^8

template <int D, int FMT, int NB>
struct StreamGeom {
    static constexpr bool QUANT = FMT != TGVKV_CACHE_BF16;
    static constexpr int ROWB = FMT == TGVKV_CACHE_BF16 ? 2 * D : FMT == TGVKV_CACHE_INT8 ? D : D / 2;
    // Streams (warps) per CTA and bytes of a chunk's K.  8 streams of 4 KB, but for integer
    // caches of 64 dims and up to 8 query rows, whose loop has the registers for 16
    // streams of 2 KB: 32 layers x 32 heads x 2257 slots of int4 take 55 us instead of 62.
    // (128 dims: 16 streams of 2 KB 92 us, 8 of 4 KB 86 us.)  24 rows of 128 dims leave
    // the integer caches room for 2 KB only.
    static constexpr bool MANY = QUANT && NB == 1 && D == 64;
    static constexpr int W = MANY ? 16 : 8;
    static constexpr int TB = MANY || (QUANT && NB > 2 && D == 128) ? 2048 : 4096;
    static constexpr int CH = TB / ROWB > 64 ? 64 : TB / ROWB < 16 ? 16 : TB / ROWB;   // slots a chunk
    static constexpr int KT = QUANT ? 1 : D / 64; // tiles of a row
    static constexpr int TROW = ROWB / KT;        // bytes of a tile's row
    static constexpr int kTile = CH * TROW;
    static constexpr int SCB = QUANT ? D / kGroup : 0;   // scale bytes a row
    // a stage: K, V; aside from the swizzled tiles: K's scales, V's, NB * 8 query rows
    static constexpr int kK = 0;
    static constexpr int kV = KT * kTile;
    static constexpr int kStage = 2 * KT * kTile;
    static constexpr int kKS = 0;
    static constexpr int kVS = CH * SCB;
    static constexpr int kQ = 2 * CH * SCB;
    static constexpr int kSide = kQ + NB * 8 * 2 * D;
    static constexpr int kRing = W * kStages * (kStage + kSide);
    static_assert(kStage % 1024 == 0 && kTile % 256 == 0, "swizzled tiles");
};

template <int W>
struct StreamTail {
    uint64_t full[W][kStages];
    int2 start[W];                     // each stream's first set, and chunk in it
    long long warp_sum[W];
    int never;
};

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr) {
    uint32_t r;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(addr));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "r"(addr));
    return r;
}

// The 8 x 8 transpose of a fragment of 16-bit elements.
__device__ __forceinline__ uint32_t movm_trans(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// c += A B over one 16 x 8 x 16 tile.
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// bf16 bits of 2^(62 + e): with fp4x2_small()'s 2^-126, a 4-bit float of scale 2^e times
// 2^-64, exact for e in [-60, 56] (255: infinity, which times a code of 0 is NaN).
__device__ __forceinline__ uint32_t fp4_scale(uint32_t byte) { return min(byte + 62u, 255u) << 7; }

// Byte offset of 16-byte unit u of row r in a tile that TMA wrote with the
// swizzle of its row length (128, 64 or 32 bytes).
template <int TROW>
__device__ __forceinline__ uint32_t swz(int r, int u) {
    constexpr int shift = TROW == 128 ? 0 : TROW == 64 ? 1 : 2;
    constexpr int mask = TROW / 16 - 1;
    return (uint32_t)(r * TROW + ((u ^ ((r >> shift) & mask)) << 4));
}

// Chunks of a set: its last new token sees every slot.
template <int CH>
__device__ __forceinline__ int set_chunks(const SetSpan& sp) {
    return sp.n > 0 ? (sp.len + CH - 1) / CH : 0;
}

// A stream's walk over its chunks [c, c1) of the sequence.
template <int CH>
struct Walk {
    SetSpan sp;
    int s, at, chunks, left;           // set, the chunk in it, its chunks, chunks left of the share
    bool fresh;                        // the chunk starts a segment

    __device__ __forceinline__ void load(const CacheProblem& p, const ChunkArgs& a) {
        sp = set_span(p, a, s);
        chunks = set_chunks<CH>(sp);
    }
    __device__ __forceinline__ void init(const CacheProblem& p, const ChunkArgs& a, int2 start,
                                         int count) {
        left = count;
        fresh = true;
        s = start.x;
        at = start.y;
        load(p, a);
    }
    // the chunk: slots [key0(), key0() + n()) of set s
    __device__ __forceinline__ int key0() const { return at * CH; }
    __device__ __forceinline__ int n() const { return min(sp.len - at * CH, CH); }
    __device__ __forceinline__ bool ends() const { return at + 1 == chunks || left == 1; }
    __device__ __forceinline__ void step(const CacheProblem& p, const ChunkArgs& a) {
        fresh = false;
        if (--left <= 0) return;
        if (++at < chunks) return;
        fresh = true;
        at = 0;
        do {
            if (++s >= p.S) {
                left = 0;
                return;
            }
            load(p, a);
        } while (chunks == 0);
    }
};

// The copies of the walk's chunk into one stage, spread over the warp's lanes.
// Lane b < boxes holds the page number of the chunk's b-th page slice.
template <int D, int FMT, int NB>
__device__ __forceinline__ void issue(unsigned char* stage, unsigned char* side, uint64_t* bar,
                                      const Walk<StreamGeom<D, FMT, NB>::CH>& w, int page, int box,
                                      int box_shift, const CUtensorMap* mk, const CUtensorMap* mv,
                                      const CacheProblem& p, const CachePools& pool,
                                      const ChunkArgs& a, int lane) {
    using Gm = StreamGeom<D, FMT, NB>;
    const int nb = (w.n() + box - 1) >> box_shift;
    const uint32_t per_box = (uint32_t)box * (2 * Gm::ROWB + 2 * Gm::SCB);
    uint32_t bytes = nb * per_box;
    if (w.fresh) bytes += (uint32_t)(w.sp.n * p.G) * 2 * D;
    if (lane == 0) tc::mbar_arrive_expect_tx(bar, bytes);
    __syncwarp();
    if (lane < nb) {
        const int row = page * p.page + ((w.key0() + lane * box) & (p.page - 1));
        const uint32_t at = (uint32_t)(lane * box);
#pragma unroll
        for (int kt = 0; kt < Gm::KT; ++kt) {
            tc::tma_load_2d(stage + Gm::kK + kt * Gm::kTile + at * Gm::TROW, mk, 128 * kt, row, bar);
            tc::tma_load_2d(stage + Gm::kV + kt * Gm::kTile + at * Gm::TROW, mv, 128 * kt, row, bar);
        }
        if (FMT != TGVKV_CACHE_BF16) {
            const size_t off = (size_t)row * Gm::SCB;
            tc::bulk_load(smem_u32(side + Gm::kKS) + at * Gm::SCB, pool.ks + off, box * Gm::SCB, bar);
            tc::bulk_load(smem_u32(side + Gm::kVS) + at * Gm::SCB, pool.vs + off, box * Gm::SCB, bar);
        }
    }
    if (w.fresh && lane < w.sp.n * p.G) {
        const int i = lane / p.G, h = lane - i * p.G;
        const uint16_t* src = a.q + (long long)(w.sp.tok0 + i) * a.q_tok +
                              (long long)((w.s % p.H_kv) * p.G + h) * a.q_head;
        tc::bulk_load(smem_u32(side + Gm::kQ) + lane * 2 * D, src, 2 * D, bar);
    }
}

__device__ __forceinline__ int valid_page(const CacheProblem& p, int page, uint32_t* status) {
    if (page >= 0 && page < p.n_pages) return page;
    raise_status(status, TGVKV_STATUS_INDEX);
    return 0;
}

// The dims of a lane's results in the 16-dim row tile mt of O^T: its row g is
// dim out_dim(mt, g), its row g + 8 the dim out_step later.
template <int FMT>
__device__ __forceinline__ int out_dim(int mt, int g) {
    if (FMT == TGVKV_CACHE_BF16) return 16 * mt + g;
    if (FMT == TGVKV_CACHE_INT8) return 16 * mt + 2 * g;
    return 32 * (mt >> 1) + 4 * g + 2 * (mt & 1);
}

// SHORT: CTA b has set b, its warps one stretch of it each, joined through shared
// memory; else the warps of all CTAs share all sets, and split sets are left to
// chunk_stream_merge.
template <int D, int FMT, int NB, bool SHORT>
__global__ void __launch_bounds__(StreamGeom<D, FMT, NB>::W * 32, 1)
chunk_stream_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                    const CacheProblem p, const CachePools pool, const ChunkArgs a, int box,
                    int box_shift, int rec_rows, float* __restrict__ part,
                    long long* __restrict__ plan, uint32_t* __restrict__ status) {
    using Gm = StreamGeom<D, FMT, NB>;
    constexpr int CH = Gm::CH, W = Gm::W;
    constexpr int KS = D / 16, MT = D / 16, KB = CH / 16;
    // 4-bit floats are multiplied as K 2^-64 (fp4_scale), and as V's codes 2^-126 against
    // P 2^62 (kBf16x2Up62) with V's scale, P V 2^-64: one factor of 2^64 on S and on O, and one on
    // every two weights, in the place of one on every K and V.  (The 2^62 as 62 on the exponent
    // rounds m - 62: two warps' weights were off against each other by up to 2^4 at logits of 2^25,
    // and small values lost from 2^30 on.)  One token of 64 x 4 sets
    // of 4353 .. 8705 slots, 7 rows: 77.0 us (int4 65, int8 87.8); two warps a scheduler in one
    // chain of dependent steps each.  S in fp16 from the hardware's conversion of codes: a sixth
    // fewer instructions, but a longer chain, 77.4 against 76.6 us; twelve or sixteen warps of half
    // a chunk 76.5 and 76.7 (twelve with S in fp16 73.4, for a second form of the loop and a test
    // of every chunk's scales), ten 85; four accumulators a chain 78; codes shifted right by
    // products or byte swaps, off the integer pipe, 83.  Shares as even as can be instead of
    // rounded up: 75.1, but 23.0 against 19.6 for one sequence of 34000 slots (more split sets).
    constexpr float kUp = FMT == TGVKV_CACHE_FP4 ? 0x1p64f : 1.f;
    if (threadIdx.x == 0) {
        tc::tma_prefetch_desc(&mk);
        tc::tma_prefetch_desc(&mv);
    }
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    StreamTail<W>& tl = *reinterpret_cast<StreamTail<W>*>(ring + Gm::kRing);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) tl.never = 0;
    if (lane == 0) {
        for (int st = 0; st < kStages; ++st) tc::mbar_init(&tl.full[warp][st], 1);
        tc::fence_mbar_init();
    }
    // The kernel before has finished; the merge, which may start from now on, reads this
    // call's inputs before it waits in turn.
    griddep_wait();
    griddep_launch_dependents();
    if (blockIdx.x == 0) check_spans(p, a, tid, W * 32, status);

    const int si = blockIdx.x * W + warp;
    int per;                           // chunks a stream
    long long total = 0, c_lo;         // chunks of all (SHORT: of the set), this stream's first
    if constexpr (SHORT) {
        total = set_chunks<CH>(set_span(p, a, blockIdx.x));
        per = max((int)((total + W - 1) / W), 1);
        c_lo = (long long)warp * per;
        if (lane == 0) tl.start[warp] = make_int2(blockIdx.x, (int)c_lo);
        __syncthreads();
    } else {
        // ---- the plan: thread t counts the chunks of sets [t * run, (t + 1) * run)
        const int run = (p.S + W * 32 - 1) / (W * 32);
        const int s_lo = min(tid * run, p.S), s_hi = min(s_lo + run, p.S);
        long long sum = 0;
        for (int s = s_lo; s < s_hi; ++s) sum += set_chunks<CH>(set_span(p, a, s));
        long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) tl.warp_sum[warp] = incl;
        __syncthreads();
        long long base = incl - sum;
#pragma unroll
        for (int x = 0; x < W; ++x) {
            if (x < warp) base += tl.warp_sum[x];
            total += tl.warp_sum[x];
        }
        const int n_streams = gridDim.x * W;
        per = max((int)((total + n_streams - 1) / n_streams), 1);      // chunks a stream
        // the starts of this CTA's streams that lie in my sets; CTA 0 also writes the plan
        {
            const long long first = (long long)blockIdx.x * W * per;
            if (blockIdx.x == 0 || (first < base + sum && first + (long long)W * per > base)) {
                long long at = base;
                for (int s = s_lo; s < s_hi; ++s) {
                    const int n = set_chunks<CH>(set_span(p, a, s));
                    if (blockIdx.x == 0) plan[s] = at;
                    for (int x = 0; x < W; ++x) {
                        const long long c = first + (long long)x * per;
                        if (c >= at && c < at + n) tl.start[x] = make_int2(s, (int)(c - at));
                    }
                    at += n;
                }
            }
            if (blockIdx.x == 0 && tid == 0) plan[p.S] = total;
        }
        __syncthreads();
        c_lo = (long long)si * per;
        if (c_lo >= total) return;
    }

    unsigned char* wring = ring + warp * kStages * Gm::kStage;
    unsigned char* wside = ring + W * kStages * Gm::kStage + warp * kStages * Gm::kSide;
    Walk<CH> ahead;                    // the next chunk to fetch
    ahead.init(p, a, tl.start[warp], (int)max(min((long long)per, total - c_lo), 0ll));
    Walk<CH> w = ahead;                // the next chunk to work on
    const int32_t* table = a.page_table + (size_t)ahead.s * p.max_pages;
    auto page_of = [&]() {             // lane b: page number of the chunk's slice b
        const int slot = ahead.key0() + (lane << box_shift);
        return (lane << box_shift) < ahead.n() ? table[slot >> p.page_shift] : 0;
    };
    int page = ahead.left > 0 ? page_of() : 0;
    int issued = 0;
    auto refill = [&]() {              // the next chunk into the stage just read
        const int st = issued % kStages;
        issue<D, FMT, NB>(wring + st * Gm::kStage, wside + st * Gm::kSide, &tl.full[warp][st], ahead,
                          valid_page(p, page, status), box, box_shift, &mk, &mv, p, pool, a, lane);
        ++issued;
        ahead.step(p, a);
        if (ahead.left > 0) {          // its page numbers, a chunk ahead of their use
            if (ahead.fresh) table = a.page_table + (size_t)ahead.s * p.max_pages;
            page = page_of();
        }
    };
    for (int st = 0; st < kStages && ahead.left > 0; ++st) refill();
    __syncwarp();

    const int g = lane >> 2, tq = lane & 3;
    uint32_t qb[KS][NB][2];
    float o[MT][NB][4];
    float m[NB][2], l[NB][2];          // of rows 8 nb + 2 tq and the next
    bool seg_starts = true;            // the segment began at its set's first chunk
    bool share_starts = true;          // ... is the first of this stream
    if constexpr (SHORT) {             // a stretch without a chunk
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) m[nb][e] = -INFINITY, l[nb][e] = 0.f;
    }
    int i = 0;
    for (; w.left > 0; ++i) {
        const int st = i % kStages;
        const bool got = tc::mbar_wait(&tl.full[warp][st], (i / kStages) & 1, &tl.never);
        if (!__all_sync(~0u, got)) break;
        unsigned char* stage = wring + st * Gm::kStage;
        const uint32_t sb = smem_u32(stage), sd = smem_u32(wside + st * Gm::kSide);
        const int key0 = w.key0(), n = w.n();
        if (w.fresh) {
            seg_starts = w.at == 0;
            share_starts = i == 0;
            // Q^T fragments: pairs of dims in the order the K fragments have; 0 in
            // rows the set does not have
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const uint32_t q0 = sd + Gm::kQ + (8 * nb + g) * 2 * D;
                if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        qb[s][nb][0] = lds32(q0 + 32 * s + 4 * tq);
                        qb[s][nb][1] = lds32(q0 + 32 * s + 16 + 4 * tq);
                    }
                } else if (FMT == TGVKV_CACHE_INT8) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) {   // 4 values: (0, 2) and (1, 3)
                        const uint2 x = lds64(q0 + tq * (D / 2) + 8 * s);
                        qb[s][nb][0] = __byte_perm(x.x, x.y, 0x5410);
                        qb[s][nb][1] = __byte_perm(x.x, x.y, 0x7632);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < KS / 2; ++s) {   // 8: (0, 4) (1, 5), (2, 6) (3, 7)
                        const uint4 x = lds128(q0 + tq * (D / 2) + 16 * s);
                        qb[2 * s][nb][0] = __byte_perm(x.x, x.z, 0x5410);
                        qb[2 * s][nb][1] = __byte_perm(x.x, x.z, 0x7632);
                        qb[2 * s + 1][nb][0] = __byte_perm(x.y, x.w, 0x5410);
                        qb[2 * s + 1][nb][1] = __byte_perm(x.y, x.w, 0x7632);
                    }
                }
                if (8 * nb + g >= w.sp.n * p.G) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) qb[s][nb][0] = qb[s][nb][1] = 0u;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) m[nb][e] = -INFINITY, l[nb][e] = 0.f;
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][nb][e] = 0.f;
            }
        }
        // ---- S^T = K Q^T; tile kb holds slots 16 kb + g and 16 kb + g + 8
        float sc[KB][NB][4];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            float acc[2][NB][4];       // two halves of the dims: independent chains
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[y][nb][e] = 0.f;
            if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int unit = 2 * s + (lane >> 4);
                    uint32_t r[4];
                    ldsm_x4(sb + Gm::kK + (unit >> 3) * Gm::kTile +
                                swz<128>(16 * kb + (lane & 15), unit & 7),
                            r);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        mma(acc[s & 1][nb], r, qb[s][nb][0], qb[s][nb][1]);
                }
            } else {
                constexpr int NW = Gm::ROWB / 16;    // words of codes a lane holds of a row
                uint32_t wd[2][NW], kb_s[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * kb + 8 * x + g;
                    if (NW == 2) {
                        const uint2 t = lds64(sb + Gm::kK + swz<Gm::TROW>(row, tq >> 1) + (tq & 1) * 8);
                        wd[x][0] = t.x, wd[x][1 % NW] = t.y;
                    } else {
#pragma unroll
                        for (int b = 0; b < NW / 4; ++b) {
                            const uint4 t =
                                lds128(sb + Gm::kK + swz<Gm::TROW>(row, tq * (NW / 4) + b));
                            wd[x][(4 * b) % NW] = t.x, wd[x][(4 * b + 1) % NW] = t.y;
                            wd[x][(4 * b + 2) % NW] = t.z, wd[x][(4 * b + 3) % NW] = t.w;
                        }
                    }
                    const uint32_t byte =
                        lds8(sd + Gm::kKS + row * Gm::SCB + (D == 128 ? tq : tq >> 1));
                    kb_s[x] = both(FMT == TGVKV_CACHE_INT8   ? scale_bf16(byte)
                                   : FMT == TGVKV_CACHE_INT4 ? int4_base(byte)
                                                             : fp4_scale(byte));
                }
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    uint32_t r[4];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (FMT == TGVKV_CACHE_INT8) {
                            const uint32_t c = wd[x][s % NW];
                            r[x] = bf16x2_mul(int8x2_to_bf16(c, p.magic), kb_s[x]);
                            r[2 + x] = bf16x2_mul(int8x2_to_bf16(c >> 8, p.magic), kb_s[x]);
                        } else if (FMT == TGVKV_CACHE_INT4) {
                            const uint32_t c = wd[x][(s / 2) % NW];
                            r[x] = int4x2_to_bf16(c >> (8 * (s & 1)), kb_s[x]);
                            r[2 + x] = int4x2_to_bf16(c >> (8 * (s & 1) + 4), kb_s[x]);
                        } else {
                            const uint32_t c = wd[x][(s / 2) % NW];
                            r[x] = bf16x2_mul(s & 1 ? fp4x2_small<8>(c) : fp4x2_small<0>(c), kb_s[x]);
                            r[2 + x] = bf16x2_mul(s & 1 ? fp4x2_small<12>(c) : fp4x2_small<4>(c), kb_s[x]);
                        }
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        mma(acc[s & 1][nb], r, qb[s][nb][0], qb[s][nb][1]);
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc[kb][nb][e] = (acc[0][nb][e] + acc[1][nb][e]) * kUp * p.scale_log2;
        }
        // ---- hide what a row must not see: slots from its token's on
        if (n < CH || key0 + CH > w.sp.len - w.sp.n + 1) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int lim =
                        min(w.sp.len - w.sp.n + (8 * nb + 2 * tq + e) / p.G + 1 - key0, n);
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        if (16 * kb + g >= lim) sc[kb][nb][e] = -INFINITY;
                        if (16 * kb + 8 + g >= lim) sc[kb][nb][2 + e] = -INFINITY;
                    }
                }
        }
        // ---- online softmax; a row's 8 lanes share m
        bool move = false;
        float cm[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                cm[nb][e] = fmaxf(sc[0][nb][e], sc[0][nb][2 + e]);
#pragma unroll
                for (int kb = 1; kb < KB; ++kb)
                    cm[nb][e] = fmaxf(cm[nb][e], fmaxf(sc[kb][nb][e], sc[kb][nb][2 + e]));
                move |= cm[nb][e] > m[nb][e] + kStale;
            }
        if (__any_sync(~0u, move)) {   // also a segment's first chunk
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float c = cm[nb][e];
                    c = fmaxf(c, __shfl_xor_sync(~0u, c, 4));
                    c = fmaxf(c, __shfl_xor_sync(~0u, c, 8));
                    c = fmaxf(c, __shfl_xor_sync(~0u, c, 16));
                    const float mn = fmaxf(m[nb][e], c);
                    const float alpha = mn == -INFINITY ? 1.f : fast_exp2(m[nb][e] - mn);
                    m[nb][e] = mn;
                    l[nb][e] *= alpha;
#pragma unroll
                    for (int t = 0; t < MT; ++t) o[t][nb][e] *= alpha, o[t][nb][2 + e] *= alpha;
                }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float ref = m[nb][e] == -INFINITY ? 0.f : m[nb][e];   // nothing seen: weights 0
                float ps = 0.f;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    sc[kb][nb][e] = fast_exp2(sc[kb][nb][e] - ref);
                    sc[kb][nb][2 + e] = fast_exp2(sc[kb][nb][2 + e] - ref);
                    ps += sc[kb][nb][e] + sc[kb][nb][2 + e];
                }
                l[nb][e] += ps;
            }
        // ---- slots past the set's end hold what the pool holds there: their
        // weights are 0, and 0 x NaN is not, so V must be 0 (integer V is finite, its scale 0)
        if (FMT == TGVKV_CACHE_BF16 && n < CH) {
            const int end = (n + 15) & ~15;
            for (int x = lane; x < (end - n) * 8 * Gm::KT; x += 32) {
                const int r = n + x / (8 * Gm::KT), u = x % (8 * Gm::KT);
                *reinterpret_cast<uint4*>(stage + Gm::kV + (u >> 3) * Gm::kTile + r * 128 + (u & 7) * 16) =
                    make_uint4(0u, 0u, 0u, 0u);
            }
            tc::fence_proxy_async_smem();   // before TMA writes the stage again
            __syncwarp();
        }
        // ---- O^T += V^T P^T over 16 slots at a time
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            if (16 * kb >= n) break;
            uint32_t pb[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                pb[nb][0] = movm_trans(pack_bf16x2(sc[kb][nb][0], sc[kb][nb][1]));
                pb[nb][1] = movm_trans(pack_bf16x2(sc[kb][nb][2], sc[kb][nb][3]));
                if (FMT == TGVKV_CACHE_FP4) {              // (kUp)
                    pb[nb][0] = bf16x2_mul(pb[nb][0], kBf16x2Up62);
                    pb[nb][1] = bf16x2_mul(pb[nb][1], kBf16x2Up62);
                }
            }
            if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int unit = 2 * t + ((lane >> 3) & 1);
                    uint32_t r[4];
                    ldsm_x4_trans(sb + Gm::kV + (unit >> 3) * Gm::kTile +
                                      swz<128>(16 * kb + (lane & 7) + (lane >> 4) * 8, unit & 7),
                                  r);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma(o[t][nb], r, pb[nb][0], pb[nb][1]);
                }
            } else {
                // V's scales go to P instead, 2 values a group where V has 32 (exactly, as they are
                // powers of two, while P 2^e, P at most 2^8, stays a normal bf16 number: not
                // for P below 2^-126-e or e above 119): the scales of this lane's slot pairs
                // (2 tq, + 1) and (2 tq + 8, + 9)
                constexpr int NG = D / kGroup, UPG = Gm::ROWB / 16 / NG;   // units a group
                uint32_t sw[2][2];     // scale bytes of slot pair h, one slot and the next
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k0 = 16 * kb + 2 * tq + 8 * h;
                    if (D == 128) {
                        const uint2 t = lds64(sd + Gm::kVS + k0 * 4);
                        sw[h][0] = t.x, sw[h][1] = t.y;
                    } else {
                        const uint32_t t = lds32(sd + Gm::kVS + k0 * 2);
                        sw[h][0] = t & 0xFFFFu, sw[h][1] = t >> 16;
                    }
                    if (k0 >= n) sw[h][0] = 0u;
                    if (k0 + 1 >= n) sw[h][1] = 0u;
                }
                uint32_t r[4] = {0u, 0u, 0u, 0u}, pg[NB][2];
#pragma unroll
                for (int u = 0; u < Gm::ROWB / 16; ++u) {        // 16-byte units of a row
                    if (u % UPG == 0) {
                        const int x = u / UPG;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t sc2 =
                                (__byte_perm(sw[h][0], sw[h][1], (x << 4) | ((4 + x) << 12)) >> 1) &
                                0x7F807F80u;
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) pg[nb][h] = bf16x2_mul(pb[nb][h], sc2);
                        }
                    }
                    if (u % 2 == 0)
                        ldsm_x4_trans(sb + Gm::kV + swz<Gm::TROW>(16 * kb + (lane & 15), u + (lane >> 4)), r);
                    const uint32_t r0 = r[2 * (u % 2)], r1 = r[2 * (u % 2) + 1];
                    if (FMT == TGVKV_CACHE_INT8) {
                        const uint32_t v[4] = {int8x2_to_bf16(r0, p.magic), int8x2_to_bf16(r0 >> 8, p.magic),
                                               int8x2_to_bf16(r1, p.magic), int8x2_to_bf16(r1 >> 8, p.magic)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma(o[u % MT][nb], v, pg[nb][0], pg[nb][1]);
                    } else if (FMT == TGVKV_CACHE_FP4) {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const uint32_t v[4] = {y ? fp4x2_small<8>(r0) : fp4x2_small<0>(r0),
                                                   y ? fp4x2_small<12>(r0) : fp4x2_small<4>(r0),
                                                   y ? fp4x2_small<8>(r1) : fp4x2_small<0>(r1),
                                                   y ? fp4x2_small<12>(r1) : fp4x2_small<4>(r1)};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma(o[(2 * u + y) % MT][nb], v, pg[nb][0], pg[nb][1]);
                        }
                    } else {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const uint32_t v[4] = {int4x2_to_bf16(r0 >> (8 * y), p.magic),
                                                   int4x2_to_bf16(r0 >> (8 * y + 4), p.magic),
                                                   int4x2_to_bf16(r1 >> (8 * y), p.magic),
                                                   int4x2_to_bf16(r1 >> (8 * y + 4), p.magic)};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma(o[(2 * u + y) % MT][nb], v, pg[nb][0], pg[nb][1]);
                        }
                    }
                }
            }
        }
        __syncwarp();                  // the stage is read: refill it
        if (ahead.left > 0) refill();
        const bool ends = w.ends();
        if (ends) {
            // ---- the segment of set w.s is complete
            if (FMT == TGVKV_CACHE_FP4) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][nb][e] *= kUp;
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[nb][e] += __shfl_xor_sync(~0u, l[nb][e], 4);
                    l[nb][e] += __shfl_xor_sync(~0u, l[nb][e], 8);
                    l[nb][e] += __shfl_xor_sync(~0u, l[nb][e], 16);
                }
            if constexpr (!SHORT) {
                const bool whole = seg_starts && w.at + 1 == w.chunks;
                float* pp = part + ((size_t)si * 2 + (share_starts ? 0 : 1)) *
                                       (size_t)chunk_record_floats(rec_rows, D);
                constexpr int STEP = FMT == TGVKV_CACHE_BF16 ? 8 : 1;   // dims between rows g and g + 8
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = 8 * nb + 2 * tq + e;
                        if (r >= w.sp.n * p.G) continue;
                        if (whole) {       // the whole set: written out
                            const float ls = l[nb][e];
                            const float inv = ls > 0.f ? 1.f / ls : (ls == ls ? 0.f : ls);
                            const int t = r / p.G, hh = r - t * p.G;
                            uint16_t* op = a.out +
                                           ((size_t)(w.sp.tok0 + t) * p.H_q + (w.s % p.H_kv) * p.G + hh) * D;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                const uint32_t two =
                                    pack_bf16x2(o[mt][nb][e] * inv, o[mt][nb][2 + e] * inv);
                                uint16_t* od = op + out_dim<FMT>(mt, g);
                                if (STEP == 1) {
                                    *reinterpret_cast<uint32_t*>(od) = two;
                                } else {
                                    od[0] = (uint16_t)two;
                                    od[STEP] = (uint16_t)(two >> 16);
                                }
                            }
                        } else {
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                float* od = pp + r * D + out_dim<FMT>(mt, g);
                                if (STEP == 1) {
                                    *reinterpret_cast<float2*>(od) = make_float2(o[mt][nb][e], o[mt][nb][2 + e]);
                                } else {
                                    od[0] = o[mt][nb][e];
                                    od[STEP] = o[mt][nb][2 + e];
                                }
                            }
                            if (g == 0) {
                                pp[rec_rows * D + r] = m[nb][e];
                                pp[rec_rows * D + rec_rows + r] = l[nb][e];
                            }
                        }
                    }
            }
        }
        w.step(p, a);
    }
    if (i < issued) {
        // a wait gave up: report it and let the copies in flight land
        if (lane == 0) raise_status(status, TGVKV_STATUS_TIMEOUT);
        for (; i < issued; ++i)
            if (!tc::mbar_wait(&tl.full[warp][i % kStages], (i / kStages) & 1, &tl.never)) break;
    }
    if constexpr (SHORT) {
        // the warps' partials, as their lanes hold them, in their rings (read by now):
        // float4 x of lane t at 32 x + t; a warp joins every W-th float4
        constexpr int X = MT * NB;
        static_assert(16 * 32 * (X + NB) <= kStages * Gm::kStage, "a partial fits a ring");
        const int used = (int)min((total + per - 1) / per, (long long)W);
        float4* mine = reinterpret_cast<float4*>(wring) + lane;
        if (warp < used) {
#pragma unroll
            for (int x = 0; x < X; ++x) {
                const float(&c)[4] = o[x / NB][x % NB];
                mine[32 * x] = make_float4(c[0], c[1], c[2], c[3]);
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                mine[32 * (X + nb)] = make_float4(m[nb][0], m[nb][1], l[nb][0], l[nb][1]);
        }
        __syncthreads();
        for (int x = warp; x < X; x += W) {
            const int mt = x / NB, nb = x % NB;
            const float4* recs = reinterpret_cast<const float4*>(ring) + lane;
            constexpr int REC = kStages * Gm::kStage / 16;
            float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f}, c[4] = {0.f, 0.f, 0.f, 0.f};
            for (int j = 0; j < used; ++j) {
                const float4 ml = recs[j * REC + 32 * (X + nb)];
                M[0] = fmaxf(M[0], ml.x), M[1] = fmaxf(M[1], ml.y);
            }
            const float r0 = M[0] == -INFINITY ? 0.f : M[0], r1 = M[1] == -INFINITY ? 0.f : M[1];
            for (int j = 0; j < used; ++j) {
                const float4 ml = recs[j * REC + 32 * (X + nb)], t = recs[j * REC + 32 * x];
                const float f0 = fast_exp2(ml.x - r0), f1 = fast_exp2(ml.y - r1);
                L[0] += ml.z * f0, L[1] += ml.w * f1;
                c[0] += t.x * f0, c[1] += t.y * f1, c[2] += t.z * f0, c[3] += t.w * f1;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * nb + 2 * tq + e;
                if (r >= w.sp.n * p.G) continue;
                const float inv = L[e] > 0.f ? 1.f / L[e] : (L[e] == L[e] ? 0.f : L[e]);
                const int t = r / p.G, hh = r - t * p.G;
                uint16_t* od = a.out + ((size_t)(w.sp.tok0 + t) * p.H_q + (w.s % p.H_kv) * p.G + hh) * D +
                               out_dim<FMT>(mt, g);
                const uint32_t two = pack_bf16x2(c[e] * inv, c[2 + e] * inv);
                if (FMT == TGVKV_CACHE_BF16) {
                    od[0] = (uint16_t)two;
                    od[8] = (uint16_t)(two >> 16);
                } else {
                    *reinterpret_cast<uint32_t*>(od) = two;
                }
            }
        }
    }
}

// The split sets' merge and the rows that see nothing: WPR warps per (set, query
// row), a programmatic dependent of the stream kernel.  A set's partials are
// combined in stream order.
template <int D, int WPR>
__global__ void __launch_bounds__(WPR == 1 ? 128 : WPR * 32)
chunk_stream_merge(const CacheProblem p, const ChunkArgs a, int n_streams, int rec_rows,
                   const float* __restrict__ part,
                   const long long* __restrict__ plan) {
    constexpr int DPL = D / 32;
    __shared__ float shared[WPR == 1 ? 1 : WPR * (D + 2)];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long gw = WPR == 1 ? (long long)blockIdx.x * 4 + warp : (long long)blockIdx.x;
    const int s = (int)(gw / rec_rows), r = (int)(gw % rec_rows);
    griddep_launch_dependents();       // the next call's set-up may overlap
    SetSpan sp{0, 0, 0};
    if (s < p.S) sp = set_span(p, a, s);
    griddep_wait();
    if (s >= p.S || r >= sp.n * p.G) return;
    const long long c0 = __ldcg(plan + s), c1 = __ldcg(plan + s + 1), total = __ldcg(plan + p.S);
    float acc[DPL];
#pragma unroll
    for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
    if (c1 > c0) {
        const int per = max((int)((total + n_streams - 1) / n_streams), 1);
        const int w0 = (int)(c0 / per), w1 = (int)((c1 - 1) / per);
        if (w0 == w1) return;          // inside one stream: written by it
        // a segment starts its stream's share, but for a set that begins inside it
        const int first = c0 != (long long)w0 * per ? 1 : 0;
        const size_t rec = chunk_record_floats(rec_rows, D);
        merge_records<D, WPR, false>(w1 - w0 + 1, rec_rows, r, [&](int i) {
            return part + ((size_t)(w0 + i) * 2 + (i == 0 ? first : 0)) * rec;
        }, acc, shared, WPR == 1 ? 0 : warp);
    }
    if (WPR > 1 && warp != 0) return;
    const int t = r / p.G, hh = r - t * p.G;
    uint16_t* out = a.out + ((size_t)(sp.tok0 + t) * p.H_q + (s % p.H_kv) * p.G + hh) * D + DPL * lane;
#pragma unroll
    for (int c = 0; c < DPL; c += 2)
        *reinterpret_cast<uint32_t*>(out + c) = pack_bf16x2(acc[c], acc[(c + 1) % DPL]);
}

// SHORT takes calls of up to 16 rows with a CTA for every set at once, whose page
// tables hold at most this many chunks a warp.  One kernel and no records in global
// memory against shares of equal size (one token, us): 8 sets of bf16, d = 64,
// 113 slots 4.4 / 7.6, 1000 (4 chunks) 7.3 / 7.2, 2000 10.7 / 7.3; d = 128, 500 (4) 7.7 / 8.0,
// 1000 10.8 / 8.6; int4, d = 128, 500 (1) 6.8 / 9.5, 1000 (2) 9.7 / 9.4, 2000 15.4 / 9.8.
template <int FMT>
constexpr int short_chunks() {
    return FMT == TGVKV_CACHE_BF16 ? 4 : 2;
}

template <int D, int FMT, int NB>
cudaError_t launch_stream(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                          float* part, long long* plan, uint32_t* status, cudaStream_t stream) {
    using Gm = StreamGeom<D, FMT, NB>;
    const int box = p.page < Gm::CH ? p.page : Gm::CH;
    int box_shift = 0;
    while ((1 << box_shift) < box) ++box_shift;
    alignas(64) CUtensorMap mk, mv;
    const uint64_t rows = (uint64_t)p.n_pages * p.page;
    const int box_bytes = FMT == TGVKV_CACHE_BF16 ? 128 : Gm::ROWB;
    if (!make_pool_map(&mk, pool.k, rows, Gm::ROWB, box_bytes, box) ||
        !make_pool_map(&mv, pool.v, rows, Gm::ROWB, box_bytes, box))
        return cudaErrorInvalidValue;
    const size_t smem = 1024 + Gm::kRing + sizeof(StreamTail<Gm::W>);
    static_assert(1024 + Gm::kRing + sizeof(StreamTail<Gm::W>) <= 227 * 1024, "shared memory of one CTA");
    auto prepare = [&](auto kernel) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    };
    cudaError_t e;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    if constexpr (NB <= 2) {
        if (p.S <= sms && (p.cap + Gm::CH - 1) / Gm::CH <= short_chunks<FMT>() * Gm::W) {
            const auto kernel = chunk_stream_kernel<D, FMT, NB, true>;
            if ((e = prepare(kernel)) != cudaSuccess) return e;
            return launch_dependent(kernel, dim3((unsigned)p.S), dim3(Gm::W * 32), smem, stream, mk, mv, p,
                                    pool, a, box, box_shift, 0, part, plan, status);
        }
    }
    const auto kernel = chunk_stream_kernel<D, FMT, NB, false>;
    if ((e = prepare(kernel)) != cudaSuccess) return e;
    const int ctas = sms < kStreamMaxCtas ? sms : kStreamMaxCtas;
    const int rec_rows = a.max_q * p.G;
    e = launch_dependent(kernel, dim3((unsigned)ctas), dim3(Gm::W * 32), smem, stream, mk, mv, p, pool, a,
                         box, box_shift, rec_rows, part, plan, status);
    if (e != cudaSuccess) return e;
    // A set has about n_streams / S records: from 16 on, 8 warps join a row.  8 warps / 1,
    // one int8 token over 17409 .. 34816 slots, us: 4 sets 21 / 60, 16 sets 32 / 44, 64 sets
    // 86 / 89; fewer records, 256 sets of 4353 .. 8705 slots 96 / 88.
    const long long rows_out = (long long)p.S * rec_rows;
    const float* parts = part;
    const long long* plans = plan;
    if ((long long)p.S * 16 <= ctas * Gm::W)
        return launch_dependent(chunk_stream_merge<D, 8>, dim3((unsigned)rows_out), dim3(256), 0, stream,
                                p, a, ctas * Gm::W, rec_rows, parts, plans);
    return launch_dependent(chunk_stream_merge<D, 1>, dim3((unsigned)((rows_out + 3) / 4)), dim3(128),
                            0, stream, p, a, ctas * Gm::W, rec_rows, parts, plans);
}

template <int D, int FMT>
cudaError_t launch_rows(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                        float* part, long long* plan, uint32_t* status, cudaStream_t stream) {
    const int rows = a.max_q * p.G;    // at most stream_rows(D, FMT)
    constexpr int most = stream_rows(D, FMT);
    if (rows <= 8) return launch_stream<D, FMT, 1>(p, pool, a, part, plan, status, stream);
    if (rows <= 16) return launch_stream<D, FMT, 2>(p, pool, a, part, plan, status, stream);
    if constexpr (most > 24)
        if (rows > 24) return launch_stream<D, FMT, 4>(p, pool, a, part, plan, status, stream);
    if constexpr (most > 16) return launch_stream<D, FMT, 3>(p, pool, a, part, plan, status, stream);
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_chunk_stream(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                                float* part, long long* plan, uint32_t* status, cudaStream_t stream) {
    const auto by_dim = [&](auto kernels_of_64, auto kernels_of_128) {
        return p.d == 64 ? kernels_of_64(p, pool, a, part, plan, status, stream)
                         : kernels_of_128(p, pool, a, part, plan, status, stream);
    };
    switch (p.format) {
        case TGVKV_CACHE_BF16: return by_dim(launch_rows<64, TGVKV_CACHE_BF16>, launch_rows<128, TGVKV_CACHE_BF16>);
        case TGVKV_CACHE_INT8: return by_dim(launch_rows<64, TGVKV_CACHE_INT8>, launch_rows<128, TGVKV_CACHE_INT8>);
        case TGVKV_CACHE_INT4: return by_dim(launch_rows<64, TGVKV_CACHE_INT4>, launch_rows<128, TGVKV_CACHE_INT4>);
        default: return by_dim(launch_rows<64, TGVKV_CACHE_FP4>, launch_rows<128, TGVKV_CACHE_FP4>);
    }
}

}  // namespace tgvkv
