// Attention of a few new tokens over the paged cache (a decode step, drafted
// tokens): the query rows of a set, n tokens x G heads, fit one 16-row tile.
//
//   o[t][h] = sum_{j <= len - n + i} softmax_j(scale <q[t][h], k_j>) v_j
//
// for token i of the n new tokens of its sequence (t = its row of q), over the
// slots j of set (b, h / G).  A row that sees no slot gives 0.
//
// HBM-bound: each slot's K and V row is read once, for up to 16 query rows (4
// d * 16 flops against 4 d bytes at most, far below the 278 flops a byte where
// the tensor cores would bound).  The sets' slots form one sequence of chunks
// (CH slots, never across a set); each warp of a persistent CTA takes one
// contiguous share of it, so ragged lengths and long caches split evenly.  A
// chunk moves as whole page slices by TMA into the warp's own two-stage ring,
// with the scale bytes and, at a segment's start, the query rows; the next
// chunk's page numbers are fetched one chunk ahead.
//
// Arithmetic per chunk on the tensor cores (mma.sync m16n8k16: bf16 operands,
// fp32 accumulation), which can take operands converted in registers:
//   S = Q K^T    integer K: a lane holds D / 4 consecutive values of a key
//                (whole scale groups), Q's fragments follow the same order;
//   O += P V     integer V: ldmatrix transposes pairs of slots; the values
//                they hold spread over neighbouring column tiles of O.
// Online softmax in base 2 (fp32); P is rounded to bf16 for the product, the
// normaliser sums the unrounded P.  A set inside one stream is written out at
// once; a split one leaves a partial (m, l, O) per stream, merged by a second
// kernel in stream order, so results do not depend on timing.
#include "cache_launch.h"
#include "launch.h"
#include "tc05.cuh"

namespace tgvkv {
namespace {

constexpr int kW = 8;                  // streams (warps) per CTA
constexpr int kStages = 2;
constexpr int kPlanSets = 2048;        // plan entries kept in shared memory

template <int D, int FMT>
struct StreamGeom {
    static constexpr int ROWB = FMT == TGVKV_CACHE_BF16 ? 2 * D : FMT == TGVKV_CACHE_INT8 ? D : D / 2;
    // slots per chunk: 4 KB of K and of V, at most 64
    static constexpr int CH = 4096 / ROWB > 64 ? 64 : 4096 / ROWB;
    static constexpr int KT = FMT == TGVKV_CACHE_BF16 ? D / 64 : 1;   // tiles of a row
    static constexpr int TROW = ROWB / KT;                            // bytes of a tile's row
    static constexpr int kTile = CH * TROW;
    static constexpr int SCB = FMT == TGVKV_CACHE_BF16 ? 0 : D / kGroup;   // scale bytes a row
    static constexpr int kK = 0;
    static constexpr int kV = KT * kTile;
    static constexpr int kKS = 2 * KT * kTile;
    static constexpr int kVS = kKS + CH * SCB;
    static constexpr int kQ = kVS + CH * SCB;
    static constexpr int kStage = (kQ + kStreamRows * 2 * D + 1023) & ~1023;
    static constexpr int kRing = kW * kStages * kStage;
};

// A chunk: slots [key0, key0 + n) of set s.
struct Chunk {
    int s, key0, n, first, last;
    int len, nq, tok0;
};

struct StreamTail {
    uint64_t full[kW][kStages];
    Chunk chunk[kW][kStages];
    int warp_sum[kW];
    int never;
    int pref[kPlanSets + 1];           // first chunk of entry e (a run of `run` sets)
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

// c += A B over one 16 x 8 x 16 tile.
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte unit u of row r in a tile that TMA wrote with the
// swizzle of its row length (128, 64 or 32 bytes).
template <int TROW>
__device__ __forceinline__ uint32_t swz(int r, int u) {
    constexpr int shift = TROW == 128 ? 0 : TROW == 64 ? 1 : 2;
    constexpr int mask = TROW / 16 - 1;
    return (uint32_t)(r * TROW + ((u ^ ((r >> shift) & mask)) << 4));
}

// Plain (untiled) copy of `bytes` (a multiple of 16, both sides aligned).
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes,
                                          uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            dst),
        "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}

// Chunks of a set: its last new token sees every slot.
template <int CH>
__device__ __forceinline__ int set_chunks(const SetSpan& sp) {
    return sp.n > 0 ? (sp.len + CH - 1) / CH : 0;
}

// A stream's walk over its chunks [c, c1) of the sequence.
template <int CH>
struct Walk {
    int s, at, left, chunks;           // set, next chunk in it, chunks left of the share
    SetSpan sp;

    __device__ __forceinline__ void load(const CacheProblem& p, const ChunkArgs& a) {
        sp = set_span(p, a, s);
        chunks = set_chunks<CH>(sp);
    }
    __device__ __forceinline__ void init(const CacheProblem& p, const ChunkArgs& a,
                                         const int* pref, int entries, int run, int c, int c1) {
        left = c1 - c;
        int lo = 0, hi = entries - 1;  // the last entry that starts at or before c
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pref[mid] <= c) lo = mid;
            else hi = mid - 1;
        }
        s = lo * run;
        at = c - pref[lo];
        load(p, a);
        while (at >= chunks) {         // c is below the total: a set holds it
            at -= chunks;
            if (++s >= p.S) {
                left = 0;
                return;
            }
            load(p, a);
        }
    }
    __device__ __forceinline__ bool next(const CacheProblem& p, const ChunkArgs& a, Chunk& c,
                                         bool& fresh) {
        if (left <= 0) return false;
        while (at >= chunks) {
            at = 0;
            if (++s >= p.S) return false;
            load(p, a);
            fresh = true;
        }
        c.s = s;
        c.key0 = at * CH;
        c.n = min(sp.len - c.key0, CH);
        c.first = fresh;
        c.last = at + 1 == chunks || left == 1;
        c.len = sp.len;
        c.nq = sp.n;
        c.tok0 = sp.tok0;
        fresh = false;
        ++at;
        --left;
        return true;
    }
};

// The copies of chunk c into one stage, spread over the warp's lanes.  Lane
// b < boxes holds the page number of the chunk's b-th page slice.
template <int D, int FMT>
__device__ __forceinline__ void issue(unsigned char* stage, uint64_t* bar, const Chunk& c, int page,
                                      int box, const CUtensorMap* mk, const CUtensorMap* mv,
                                      const CacheProblem& p, const CachePools& pool,
                                      const ChunkArgs& a, int lane) {
    using Gm = StreamGeom<D, FMT>;
    const int nb = (c.n + box - 1) / box;
    const int rows = c.nq * p.G;
    const uint32_t per_box = (uint32_t)box * (2 * Gm::ROWB + 2 * Gm::SCB);
    if (lane == 0)
        tc::mbar_arrive_expect_tx(bar, nb * per_box + (c.first ? (uint32_t)rows * 2 * D : 0u));
    __syncwarp();
    if (c.first && lane < rows) {
        const int i = lane / p.G, h = lane - i * p.G;
        const uint16_t* src = a.q + (long long)(c.tok0 + i) * a.q_tok +
                              (long long)((c.s % p.H_kv) * p.G + h) * a.q_head;
        bulk_copy(smem_u32(stage + Gm::kQ) + lane * 2 * D, src, 2 * D, bar);
    }
    if (lane < nb) {
        const int row = page * p.page + ((c.key0 + lane * box) & (p.page - 1));
        const uint32_t at = (uint32_t)(lane * box);
#pragma unroll
        for (int kt = 0; kt < Gm::KT; ++kt) {
            tc::tma_load_2d(stage + Gm::kK + kt * Gm::kTile + at * Gm::TROW, mk, 128 * kt, row, bar);
            tc::tma_load_2d(stage + Gm::kV + kt * Gm::kTile + at * Gm::TROW, mv, 128 * kt, row, bar);
        }
        if (FMT != TGVKV_CACHE_BF16) {
            const size_t off = (size_t)row * Gm::SCB;
            bulk_copy(smem_u32(stage + Gm::kKS) + at * Gm::SCB, pool.ks + off, box * Gm::SCB, bar);
            bulk_copy(smem_u32(stage + Gm::kVS) + at * Gm::SCB, pool.vs + off, box * Gm::SCB, bar);
        }
    }
}

// The page number of lane b's slice of chunk c (0 and the status bit where the
// table holds none).
__device__ __forceinline__ int chunk_page(const CacheProblem& p, const ChunkArgs& a, const Chunk& c,
                                          int box, int lane) {
    const int nb = (c.n + box - 1) / box;
    if (lane >= nb) return 0;
    return __ldg(a.page_table + (size_t)c.s * p.max_pages + ((c.key0 + lane * box) >> p.page_shift));
}
__device__ __forceinline__ int valid_page(const CacheProblem& p, int page, uint32_t* status) {
    if (page >= 0 && page < p.n_pages) return page;
    raise_status(status, TGVKV_STATUS_INDEX);
    return 0;
}

// The first of the two columns (dims) whose results a lane's c0 and c1 (rows g)
// hold in column tile t: dim of c0 is out_dim(t, tq), of c1 out_dim + step.
template <int D, int FMT>
__device__ __forceinline__ int out_dim(int t, int tq) {
    if (FMT == TGVKV_CACHE_BF16) return 8 * t + 2 * tq;
    if (FMT == TGVKV_CACHE_INT8) return 16 * (t >> 1) + 4 * tq + (t & 1);
    return 32 * (t >> 2) + 8 * tq + (t & 3);
}
template <int FMT>
constexpr int out_step() {
    return FMT == TGVKV_CACHE_BF16 ? 1 : FMT == TGVKV_CACHE_INT8 ? 2 : 4;
}

template <int D, int FMT>
__global__ void __launch_bounds__(kW * 32, 1)
chunk_stream_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                    const CacheProblem p, const CachePools pool, const ChunkArgs a, int box,
                    int min_chunks, int rec_rows, float* __restrict__ part,
                    long long* __restrict__ plan, uint32_t* __restrict__ status) {
    using Gm = StreamGeom<D, FMT>;
    constexpr int CH = Gm::CH;
    constexpr int KS = D / 16, ND = D / 8, NT = CH / 8, KK = CH / 16;
    griddep_launch_dependents();
    if (threadIdx.x == 0) {
        tc::tma_prefetch_desc(&mk);
        tc::tma_prefetch_desc(&mv);
    }
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    StreamTail& tl = *reinterpret_cast<StreamTail*>(ring + Gm::kRing);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) tl.never = 0;
    if (lane == 0) {
        for (int st = 0; st < kStages; ++st) tc::mbar_init(&tl.full[warp][st], 1);
        tc::fence_mbar_init();
    }
    if (blockIdx.x == 0) check_spans(p, a, tid, kW * 32, status);

    // ---- the plan: the first chunk of every entry (`run` consecutive sets)
    const int run = (p.S + kPlanSets - 1) / kPlanSets;
    const int entries = (p.S + run - 1) / run;
    constexpr int PER = kPlanSets / (kW * 32);       // entries a thread sums
    int cnt[PER], sum = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int e = tid * PER + u;
        cnt[u] = 0;
        if (e < entries)
            for (int s = e * run; s < min((e + 1) * run, p.S); ++s)
                cnt[u] += set_chunks<CH>(set_span(p, a, s));
        sum += cnt[u];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) tl.warp_sum[warp] = incl;
    __syncthreads();
    int base = incl - sum, total = 0;
    for (int w = 0; w < kW; ++w) {
        if (w < warp) base += tl.warp_sum[w];
        total += tl.warp_sum[w];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int e = tid * PER + u;
        if (e < entries) tl.pref[e] = base;
        if (blockIdx.x == 0 && e < entries) {        // the plan, for the merge kernel
            int at = base;
            for (int s = e * run; s < min((e + 1) * run, p.S); ++s) {
                plan[s] = at;
                at += run == 1 ? cnt[u] : set_chunks<CH>(set_span(p, a, s));
            }
        }
        base += cnt[u];
    }
    if (blockIdx.x == 0 && tid == 0) plan[p.S] = total;
    __syncthreads();

    const int n_streams = gridDim.x * kW;
    const int per = max((total + n_streams - 1) / n_streams, min_chunks);
    const int si = blockIdx.x * kW + warp;
    const long long c_lo = (long long)si * per;
    if (c_lo >= total) return;
    const int c0 = (int)c_lo, c1 = min(c0 + per, total);

    unsigned char* wring = ring + warp * kStages * Gm::kStage;
    Walk<CH> walk;
    bool fresh = true;
    walk.init(p, a, tl.pref, entries, run, c0, c1);
    Chunk nxt;
    bool more = walk.next(p, a, nxt, fresh);
    int nxt_page = more ? chunk_page(p, a, nxt, box, lane) : 0;
    int issued = 0;
    auto refill = [&]() {              // the next chunk into the stage just read
        const int st = issued % kStages;
        if (lane == 0) tl.chunk[warp][st] = nxt;
        issue<D, FMT>(wring + st * Gm::kStage, &tl.full[warp][st], nxt,
                      valid_page(p, nxt_page, status), box, &mk, &mv, p, pool, a, lane);
        ++issued;
        more = walk.next(p, a, nxt, fresh);
        if (more) nxt_page = chunk_page(p, a, nxt, box, lane);
    };
    for (int st = 0; st < kStages && more; ++st) refill();
    __syncwarp();

    const int g = lane >> 2, tq = lane & 3;
    uint32_t qa[KS][4];
    float o[ND][4];
    float m[2], l[2];
    int seg_chunk = c0;                // chunk index at which the current segment began
    int i = 0;
    for (; i < issued; ++i) {
        const int st = i % kStages;
        const bool got = tc::mbar_wait(&tl.full[warp][st], (i / kStages) & 1, &tl.never);
        if (!__all_sync(~0u, got)) break;
        const Chunk c = tl.chunk[warp][st];
        unsigned char* stage = wring + st * Gm::kStage;
        const uint32_t sb = smem_u32(stage);
        if (c.first) {
            seg_chunk = c0 + i;
            // Q fragments: pairs of dims in the order the K fragments have; 0 in
            // rows the tile does not have
            const int rows = c.nq * p.G;
            const uint32_t q0 = sb + Gm::kQ + g * 2 * D, q1 = q0 + 8 * 2 * D;
            if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    qa[s][0] = lds32(q0 + 32 * s + 4 * tq);
                    qa[s][1] = lds32(q1 + 32 * s + 4 * tq);
                    qa[s][2] = lds32(q0 + 32 * s + 16 + 4 * tq);
                    qa[s][3] = lds32(q1 + 32 * s + 16 + 4 * tq);
                }
            } else if (FMT == TGVKV_CACHE_INT8) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {       // 4 values: (0, 2) and (1, 3)
                    const uint2 x = lds64(q0 + tq * (D / 2) + 8 * s);
                    const uint2 y = lds64(q1 + tq * (D / 2) + 8 * s);
                    qa[s][0] = __byte_perm(x.x, x.y, 0x5410);
                    qa[s][1] = __byte_perm(y.x, y.y, 0x5410);
                    qa[s][2] = __byte_perm(x.x, x.y, 0x7632);
                    qa[s][3] = __byte_perm(y.x, y.y, 0x7632);
                }
            } else {
#pragma unroll
                for (int w = 0; w < KS / 2; ++w) {   // 8 values: (0, 4) (1, 5), (2, 6) (3, 7)
                    const uint4 x = lds128(q0 + tq * (D / 2) + 16 * w);
                    const uint4 y = lds128(q1 + tq * (D / 2) + 16 * w);
                    qa[2 * w][0] = __byte_perm(x.x, x.z, 0x5410);
                    qa[2 * w][1] = __byte_perm(y.x, y.z, 0x5410);
                    qa[2 * w][2] = __byte_perm(x.x, x.z, 0x7632);
                    qa[2 * w][3] = __byte_perm(y.x, y.z, 0x7632);
                    qa[2 * w + 1][0] = __byte_perm(x.y, x.w, 0x5410);
                    qa[2 * w + 1][1] = __byte_perm(y.y, y.w, 0x5410);
                    qa[2 * w + 1][2] = __byte_perm(x.y, x.w, 0x7632);
                    qa[2 * w + 1][3] = __byte_perm(y.y, y.w, 0x7632);
                }
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (g >= rows) qa[s][0] = qa[s][2] = 0u;
                if (g + 8 >= rows) qa[s][1] = qa[s][3] = 0u;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) m[e] = -INFINITY, l[e] = 0.f;
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][e] = 0.f;
        }
        // ---- S = Q K^T; column tile j holds slots 8j .. 8j + 7
        float sc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
            // two tiles x two halves of the dims: four independent chains
            float acc[2][2][4];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x][y][e] = 0.f;
            if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                for (int u = 0; u < KS / 2; ++u) {
                    const int unit = 4 * u + (lane >> 3);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint32_t r[4];
                        ldsm_x4(sb + Gm::kK + (unit >> 3) * Gm::kTile +
                                    swz<128>(8 * (j + x) + (lane & 7), unit & 7),
                                r);
                        mma(acc[x][u & 1], qa[2 * u], r[0], r[1]);
                        mma(acc[x][u & 1], qa[2 * u + 1], r[2], r[3]);
                    }
                }
            } else {
                constexpr int NW = Gm::ROWB / 16;    // words of codes a lane holds of a row
                uint32_t w[2][NW], kb[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 8 * (j + x) + g;
                    if (NW == 2) {
                        const uint2 t = lds64(sb + Gm::kK + swz<Gm::TROW>(row, tq >> 1) + (tq & 1) * 8);
                        w[x][0] = t.x, w[x][1 % NW] = t.y;
                    } else {
#pragma unroll
                        for (int b = 0; b < NW / 4; ++b) {
                            const uint4 t =
                                lds128(sb + Gm::kK + swz<Gm::TROW>(row, tq * (NW / 4) + b));
                            w[x][(4 * b) % NW] = t.x, w[x][(4 * b + 1) % NW] = t.y;
                            w[x][(4 * b + 2) % NW] = t.z, w[x][(4 * b + 3) % NW] = t.w;
                        }
                    }
                    kb[x] = lds8(sb + Gm::kKS + row * Gm::SCB + (D == 128 ? tq : tq >> 1));
                    kb[x] = both(FMT == TGVKV_CACHE_INT8 ? scale_bf16(kb[x]) : int4_base(kb[x]));
                }
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint32_t b0, b1;
                        if (FMT == TGVKV_CACHE_INT8) {
                            b0 = bf16x2_mul(int8x2_to_bf16(w[x][s % NW]), kb[x]);
                            b1 = bf16x2_mul(int8x2_to_bf16(w[x][s % NW] >> 8), kb[x]);
                        } else {
                            b0 = int4x2_to_bf16(w[x][(s / 2) % NW] >> (8 * (s & 1)), kb[x]);
                            b1 = int4x2_to_bf16(w[x][(s / 2) % NW] >> (8 * (s & 1) + 4), kb[x]);
                        }
                        mma(acc[x][s & 1], qa[s], b0, b1);
                    }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc[j + x][e] = (acc[x][0][e] + acc[x][1][e]) * p.scale_log2;
        }
        // ---- hide what a row must not see: slots from its token's on
        if (c.n < CH || c.key0 + CH > c.len - c.nq + 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int lim = min(c.len - c.nq + (g + 8 * h) / p.G + 1 - c.key0, c.n);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (8 * j + 2 * tq + e >= lim) sc[j][2 * h + e] = -INFINITY;
            }
        }
        // ---- online softmax of rows g and g + 8 (the 4 lanes of a row share it)
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float cm = fmaxf(sc[0][2 * h], sc[0][2 * h + 1]);
#pragma unroll
            for (int j = 1; j < NT; ++j) cm = fmaxf(cm, fmaxf(sc[j][2 * h], sc[j][2 * h + 1]));
            cm = fmaxf(cm, __shfl_xor_sync(~0u, cm, 1));
            cm = fmaxf(cm, __shfl_xor_sync(~0u, cm, 2));
            const float mn = fmaxf(m[h], cm);
            const float ref = mn == -INFINITY ? 0.f : mn;   // nothing seen yet: all weights 0
            alpha[h] = fast_exp2(m[h] - ref);
            float ps = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sc[j][2 * h + e] = fast_exp2(sc[j][2 * h + e] - ref);
                    ps += sc[j][2 * h + e];
                }
            l[h] = l[h] * alpha[h] + ps;
            m[h] = mn;
        }
        if (__any_sync(~0u, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
            for (int t = 0; t < ND; ++t) {
                o[t][0] *= alpha[0], o[t][1] *= alpha[0];
                o[t][2] *= alpha[1], o[t][3] *= alpha[1];
            }
        }
        // ---- slots past the set's end hold what the pool holds there: their
        // weights are 0, and 0 x NaN is not, so V must be 0 (integer V: scale 0)
        if (FMT == TGVKV_CACHE_BF16 && c.n < CH) {
            const int end = (c.n + 15) & ~15;
            for (int x = lane; x < (end - c.n) * 8 * Gm::KT; x += 32) {
                const int r = c.n + x / (8 * Gm::KT), u = x % (8 * Gm::KT);
                *reinterpret_cast<uint4*>(stage + Gm::kV + (u >> 3) * Gm::kTile + r * 128 + (u & 7) * 16) =
                    make_uint4(0u, 0u, 0u, 0u);
            }
            tc::fence_proxy_async_smem();   // before TMA writes the stage again
            __syncwarp();
        }
        // ---- O += P V over 16 slots at a time
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (16 * kk >= c.n) break;
            const uint32_t pa[4] = {pack_bf16x2(sc[2 * kk][0], sc[2 * kk][1]),
                                    pack_bf16x2(sc[2 * kk][2], sc[2 * kk][3]),
                                    pack_bf16x2(sc[2 * kk + 1][0], sc[2 * kk + 1][1]),
                                    pack_bf16x2(sc[2 * kk + 1][2], sc[2 * kk + 1][3])};
            const int row = 16 * kk + (lane & 7) + ((lane >> 3) & 1) * 8;
            // scales of this lane's slot pairs (2 tq, + 1) and (2 tq + 8, + 9), by group
            constexpr int NG = D / kGroup;
            uint32_t vs[2][NG];
            if (FMT != TGVKV_CACHE_BF16) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k0 = 16 * kk + 2 * tq + 8 * h;
                    uint32_t w0, w1;
                    if (D == 128) {
                        const uint2 t = lds64(sb + Gm::kVS + k0 * 4);
                        w0 = t.x, w1 = t.y;
                    } else {
                        const uint32_t t = lds32(sb + Gm::kVS + k0 * 2);
                        w0 = t & 0xFFFFu, w1 = t >> 16;
                    }
                    if (k0 >= c.n) w0 = 0u;
                    if (k0 + 1 >= c.n) w1 = 0u;
#pragma unroll
                    for (int x = 0; x < NG; ++x) {
                        const uint32_t both_e =
                            __byte_perm(w0, w1, (x << 4) | ((4 + x) << 12)) >> 1 & 0x7F807F80u;
                        vs[h][x] = FMT == TGVKV_CACHE_INT8
                                       ? both_e
                                       : __vminu2(both_e + 0x03800380u, 0x7F807F80u);
                    }
                }
            }
#pragma unroll
            for (int u2 = 0; u2 < Gm::ROWB / 32; ++u2) {
                const int unit = 2 * u2 + (lane >> 4);
                uint32_t r[4];
                ldsm_x4_trans(sb + Gm::kV + (unit / (Gm::TROW / 16)) * Gm::kTile +
                                  swz<Gm::TROW>(row, unit % (Gm::TROW / 16)),
                              r);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int u = 2 * u2 + x;        // 16-byte unit of the row
                    const uint32_t r0 = r[2 * x], r1 = r[2 * x + 1];
                    if (FMT == TGVKV_CACHE_BF16) {
                        mma(o[u], pa, r0, r1);
                    } else if (FMT == TGVKV_CACHE_INT8) {
                        const uint32_t s0 = vs[0][(u / 2) % NG], s1 = vs[1][(u / 2) % NG];
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            mma(o[(2 * u + y) % ND], pa, bf16x2_mul(int8x2_to_bf16(r0 >> (8 * y)), s0),
                                bf16x2_mul(int8x2_to_bf16(r1 >> (8 * y)), s1));
                    } else {
                        const uint32_t s0 = vs[0][u % NG], s1 = vs[1][u % NG];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            mma(o[(4 * u + y) % ND], pa, int4x2_to_bf16(r0 >> (4 * y), s0),
                                int4x2_to_bf16(r1 >> (4 * y), s1));
                    }
                }
            }
        }
        __syncwarp();                  // the stage is read: refill it
        if (more) refill();
        if (!c.last) continue;
        // ---- the segment of set c.s is complete
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(~0u, l[h], 1);
            l[h] += __shfl_xor_sync(~0u, l[h], 2);
        }
        const int rows = c.nq * p.G;
        const bool whole = seg_chunk == c0 + i - c.key0 / CH && c.key0 + CH >= c.len;
        const int gk = c.s % p.H_kv;
        float* pp = part + ((size_t)si * 2 + (seg_chunk == c0 ? 0 : 1)) *
                               (size_t)chunk_record_floats(rec_rows, D);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h;
            if (r >= rows) continue;
            if (whole) {               // the whole set: written out
                const float inv = l[h] > 0.f ? 1.f / l[h] : (l[h] == l[h] ? 0.f : l[h]);
                const int t = r / p.G, hh = r - t * p.G;
                uint16_t* op = a.out + ((size_t)(c.tok0 + t) * p.H_q + gk * p.G + hh) * D;
                if (FMT == TGVKV_CACHE_BF16) {
#pragma unroll
                    for (int t8 = 0; t8 < ND; ++t8)
                        *reinterpret_cast<uint32_t*>(op + 8 * t8 + 2 * tq) =
                            pack_bf16x2(o[t8][2 * h] * inv, o[t8][2 * h + 1] * inv);
                } else if (FMT == TGVKV_CACHE_INT8) {
#pragma unroll
                    for (int u = 0; u < ND / 2; ++u)
                        *reinterpret_cast<uint2*>(op + 16 * u + 4 * tq) = make_uint2(
                            pack_bf16x2(o[2 * u][2 * h] * inv, o[2 * u + 1][2 * h] * inv),
                            pack_bf16x2(o[2 * u][2 * h + 1] * inv, o[2 * u + 1][2 * h + 1] * inv));
                } else {
#pragma unroll
                    for (int u = 0; u < ND / 4; ++u)
                        *reinterpret_cast<uint4*>(op + 32 * u + 8 * tq) = make_uint4(
                            pack_bf16x2(o[4 * u][2 * h] * inv, o[4 * u + 1][2 * h] * inv),
                            pack_bf16x2(o[4 * u + 2][2 * h] * inv, o[4 * u + 3][2 * h] * inv),
                            pack_bf16x2(o[4 * u][2 * h + 1] * inv, o[4 * u + 1][2 * h + 1] * inv),
                            pack_bf16x2(o[4 * u + 2][2 * h + 1] * inv, o[4 * u + 3][2 * h + 1] * inv));
                }
            } else {
                float* op = pp + r * D;
#pragma unroll
                for (int t8 = 0; t8 < ND; ++t8) {
                    op[out_dim<D, FMT>(t8, tq)] = o[t8][2 * h];
                    op[out_dim<D, FMT>(t8, tq) + out_step<FMT>()] = o[t8][2 * h + 1];
                }
                if (tq == 0) {
                    pp[rec_rows * D + r] = m[h];
                    pp[rec_rows * D + rec_rows + r] = l[h];
                }
            }
        }
    }
    if (i < issued) {
        // a wait gave up: report it and let the copies in flight land
        if (lane == 0) raise_status(status, TGVKV_STATUS_TIMEOUT);
        for (; i < issued; ++i)
            if (!tc::mbar_wait(&tl.full[warp][i % kStages], (i / kStages) & 1, &tl.never)) break;
    }
}

// The split sets' merge and the rows that see nothing: one warp per (set, query
// row), a programmatic dependent of the stream kernel.  A set's partials are
// combined in stream order.
template <int D>
__global__ void __launch_bounds__(128)
chunk_stream_merge(const CacheProblem p, const ChunkArgs a, int n_streams, int min_chunks,
                   int rec_rows, const float* __restrict__ part,
                   const long long* __restrict__ plan) {
    constexpr int DPL = D / 32;
    const int lane = threadIdx.x & 31;
    const long long gw = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int s = (int)(gw / rec_rows), r = (int)(gw % rec_rows);
    SetSpan sp{0, 0, 0};
    if (s < p.S) sp = set_span(p, a, s);
    griddep_wait();
    if (s >= p.S || r >= sp.n * p.G) return;
    const int c0 = (int)__ldcg(plan + s), c1 = (int)__ldcg(plan + s + 1);
    const int total = (int)__ldcg(plan + p.S);
    float acc[DPL];
#pragma unroll
    for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
    if (c1 > c0) {
        const int per = max((total + n_streams - 1) / n_streams, min_chunks);
        const int w0 = c0 / per, w1 = (c1 - 1) / per;
        if (w0 == w1) return;          // inside one stream: written by it
        // a segment starts its stream's share, but for a set that begins inside it
        const int first = c0 != w0 * per ? 1 : 0;
        const size_t rec = chunk_record_floats(rec_rows, D);
        merge_records<D>(w1 - w0 + 1, rec_rows, r, [&](int i) {
            return part + ((size_t)(w0 + i) * 2 + (i == 0 ? first : 0)) * rec;
        }, acc);
    }
    const int t = r / p.G, hh = r - t * p.G;
    uint16_t* out = a.out + ((size_t)(sp.tok0 + t) * p.H_q + (s % p.H_kv) * p.G + hh) * D + DPL * lane;
#pragma unroll
    for (int c = 0; c < DPL; c += 2)
        *reinterpret_cast<uint32_t*>(out + c) = pack_bf16x2(acc[c], acc[(c + 1) % DPL]);
}

// Chunks a stream takes at least: below this, splitting costs more than it saves.
constexpr int kMinChunks = 2;

template <int D, int FMT>
cudaError_t launch_stream(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                          float* part, long long* plan, uint32_t* status, cudaStream_t stream) {
    using Gm = StreamGeom<D, FMT>;
    const int box = p.page < Gm::CH ? p.page : Gm::CH;
    alignas(64) CUtensorMap mk, mv;
    const uint64_t rows = (uint64_t)p.n_pages * p.page;
    const int box_bytes = FMT == TGVKV_CACHE_BF16 ? 128 : Gm::ROWB;
    if (!make_pool_map(&mk, pool.k, rows, Gm::ROWB, box_bytes, box) ||
        !make_pool_map(&mv, pool.v, rows, Gm::ROWB, box_bytes, box))
        return cudaErrorInvalidValue;
    const size_t smem = 1024 + Gm::kRing + sizeof(StreamTail);
    static_assert(1024 + Gm::kRing + sizeof(StreamTail) <= 227 * 1024, "shared memory of one CTA");
    cudaError_t e = cudaFuncSetAttribute(chunk_stream_kernel<D, FMT>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int ctas = sms < kStreamMax / kW ? sms : kStreamMax / kW;
    const int rec_rows = a.max_q * p.G;
    chunk_stream_kernel<D, FMT><<<ctas, kW * 32, smem, stream>>>(mk, mv, p, pool, a, box, kMinChunks,
                                                                 rec_rows, part, plan, status);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const long long warps = (long long)p.S * rec_rows;
    return launch_dependent(chunk_stream_merge<D>, dim3((unsigned)((warps + 3) / 4)), dim3(128), 0,
                            stream, p, a, ctas * kW, (int)kMinChunks, rec_rows,
                            static_cast<const float*>(part), static_cast<const long long*>(plan));
}

}  // namespace

cudaError_t launch_chunk_stream(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                                float* part, long long* plan, uint32_t* status, cudaStream_t stream) {
    if (p.d == 64) {
        if (p.format == TGVKV_CACHE_BF16)
            return launch_stream<64, TGVKV_CACHE_BF16>(p, pool, a, part, plan, status, stream);
        if (p.format == TGVKV_CACHE_INT8)
            return launch_stream<64, TGVKV_CACHE_INT8>(p, pool, a, part, plan, status, stream);
        return launch_stream<64, TGVKV_CACHE_INT4>(p, pool, a, part, plan, status, stream);
    }
    if (p.format == TGVKV_CACHE_BF16)
        return launch_stream<128, TGVKV_CACHE_BF16>(p, pool, a, part, plan, status, stream);
    if (p.format == TGVKV_CACHE_INT8)
        return launch_stream<128, TGVKV_CACHE_INT8>(p, pool, a, part, plan, status, stream);
    return launch_stream<128, TGVKV_CACHE_INT4>(p, pool, a, part, plan, status, stream);
}

}  // namespace tgvkv
