// Attention of a chunk of new tokens over the paged cache on the 5th-generation
// tensor cores (tcgen05), for sets with more query rows than the row streams take
// (stream_rows()).
//
//   o[t][h] = sum_{j <= len - n + i} softmax_j(scale <q[t][h], k_j>) v_j
//
// A row tile is 128 query rows of a set: tpt = floor(128 / G) whole tokens times
// the G query heads of the KV head, so every row of a tile reads the same K
// and V.  Two groups of four softmax warps (thread = row) work in ping-pong, so
// that the tensor cores have one group's products while the other does its
// exponentials.  Their two streams are, by the call's longest chunk,
//   PAIR   two consecutive row tiles over the same key tiles (each K / V tile is
//          loaded once for 256 rows), when a chunk spans several row tiles;
//   SPLIT  alternate key tiles of one row tile, joined at the segment's end
//          (each group reading half of both O accumulators from TMEM).
// A unit of work is one 128-slot key tile of an item (a row tile, or a pair);
// each persistent CTA takes one contiguous share of the units of all items, so
// ragged chunks, ragged lengths and single long caches all split evenly.  An item
// that spans a few CTAs is joined by the one that begins it: that is the last
// segment of its share, and the first of the others', whose partial (m, l, O) is
// there by then (a flag per warp; shares are handed out by a ticket in descending
// order, so that a CTA only ever waits for CTAs that started before it).  An item
// that spans many leaves all its partials to a second kernel.  Both join in CTA
// order.
//
// Tensor memory: one S (128 columns), P0, P1 (64 columns each: 128 bf16), O0, O1
// (D columns each).  A softmax thread takes its row of S into registers and frees
// the columns at once, so the groups share S: the tensor cores run P V of one
// group while the other reads, and Q K^T never waits for an exponential.  The
// products are issued in one order,
//   ... P0 V (j), Q0 K (j + 1), P1 V (j), Q1 K (j + 1) ...
// so that a group's S (j + 1) tells that its O holds tile j.  P is the A operand
// from tensor memory; K is the K-major and V the MN-major B operand from shared
// memory.
//
// Integer caches: TMA brings the codes of a key tile, eight converter warps write
// them as bf16 in the swizzled layout (exact: scales are powers of two), and the rest
// is the bf16 kernel.
//
// Roles: warps 0 and 2 TMA (Q and K; V), warp 1 MMA issue and tensor memory, warp 3
// rows that see nothing, warps 4-11 softmax, warps 12-19 converters (integer caches).
// Registers are split by role (setmaxnreg), so that a softmax thread holds a whole
// row of S.  P is rounded to bf16 for its product and the normaliser sums it
// unrounded; m, l and O stay in fp32; O is rescaled only when a row's maximum rises by
// more than 2^8.  Every wait is bounded; a timeout sets TGVKV_STATUS_TIMEOUT and the
// CTA unwinds after its copies and MMAs finished.
//
// What bounds it.  bf16, long chunks: the tensor cores under the power limit (28 heads,
// 2048 tokens over 34816 slots: 651 us, 1525 TFLOP/s, call after call, where a dense
// bf16 product holds 1685; 600 us in a burst of a dozen calls).  Integer caches: no unit
// is full (6 x 0 .. 500 tokens over 2001 .. 4000 slots, int8: tensor pipe 36%, integer pipe
// 43%, shared-memory wavefronts 30%, an instruction issued in half the cycles): a key
// tile passes from the copy to the converters to the products, and every pair of row
// tiles brings and converts its set's tiles again (16 x 0 .. 500 tokens over 4451 .. 8900 slots:
// int8 365 us, bf16 296).  One row tile a set: latency (256 sets of 0 .. 96 tokens over 1553 ..
// 3104 slots: int8 65 us, bf16 60 us, 4.6 TB/s): the end of a segment leaves the tensor cores
// idle for about 3 us, which only other work on the SM could fill, and there is no room
// for a second CTA.
//
// Measured and not kept: one thread as the issuer (chunks over 34816 slots 763 us
// against 627, in a burst); one producer warp; four converter warps (16 x 0 .. 500 tokens, int4
// pages: 389 us against 360) and converters that load the next tile before they store
// this one; deeper rings at d = 64; the next segment's place looked up before the
// last products end (SPLIT 1% faster, PAIR 2% slower).
#pragma once

#include "cache_launch.h"
#include "launch.h"
#include "tc05.cuh"

namespace tgvkv {

constexpr int kSoftWarp = 4;           // first softmax warp
constexpr int kConvWarp = 12;          // first converter warp
constexpr uint32_t kPCol = 128, kOCol = 256;   // first P and O columns; S at 0
constexpr float kRescale = 8.f;        // a stale maximum may trail by 2^8

// The issuing warps run as a whole, so that addresses stay in uniform registers;
// one elected lane issues.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r;
}
// D[tmem] (+)= A[smem] * B[smem]^T.  Of a descriptor only the low word (the address)
// changes between the instructions of a tile: an add and no carry.  `leader`: a
// predicate and no branch, so that the warp's operands stay uniform.
template <int ACC>
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo,
                                       uint32_t a_hi, uint32_t b_hi, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
        "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %4};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(a_hi), "r"(b_hi), "r"(idesc), "n"(ACC), "r"(leader)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem,
                                       uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                       uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void commit(uint32_t leader, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
            smem_u32(bar)),
        "r"(leader)
        : "memory");
}

// Store 16 consecutive 32-bit columns of this thread's TMEM lane (warp-wide).
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// 16 consecutive 32-bit columns of this thread's TMEM lane (warp-wide).
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
          "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
          "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D, int FMT, bool PAIR>
struct TileGeom {
    static constexpr bool QUANT = FMT != TGVKV_CACHE_BF16;
    static constexpr int TILE = D * 2 * TN;                       // bytes of a bf16 K or V tile
    static constexpr int HALF = TN * 128;                         // bytes of its 64-dim half
    static constexpr int NST = D == 64 ? 6 : QUANT ? 3 : PAIR ? 5 : 4;   // ring slots
    static constexpr int ROWB = FMT == TGVKV_CACHE_INT8 ? D : D / 2;   // stored bytes a row
    static constexpr int RAW = TN * ROWB, SC = TN * (D / kGroup); // raw tile, its scale bytes
    static constexpr int NRAW = QUANT ? (FMT == TGVKV_CACHE_INT8 ? 3 : 6) : 0;
    static constexpr int NQ = PAIR && D == 128 ? 1 : 2;           // Q slots (what there is room for)
    static constexpr int QT = PAIR ? 2 : 1;                       // row tiles a slot
    // What an item's start and end cost, in key tiles: the shares are of equal cost.  SPLIT
    // (the groups' join besides): 256 sets of 0 .. 96 tokens over 1553 .. 3104 slots take (int8, us)
    // 68.6 at 0, 67.6 at 2, 64.5 at 3, 66.6 at 4; at d = 64 54.3, 53.1, 49.2, 52.2 and 48.2 at 6.
    // PAIR: 0 .. 500 tokens of 16 sequences over 1001 .. 2000 slots 125 at 0, 114 at 2, 112 at 3.
    static constexpr int START = PAIR || D == 128 ? 3 : 6;
    static constexpr int CW = QUANT ? 8 : 0;                      // converter warps
    static constexpr int THREADS = 32 * (kConvWarp + CW);
    // registers a thread: at launch (the most that the thread count allows), then by
    // role.  The roles' sum is at most the launch's: what setmaxnreg raises one by has
    // to come from the others.
    static constexpr int LAUNCH_REGS = QUANT ? 96 : 168;
    static constexpr int FEW_REGS = QUANT ? 64 : 72, CONV_REGS = 40, SOFT_REGS = QUANT ? 168 : 208;
    static_assert(128 * FEW_REGS + 256 * SOFT_REGS + 32 * CW * CONV_REGS <= THREADS * LAUNCH_REGS,
                  "register split");
};

template <int N>
__device__ __forceinline__ void regs_down() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_up() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// ---- the work ----------------------------------------------------------------
// A segment: key tiles [j0, j1) of item u of set s.
struct Seg {
    SetSpan sp;
    int s, u, j0, j1, nk;              // nk: key tiles of the item
    int tok0;                          // the item's first token within the chunk
    bool starts;                       // begins the CTA's share
};

template <int START>
struct TileWalk {
    SetSpan sp;
    int s, u, j, left;
    bool first;

    __device__ __forceinline__ void init(const CacheProblem& p, const ChunkArgs& a, int s_, int u_,
                                         int j_, int units) {
        s = s_;
        u = u_;
        j = j_;
        left = units;
        first = true;
        if (left > 0) sp = set_span(p, a, s);
    }
    __device__ __forceinline__ bool next(const CacheProblem& p, const ChunkArgs& a,
                                         const TilePlan& pl, Seg& g) {
        while (left > 0) {
            int nk = tiles_seen(sp, (u + 1) * pl.tpi);
            while (u * pl.tpi >= sp.n || j >= item_units(nk, START)) {
                j = 0;
                if (u * pl.tpi >= sp.n || ++u * pl.tpi >= sp.n) {
                    u = 0;
                    if (++s >= p.S) return false;
                    sp = set_span(p, a, s);
                }
                nk = tiles_seen(sp, (u + 1) * pl.tpi);
            }
            const int j1 = min(item_units(nk, START), j + left);
            g.j0 = max(j - START, 0);
            g.j1 = j1 - START;
            left -= j1 - j;
            j = j1;
            if (g.j1 <= g.j0) continue;
            g.sp = sp;
            g.s = s;
            g.u = u;
            g.nk = nk;
            g.tok0 = u * pl.tpi;
            g.starts = first;
            first = false;
            return true;
        }
        return false;
    }
};

template <int D, int FMT, bool PAIR>
struct TileSmem {
    using Gm = TileGeom<D, FMT, PAIR>;
    unsigned char q[Gm::NQ * Gm::QT][D * 2 * TM];     // 64 dims each, 128-byte swizzled rows
    unsigned char kv[Gm::NST][Gm::TILE];              // the ring, in MMA order
    unsigned char raw[Gm::QUANT ? Gm::NRAW : 1][Gm::QUANT ? Gm::RAW : 16];
    unsigned char sc[Gm::QUANT ? Gm::NRAW : 1][Gm::QUANT ? Gm::SC : 16];
    uint64_t full[Gm::NST], empty[Gm::NST];
    uint64_t raw_full[Gm::QUANT ? Gm::NRAW : 1], raw_empty[Gm::QUANT ? Gm::NRAW : 1];
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_done[2], s_free;
    uint64_t join_in, join_out, mma_done;
    float2 ml[PAIR ? 1 : 2][PAIR ? 1 : TM];           // SPLIT: the groups' (m, l)
    struct {                                          // a softmax warp's place in the work:
        TileWalk<Gm::START> walk;                     // here, as its registers hold S
        Seg g;
    } at[8];
    uint32_t tmem_base;
    int abort_flag, never;
    int filled[Gm::QUANT ? Gm::NRAW : Gm::NST];       // the last copy into each slot (-1: none)
    int live[Gm::QUANT ? Gm::NRAW : 1];               // and the slots of the set in it
    long long warp_sum[Gm::THREADS / 32];
    int start_s, start_u, start_j, share, tiles;
};

// Row tile w of a segment's item (PAIR), or its one row tile: its key tiles.
template <bool PAIR>
__device__ __forceinline__ int group_tiles(const Seg& g, const TilePlan& pl, int w) {
    if (!PAIR) return g.nk;
    const int t = g.tok0 + w * pl.tpt;
    return t < g.sp.n ? tiles_seen(g.sp, t + pl.tpt) : 0;
}

// Places of K and V of key tile x (counted from the segment's first, of n) in the
// order of the ring.  PAIR: K0 V0 K1 V1 ...; SPLIT: K0 K1 V0 K2 V1 ...
template <bool PAIR>
__device__ __forceinline__ int k_place(int x) {
    return PAIR ? 2 * x : max(2 * x - 1, 0);
}
template <bool PAIR>
__device__ __forceinline__ int v_place(int x, int n) {
    return PAIR ? 2 * x + 1 : min(2 * x + 2, 2 * n - 1);
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
    return __all_sync(~0u, tc::mbar_wait(bar, parity, abort));
}

// A warp's part of a record is written / is awaited and taken (the flag is down
// again for the next call).  The wait is bounded like those on mbarriers.
__device__ __forceinline__ void give_flag(uint32_t* flag, int lane) {
    __threadfence();
    __syncwarp();
    if (lane == 0) atomicExch(flag, 1u);
}
__device__ __forceinline__ bool take_flag(uint32_t* flag, int lane, volatile int* abort) {
    int got = 1;
    if (lane == 0) {
        const long long t0 = clock64();
        while ((got = atomicExch(flag, 0u) == 1u) == 0)
            if (*abort || clock64() - t0 > tc::kWaitLimitCycles) break;
        __threadfence();
    }
    return __shfl_sync(~0u, got, 0) != 0;
}

template <int D, int FMT, bool PAIR>
__global__ void __launch_bounds__(TileGeom<D, FMT, PAIR>::THREADS, 1)
chunk_tile_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                  const __grid_constant__ CUtensorMap mv, const CacheProblem p,
                  const CachePools pool, const ChunkArgs a, const TilePlan pl,
                  float* __restrict__ part, SplitItem* __restrict__ split,
                  uint32_t* __restrict__ sync, uint32_t* __restrict__ status) {
    using Gm = TileGeom<D, FMT, PAIR>;
    constexpr bool QUANT = Gm::QUANT;
    constexpr int NST = Gm::NST, NRAW = QUANT ? Gm::NRAW : 1, START = Gm::START;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    TileSmem<D, FMT, PAIR>& sm = *reinterpret_cast<TileSmem<D, FMT, PAIR>*>(
        smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        sm.abort_flag = 0;
        sm.never = 0;
        sm.tiles = 0;
        for (int i = 0; i < (QUANT ? NRAW : NST); ++i) sm.filled[i] = -1;
        for (int i = 0; i < NST; ++i) {
            tc::mbar_init(&sm.full[i], QUANT ? Gm::CW : 1);
            tc::mbar_init(&sm.empty[i], 1);
        }
        for (int i = 0; i < NRAW; ++i) {
            tc::mbar_init(&sm.raw_full[i], 1);
            tc::mbar_init(&sm.raw_empty[i], QUANT ? Gm::CW : 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&sm.q_full[i], 1);
            tc::mbar_init(&sm.q_empty[i], 1);
            tc::mbar_init(&sm.s_full[i], 1);
            tc::mbar_init(&sm.p_full[i], 4);
            tc::mbar_init(&sm.o_done[i], 1);
        }
        tc::mbar_init(&sm.join_in, 8);
        tc::mbar_init(&sm.join_out, 8);
        tc::mbar_init(&sm.s_free, 4);
        tc::mbar_init(&sm.mma_done, 1);
        tc::fence_mbar_init();
        tc::tma_prefetch_desc(&mq);
        if (!QUANT) {
            tc::tma_prefetch_desc(&mk);
            tc::tma_prefetch_desc(&mv);
        }
    }
    // The kernels before have finished; the merge may start from now on (and waits in turn).
    griddep_wait();
    griddep_launch_dependents();
    if (warp == 1) {                   // (not before: a kernel still at work may yet want its own)
        tc::tmem_alloc(&sm.tmem_base, 512);
        tc::tmem_relinquish();
    }
    if (tid == 0) sm.share = take_share(sync, status);
    if (blockIdx.x == 0) check_spans(p, a, tid, Gm::THREADS, status);

    // ---- this CTA's share: units [c0, c0 + count) of all
    const int run = (p.S + Gm::THREADS - 1) / Gm::THREADS;    // sets a thread sums
    const int s_lo = min(tid * run, p.S), s_hi = min(s_lo + run, p.S);
    long long sum = 0;
    for (int s = s_lo; s < s_hi; ++s) sum += set_units(set_span(p, a, s), pl, START);
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) sm.warp_sum[warp] = incl;
    __syncthreads();
    long long base = incl - sum, total = 0;
#pragma unroll
    for (int w = 0; w < Gm::THREADS / 32; ++w) {
        if (w < warp) base += sm.warp_sum[w];
        total += sm.warp_sum[w];
    }
    const long long per = (total + gridDim.x - 1) / gridDim.x;
    const int share = sm.share;        // written before the barrier above
    const long long c0 = share * per;
    const int count = (int)max(min(total - c0, per), 0ll);
    if (c0 < base + sum && c0 + count > base) {          // my sets hold some of them
        int tiles = 0;
        long long at = base - c0;      // the item's first unit, counted from the share's
        for (int s = s_lo; s < s_hi; ++s) {
            const SetSpan sp = set_span(p, a, s);
            for (int u = 0; u * pl.tpi < sp.n; ++u) {
                const int n = item_units(tiles_seen(sp, (u + 1) * pl.tpi), START);
                const long long lo = max(at, 0ll), hi = min(at + n, (long long)count);
                if (lo < hi) {
                    tiles += (int)(max(hi - at - START, 0ll) - max(lo - at - START, 0ll));
                    if (lo == 0) {
                        sm.start_s = s;
                        sm.start_u = u;
                        sm.start_j = (int)-at;
                    }
                }
                at += n;
            }
        }
        if (tiles > 0) atomicAdd(&sm.tiles, tiles);
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    volatile int* abort_flag = &sm.abort_flag;
    auto begin = [&](TileWalk<START>& walk) {
        walk.init(p, a, count > 0 ? sm.start_s : 0, count > 0 ? sm.start_u : 0,
                  count > 0 ? sm.start_j : 0, count);
    };

    if (warp < kSoftWarp) {
        regs_down<Gm::FEW_REGS>();

        // ------------------------------------------------------------ producers
        // Warp 0 brings Q and K, warp 2 brings V: a single one takes longer to issue a key
        // tile's copies than the tile's products take.
        if (warp == 0 || warp == 2) {
            const bool is_v = warp == 2;
            const int box = min(p.page, TN);         // slots of a page slice of a key tile
            const uint32_t q_bytes = (uint32_t)(D / 64) * 128u * (uint32_t)(pl.tpt * p.G);
            const uint8_t* codes = is_v ? pool.v : pool.k;
            const uint8_t* scales = is_v ? pool.vs : pool.ks;
            const CUtensorMap* map = is_v ? &mv : &mk;
            constexpr int N = QUANT ? NRAW : NST;
            // lane b (and 16 + b): page slice b of the tile
            const int b = lane & 15;
            int base_it = 0, ns = 0, nq[2] = {0, 0};
            bool ok = true;
            TileWalk<START> walk;
            Seg g;
            begin(walk);
            for (; ok && walk.next(p, a, pl, g); ++ns) {
                const int gk = g.s % p.H_kv, n = g.j1 - g.j0;
                const int32_t* table = a.page_table + (size_t)g.s * p.max_pages;
                if (!is_v) {
                    const int slot = ns % Gm::NQ;
                    if (!warp_wait(&sm.q_empty[slot], ((ns / Gm::NQ) & 1) ^ 1, abort_flag)) {
                        ok = false;
                        break;
                    }
                    if (lane == 0) {
                        const int tiles = PAIR && g.tok0 + pl.tpt < g.sp.n ? 2 : 1;
                        tc::mbar_arrive_expect_tx(&sm.q_full[slot], tiles * q_bytes);
                        for (int t = 0; t < tiles; ++t)
                            for (int h = 0; h < D / 64; ++h)
                                asm volatile(
                                    "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
                                    " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                                        smem_u32(&sm.q[slot * Gm::QT + t][h * TM * 128])),
                                    "l"(reinterpret_cast<uint64_t>(&mq)), "r"(64 * h), "r"(gk * p.G),
                                    "r"(g.sp.tok0 + g.tok0 + t * pl.tpt), "r"(smem_u32(&sm.q_full[slot]))
                                    : "memory");
                    }
                    ++nq[slot];
                }
                // The set's page numbers, a window of 32 to a register (a lane each): the
                // tile's, and the next, whose load has a window's time to arrive.
                const int last_page = (g.sp.len - 1) >> p.page_shift;
                auto window = [&](int i) {
                    const int at = 32 * i + lane;
                    return at <= last_page ? table[at] : 0;
                };
                int wk = (g.j0 * TN >> p.page_shift) >> 5;
                int pages = window(wk), pages_next = window(wk + 1);
                for (int x = 0; x < n; ++x) {
                    const int slot0 = (g.j0 + x) * TN;               // the tile's first slot
                    if ((slot0 >> p.page_shift) >> 5 > wk) {
                        pages = pages_next;
                        pages_next = window(++wk + 1);
                    }
                    const int at = (slot0 + b * box) >> p.page_shift;
                    // (a tile's pages lie in one window: 32 is a multiple of their number)
                    int page = __shfl_sync(~0u, pages, at & 31);
                    const int nb = (min(g.sp.len - slot0, TN) + box - 1) / box;
                    if (b >= nb) page = 0;
                    if (page < 0 || page >= p.n_pages) {
                        raise_status(status, TGVKV_STATUS_INDEX);
                        page = 0;
                    }
                    const int row = page * p.page + ((slot0 + b * box) & (p.page - 1));
                    const int it = base_it + (is_v ? v_place<PAIR>(x, n) : k_place<PAIR>(x));
                    const int st = it % N, ph = (it / N) & 1;
                    if (!warp_wait(QUANT ? &sm.raw_empty[st] : &sm.empty[st], ph ^ 1, abort_flag)) {
                        ok = false;
                        break;
                    }
                    if (QUANT) {
                        if (lane == 0) {
                            sm.filled[st] = it;
                            sm.live[st] = min(g.sp.len - slot0, TN);
                            tc::mbar_arrive_expect_tx(&sm.raw_full[st],
                                                      (uint32_t)(nb * box) * (Gm::ROWB + D / kGroup));
                        }
                        __syncwarp();
                        if (lane < nb)
                            tc::bulk_load(smem_u32(&sm.raw[st][b * box * Gm::ROWB]),
                                          codes + (size_t)row * Gm::ROWB, box * Gm::ROWB,
                                          &sm.raw_full[st]);
                        else if (lane >= 16 && b < nb)
                            tc::bulk_load(smem_u32(&sm.sc[st][b * box * (D / kGroup)]),
                                          scales + (size_t)row * (D / kGroup), box * (D / kGroup),
                                          &sm.raw_full[st]);
                    } else {
                        if (lane == 0) {
                            sm.filled[st] = it;
                            tc::mbar_arrive_expect_tx(&sm.full[st], (uint32_t)(nb * box) * 2 * D);
                        }
                        __syncwarp();
                        const int h = lane >> 4;
                        if (b < nb && h < D / 64)
                            tc::tma_load_2d(&sm.kv[st][h * Gm::HALF + b * box * 128], map, 128 * h, row,
                                            &sm.full[st]);
                    }
                }
                base_it += 2 * n;
            }
            if (!ok && lane == 0) {
                sm.abort_flag = 1;
                raise_status(status, TGVKV_STATUS_TIMEOUT);
            }
            __syncwarp();
            // every Q copy has landed before the CTA may exit (K and V: at the teardown)
            for (int slot = 0; slot < Gm::NQ; ++slot)
                if (nq[slot] > 0) warp_wait(&sm.q_full[slot], (nq[slot] - 1) & 1, &sm.never);
        }

        // ------------------------------------------------------------ rows that see nothing
        // (the items without a key tile, which no CTA's share contains)
        if (warp == 3) {
            for (int s = blockIdx.x; s < p.S; s += gridDim.x) {
                const SetSpan sp = set_span(p, a, s);
                int none = 0;              // tokens of such items
                if (sp.len < sp.n)
                    while (none < sp.n && tiles_seen(sp, none + pl.tpi) == 0) none += pl.tpi;
                none = min(none, sp.n);
                constexpr int U = D / 8;
                for (long long e = lane; e < (long long)none * p.G * U; e += 32) {
                    const int row = (int)(e / U), t = row / p.G;
                    uint16_t* op = a.out + ((size_t)(sp.tok0 + t) * p.H_q + (s % p.H_kv) * p.G +
                                            (row - t * p.G)) * D;
                    reinterpret_cast<uint4*>(op)[e % U] = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        }

        // ------------------------------------------------------------ MMA issuer
        if (warp == 1) {
            const uint32_t leader = elect_one();
            const uint32_t tm = __shfl_sync(~0u, tmem, 0);
            const uint64_t qd0 = tc::sdesc_k_sw128(smem_u32(&sm.q[0][0]));
            const uint64_t kd0 = tc::sdesc_k_sw128(smem_u32(&sm.kv[0][0]));
            const uint64_t vd0 = tc::sdesc_mn_sw128(smem_u32(&sm.kv[0][0]), Gm::HALF);
            const uint32_t q_lo = (uint32_t)qd0, k_lo = (uint32_t)kd0, v_lo = (uint32_t)vd0;
            const uint32_t q_hi = (uint32_t)(qd0 >> 32), k_hi = (uint32_t)(kd0 >> 32),
                           v_hi = (uint32_t)(vd0 >> 32);
            constexpr uint32_t QTILE = D * 2 * TM / 16, SLOT = Gm::TILE / 16, HALF16 = Gm::HALF / 16;
            constexpr uint32_t IDESC_QK = tc::idesc_bf16(TM, TN), IDESC_PV = tc::idesc_bf16_bmn(TM, D);
            int st = 0, ph = 0;                      // next slot of the ring, and its phase
            int ns = 0, nqk = 0, np[2] = {0, 0};
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                if (ok && !warp_wait(bar, parity, abort_flag)) ok = false;
                if (ok) tc::fence_after_sync();
                return ok;
            };
            auto slot_after = [&](int x) { return x + 1 == NST ? 0 : x + 1; };
            // S = Q_w K^T with the K tile in slot k, once S has been read
            auto qk = [&](int w, int qslot, int k) {
                if (nqk > 0 && !wait(&sm.s_free, (nqk - 1) & 1)) return;
                ++nqk;
                const uint32_t qa = q_lo + (uint32_t)(qslot * Gm::QT + (PAIR ? w : 0)) * QTILE;
                const uint32_t ka = k_lo + (uint32_t)k * SLOT;
                mma_ss<0>(leader, tm, qa, ka, q_hi, k_hi, IDESC_QK);
#pragma unroll
                for (int kk = 1; kk < D / 16; ++kk) {
                    const uint32_t off = (kk >> 2) * HALF16 + (kk & 3) * 2;
                    mma_ss<1>(leader, tm, qa + off, ka + off, q_hi, k_hi, IDESC_QK);
                }
                commit(leader, &sm.s_full[w]);
            };
            // O_w (+)= P_w V with the V tile in slot v, once P_w is there
            auto pv = [&](int w, int v, bool accumulate, bool last) {
                if (!wait(&sm.p_full[w], np[w]++ & 1)) return;
                const uint32_t va = v_lo + (uint32_t)v * SLOT;
                const uint32_t to = tm + kOCol + (uint32_t)(w * D), tp = tm + kPCol + (uint32_t)(w * 64);
                mma_ts(leader, to, tp, va, v_hi, IDESC_PV, accumulate ? 1u : 0u);
#pragma unroll
                for (int kk = 1; kk < TN / 16; ++kk)
                    mma_ts(leader, to, tp + (uint32_t)(kk * 8), va + (uint32_t)(kk * (16 * 128 / 16)), v_hi,
                           IDESC_PV, 1u);
                if (last) commit(leader, &sm.o_done[w]);
            };
            auto release = [&](uint64_t* bar) { commit(leader, bar); };
            TileWalk<START> walk;
            Seg g;
            begin(walk);
            for (; ok; ++ns) {
                const int more = walk.next(p, a, pl, g);
                if (!__shfl_sync(~0u, more, 0)) break;
                const int qs = ns % Gm::NQ, n = __shfl_sync(~0u, g.j1 - g.j0, 0);
                if (!wait(&sm.q_full[qs], (ns / Gm::NQ) & 1)) break;
                if (PAIR) {
                    // group w's tiles are x < hi[w]
                    const int hi0 = __shfl_sync(~0u, min(group_tiles<PAIR>(g, pl, 0), g.j1) - g.j0, 0);
                    const int hi1 = __shfl_sync(~0u, min(group_tiles<PAIR>(g, pl, 1), g.j1) - g.j0, 0);
                    if (!wait(&sm.full[st], ph)) break;
                    if (0 < hi0) qk(0, qs, st);
                    if (ok && 0 < hi1) qk(1, qs, st);
                    if (!ok) break;
                    release(&sm.empty[st]);
                    if (n == 1) release(&sm.q_empty[qs]);
                    st = slot_after(st), ph ^= st == 0;
                    for (int x = 0; ok && x < n; ++x) {
                        const int v = st, k = slot_after(st);
                        const int kph = ph ^ (k == 0);
                        if (!wait(&sm.full[v], ph)) break;
                        if (x < hi0) pv(0, v, x > 0, x + 1 == hi0);
                        if (ok && x + 1 < n) wait(&sm.full[k], kph);
                        if (ok && x + 1 < hi0) qk(0, qs, k);
                        if (ok && x < hi1) pv(1, v, x > 0, x + 1 == hi1);
                        if (!ok) break;
                        release(&sm.empty[v]);
                        st = k, ph = kph;
                        if (x + 1 < n) {
                            if (x + 1 < hi1) qk(1, qs, k);
                            if (!ok) break;
                            release(&sm.empty[k]);
                            if (x + 2 == n) release(&sm.q_empty[qs]);
                            st = slot_after(k), ph = kph ^ (st == 0);
                        }
                    }
                } else {
                    for (int x = 0; x < min(n, 2); ++x) {
                        if (!wait(&sm.full[st], ph)) break;
                        qk(x, qs, st);
                        if (!ok) break;
                        release(&sm.empty[st]);
                        if (x + 1 == n) release(&sm.q_empty[qs]);
                        st = slot_after(st), ph ^= st == 0;
                    }
                    for (int x = 0; ok && x < n; ++x) {
                        if (!wait(&sm.full[st], ph)) break;
                        pv(x & 1, st, x > 1, x + 2 >= n);
                        if (!ok) break;
                        release(&sm.empty[st]);
                        st = slot_after(st), ph ^= st == 0;
                        if (x + 2 < n) {
                            if (!wait(&sm.full[st], ph)) break;
                            qk(x & 1, qs, st);
                            if (!ok) break;
                            release(&sm.empty[st]);
                            if (x + 3 == n) release(&sm.q_empty[qs]);
                            st = slot_after(st), ph ^= st == 0;
                        }
                    }
                }
            }
            if (!ok && lane == 0) {
                sm.abort_flag = 1;
                raise_status(status, TGVKV_STATUS_TIMEOUT);
            }
            __syncwarp();
            // every MMA this CTA issued has finished before TMEM is released
            release(&sm.mma_done);
            warp_wait(&sm.mma_done, 0, &sm.never);
        }

    } else if (warp < kConvWarp) {
        // -------------------------------------------------------- softmax
        regs_up<Gm::SOFT_REGS>();
        const int w = (warp - kSoftWarp) >> 2;               // group
        const int quarter = warp & 3;                        // TMEM lanes of this warp
        const int r = quarter * 32 + lane;                   // row of the tile
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t tp = lanes + kPCol + (uint32_t)(w * 64), to = lanes + kOCol + (uint32_t)(w * D);
        const float sl2 = p.scale_log2;
        const int ri = r / p.G, rh = r - ri * p.G;           // token within the tile, head
        int ns = 0, nso = 0, npart = 0, base_it = 0;
        bool ok = true;
        if (warp == kSoftWarp && lane == 0 && share < (int)gridDim.x)
            split[share] = SplitItem{-1, 0, 0, 0};
        auto& at = sm.at[warp - kSoftWarp];
        const volatile Seg& g = at.g;
        if (lane == 0) begin(at.walk);
        for (; ok; ++npart) {
            __syncwarp();
            int more = 0;
            if (lane == 0) more = at.walk.next(p, a, pl, at.g);
            if (!__shfl_sync(~0u, more, 0)) break;
            const int n = g.j1 - g.j0, j0 = g.j0, len = g.sp.len;
            const int nt = g.sp.n, tok = g.tok0 + (PAIR ? w * pl.tpt : 0);   // the tile's first token
            const SetSpan span{len, nt, 0};
            const int seen_tiles = !PAIR ? 0 : tok < nt ? tiles_seen(span, tok + pl.tpt) : 0;
            const int hi = PAIR ? min(seen_tiles, j0 + n) - j0 : n;
            const int toks = min(nt - tok, pl.tpt);                  // its tokens (<= 0: none)
            const bool valid = ri < toks;
            const bool warp_on = quarter * 32 < toks * p.G;          // some row of the warp is real
            // slots that this row sees: its own and those before
            const int lim = min(len - nt + min(tok + ri, nt - 1) + 1, len);
            float m = -INFINITY, l = 0.f;
            for (int x = PAIR ? 0 : w; x < hi; x += PAIR ? 1 : 2) {
                if (!warp_wait(&sm.s_full[w], ns & 1, abort_flag)) {
                    ok = false;
                    break;
                }
                ++ns;
                tc::fence_after_sync();
                const int j = j0 + x;
                const int seen = lim - j * TN;               // columns seen of this tile
                const bool masked = __any_sync(~0u, seen < TN);
                float y[TN];
#pragma unroll
                for (int c = 0; c < TN / 32; ++c) {
                    float t[32];
                    tc::tmem_ld32(lanes + (uint32_t)(32 * c), t);
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[32 * c + e] = t[e];
                }
                tc::tmem_wait_ld();
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.s_free);
                if (warp_on) {
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < TN; ++e)
                            if (e >= seen) y[e] = -INFINITY;
                    }
                    float ma = -INFINITY, mb = -INFINITY;
#pragma unroll
                    for (int e = 0; e < TN; e += 4) {
                        ma = max3(ma, y[e], y[e + 1]);
                        mb = max3(mb, y[e + 2], y[e + 3]);
                    }
                    const float mx = fmaxf(ma, mb);
                    const float mt = mx * sl2;
                    float alpha = 1.f;
                    if (mt > m + kRescale) {                 // also the first tile with something seen
                        alpha = fast_exp2(m - mt);
                        m = mt;
                        l *= alpha;
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    // O holds the tiles before this one (the commit of S covers P V before it)
                    if (x > (PAIR ? 0 : 1) && __any_sync(~0u, alpha != 1.f)) {
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {   // in pieces: S is in registers
                            uint32_t t[16];
                            tmem_ld16(to + (uint32_t)(16 * c), t);
                            tc::tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                t[e] = __float_as_uint(__uint_as_float(t[e]) * alpha);
                            tmem_st16(to + (uint32_t)(16 * c), t);
                        }
                    }
                    const float2 s2 = make_float2(sl2, sl2), n2 = make_float2(-ref, -ref);
                    float2 za = make_float2(0.f, 0.f), zb = za;
#pragma unroll
                    for (int c = 0; c < TN; c += 32) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float2 t0 = fma2(make_float2(y[c + e], y[c + e + 1]), s2, n2);
                            const float2 t1 = fma2(make_float2(y[c + e + 2], y[c + e + 3]), s2, n2);
                            const float2 e0 = make_float2(fast_exp2(t0.x), fast_exp2(t0.y));
                            const float2 e1 = make_float2(fast_exp2(t1.x), fast_exp2(t1.y));
                            za = add2(za, e0);
                            zb = add2(zb, e1);
                            pk[e / 2] = pack_bf16x2(e0.x, e0.y);
                            pk[e / 2 + 1] = pack_bf16x2(e1.x, e1.y);
                        }
                        tmem_st16(tp + (uint32_t)(c / 2), pk);
                    }
                    l += (za.x + za.y) + (zb.x + zb.y);
                    tc::tmem_wait_st();
                }
                // bf16 caches: the pool's rows past the set's end may hold anything, and
                // 0 x NaN is not 0, so V's rows there are cleared (the converters do it
                // for integer caches)
                const int live = len - j * TN;
                if (!QUANT && live < TN) {
                    const int vi = base_it + v_place<PAIR>(x, n);
                    if (!warp_wait(&sm.full[vi % NST], (vi / NST) & 1, abort_flag)) {
                        ok = false;
                        break;
                    }
                    for (int e = quarter * 32 + lane; e < (TN - live) * (D / 8); e += TM) {
                        const int row = live + e / (D / 8), u = e % (D / 8);
                        *reinterpret_cast<uint4*>(&sm.kv[vi % NST][(u >> 3) * Gm::HALF + row * 128 +
                                                                  (u & 7) * 16]) =
                            make_uint4(0u, 0u, 0u, 0u);
                    }
                    tc::fence_proxy_async_smem();
                }
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.p_full[w]);
            }
            if (!ok) break;
            base_it += 2 * n;

            // ---- the segment's end
            const int wi = warp - kSoftWarp;
            const bool begins = g.j0 == 0, ends = g.j1 == g.nk;
            // CTAs that hold earlier and later parts of the item
            const int before = begins ? 0 : (int)((g.j0 + per - 1) / per);
            const int after = ends ? 0 : (int)((g.nk - g.j1 + per - 1) / per);
            const bool few = before + after <= kJoin;
            const bool writes = begins && few;                   // joins the others' parts, if any
            const size_t rec_floats = chunk_record_floats(pl.rows, D);
            auto record = [&](int cta, int slot) {
                return part + (size_t)((cta * 2 + slot) * (PAIR ? 2 : 1) + (PAIR ? w : 0)) * rec_floats;
            };
            float* pp = record(share, g.starts ? 0 : 1);
            uint16_t* op = a.out + ((size_t)(g.sp.tok0 + (valid ? tok + ri : 0)) * p.H_q +
                                    (g.s % p.H_kv) * p.G + rh) * D;
            if (begins && !few && wi == 0 && lane == 0)
                split[share] = SplitItem{g.s, g.u, 1 + after, g.starts ? 0 : 1};

            // this CTA's result: O = f0 O0 + f1 O1 (SPLIT), its maximum M and mass L
            float M = m, L = l, f0 = 1.f, f1 = 0.f;
            if (PAIR) {
                if (hi > 0) {
                    if (!warp_wait(&sm.o_done[w], nso & 1, abort_flag)) {
                        ok = false;
                        break;
                    }
                    ++nso;
                }
            } else {
                // join the groups' halves: each takes half of the dims of both O
                sm.ml[w][r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.join_in);
                // (group 1 has no tile, and no O, in a segment of one)
                if (!warp_wait(&sm.o_done[0], npart & 1, abort_flag) ||
                    (n > 1 && !warp_wait(&sm.o_done[1], nso & 1, abort_flag)) ||
                    !warp_wait(&sm.join_in, npart & 1, abort_flag)) {
                    ok = false;
                    break;
                }
                if (n > 1) ++nso;
                const float2 a0 = sm.ml[0][r], a1 = sm.ml[PAIR ? 0 : 1][r];
                M = fmaxf(a0.x, a1.x);
                const float ref = M == -INFINITY ? 0.f : M;
                f0 = fast_exp2(a0.x - ref);
                f1 = fast_exp2(a1.x - ref);
                L = a0.y * f0 + a1.y * f1;
            }
            tc::fence_after_sync();
            // the other parts of an item that this CTA writes
            // (a record's dims 4 k .. 4 k + 3 of row r are float4 k * rows + r: a warp's rows
            // lie side by side)
            float ref = 0.f;
            const float* others = record(share + 1, 0);
            const size_t next = (size_t)(PAIR ? 4 : 2) * rec_floats;
            const int row = valid ? r : 0, m_at = pl.rows * D + row, l_at = m_at + pl.rows;
            if (writes && after > 0) {
                for (int x = 1; ok && x <= after; ++x)
                    ok = take_flag(sync + kTileFlags + (share + x) * 8 + wi, lane, abort_flag);
                if (!ok) break;
                float Mn = M;
                for (int x = 0; x < after; ++x) Mn = fmaxf(Mn, __ldcg(others + x * next + m_at));
                ref = Mn == -INFINITY ? 0.f : Mn;
                const float f = fast_exp2(M - ref);
                f0 *= f, f1 *= f, L *= f;
                for (int x = 0; x < after; ++x)
                    L += __ldcg(others + x * next + l_at) *
                         fast_exp2(__ldcg(others + x * next + m_at) - ref);
            }
            const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);
            constexpr int COLS = PAIR ? D : D / 2;               // dims this thread writes
            const int col0 = PAIR ? 0 : w * COLS;
            // (a group without a tile left its O as it was)
            const bool has0 = PAIR ? hi > 0 : true, has1 = n > 1;
            constexpr int CC = COLS < 64 ? COLS : 64;            // columns at a time
#pragma unroll 1
            for (int c = 0; c < COLS; c += CC) {
                float t[CC];
#pragma unroll
                for (int cc = 0; cc < CC; cc += 32) {
                    float o0[32], o1[32];
                    tc::tmem_ld32(lanes + kOCol + (uint32_t)((PAIR ? w * D : 0) + col0 + c + cc), o0);
                    if (!PAIR) tc::tmem_ld32(lanes + kOCol + (uint32_t)(D + col0 + c + cc), o1);
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        t[cc + e] = has0 ? o0[e] * f0 : 0.f;
                        if (!PAIR) t[cc + e] += has1 ? o1[e] * f1 : 0.f;
                    }
                }
                const int k0 = (col0 + c) / 4;
                if (valid && writes) {
#pragma unroll 1
                    for (int x = 0; x < after; ++x) {
                        const float f = fast_exp2(__ldcg(others + x * next + m_at) - ref);
                        const float4* pj =
                            reinterpret_cast<const float4*>(others + x * next) + (size_t)k0 * pl.rows + r;
                        float4 o4[CC / 4];
#pragma unroll
                        for (int e = 0; e < CC / 4; ++e) o4[e] = __ldcg(pj + e * pl.rows);
#pragma unroll
                        for (int e = 0; e < CC / 4; ++e) {
                            t[4 * e] += o4[e].x * f, t[4 * e + 1] += o4[e].y * f;
                            t[4 * e + 2] += o4[e].z * f, t[4 * e + 3] += o4[e].w * f;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < CC; e += 8)
                        *reinterpret_cast<uint4*>(op + col0 + c + e) = make_uint4(
                            pack_bf16x2(t[e] * inv, t[e + 1] * inv),
                            pack_bf16x2(t[e + 2] * inv, t[e + 3] * inv),
                            pack_bf16x2(t[e + 4] * inv, t[e + 5] * inv),
                            pack_bf16x2(t[e + 6] * inv, t[e + 7] * inv));
                } else if (valid) {
                    float4* pj = reinterpret_cast<float4*>(pp) + (size_t)k0 * pl.rows + r;
#pragma unroll
                    for (int e = 0; e < CC / 4; ++e)
                        pj[e * pl.rows] = make_float4(t[4 * e], t[4 * e + 1], t[4 * e + 2], t[4 * e + 3]);
                }
                __syncwarp();
            }
            tc::fence_before_sync();
            if (!writes) {
                if (valid) {           // (SPLIT: both groups write the same)
                    pp[pl.rows * D + r] = M;
                    pp[pl.rows * D + pl.rows + r] = L;
                }
                if (few) give_flag(sync + kTileFlags + share * 8 + wi, lane);
            }
            if (!PAIR) {
                // both O and (m, l) are free again
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.join_out);
                if (!warp_wait(&sm.join_out, npart & 1, abort_flag)) {
                    ok = false;
                    break;
                }
                tc::fence_after_sync();
            }
        }
        if (!ok) {
            sm.abort_flag = 1;
            if (lane == 0) raise_status(status, TGVKV_STATUS_TIMEOUT);
        }
    } else if constexpr (QUANT) {
        // -------------------------------------------------------- converters
        regs_down<Gm::CONV_REGS>();
        // A thread converts 8 consecutive values of every RSTEP-th row; RSTEP is a
        // multiple of 8, so the swizzle is the same in all of them.
        constexpr int T = Gm::CW * 32, UPR = D / 8, RSTEP = T / UPR, PER = TN / RSTEP, BATCH = PER / 2;
        static_assert(RSTEP % 8 == 0 && TN % RSTEP == 0 && PER % BATCH == 0, "converter threads");
        const int ct = tid - kConvWarp * 32, u = ct % UPR, r0 = ct / UPR;
        const int src = ct * (FMT == TGVKV_CACHE_INT8 ? 8 : 4), sc0 = r0 * (D / kGroup) + (u >> 2);
        const int dst0 = (u >> 3) * Gm::HALF + r0 * 128 + (((u & 7) ^ (r0 & 7)) << 4);
        bool ok = true;
        const int tiles = 2 * sm.tiles;
        for (int it = 0; it < tiles; ++it) {             // K and V tiles in the ring's order
            const int rs = it % NRAW, st = it % NST;
            if (!warp_wait(&sm.raw_full[rs], (it / NRAW) & 1, abort_flag) ||
                !warp_wait(&sm.empty[st], ((it / NST) & 1) ^ 1, abort_flag)) {
                ok = false;
                break;
            }
            const unsigned char* raw = sm.raw[rs] + src;
            const unsigned char* sc = sm.sc[rs] + sc0;
            unsigned char* dst = sm.kv[st] + dst0;
            const int live = sm.live[rs];
#pragma unroll
            for (int b0 = 0; b0 < PER; b0 += BATCH) {
                // a batch's loads before its stores: they cannot pass one another
                uint2 c[BATCH];
                uint32_t byte[BATCH];
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    const int e = b0 + b;
                    c[b] = make_uint2(0u, 0u);
                    if (FMT == TGVKV_CACHE_INT8)
                        c[b] = *reinterpret_cast<const uint2*>(raw + e * T * 8);
                    else
                        c[b].x = *reinterpret_cast<const uint32_t*>(raw + e * T * 4);
                    byte[b] = sc[e * RSTEP * (D / kGroup)];
                }
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    uint4 v = codes_to_bf16<FMT>(c[b], byte[b], p.magic);
                    // past the set's end
                    if (live < TN && r0 + (b0 + b) * RSTEP >= live) v = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(dst + (b0 + b) * RSTEP * 128) = v;
                }
            }
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(&sm.full[st]);
                tc::mbar_arrive(&sm.raw_empty[rs]);
            }
        }
        if (!ok) {
            sm.abort_flag = 1;
            if (lane == 0) raise_status(status, TGVKV_STATUS_TIMEOUT);
        }
    }

    // ------------------------------------------------------------ teardown
    __syncwarp();
    tc::fence_before_sync();
    __syncthreads();
    // every K and V copy this CTA issued has landed before it may exit (no producer
    // is at work any more: the slots' last copies are the ones to wait for)
    if (warp == 0) {
        constexpr int N = QUANT ? NRAW : NST;
        for (int st = 0; st < N; ++st)
            if (sm.filled[st] >= 0)
                warp_wait(QUANT ? &sm.raw_full[st] : &sm.full[st], (sm.filled[st] / N) & 1, &sm.never);
    }
    if (warp == 1) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
    // the last CTA leaves the tickets at zero for the next call
    if (tid == 0 && atomicAdd(sync + 1, 1u) == gridDim.x - 1) {
        atomicExch(sync, 0u);
        atomicExch(sync + 1, 0u);
    }
}

template <int D, int FMT, bool PAIR>
cudaError_t launch_tile(const CacheProblem& p, const CachePools& pool, const ChunkArgs& a,
                        float* part, SplitItem* split, uint32_t* sync, uint32_t* status,
                        cudaStream_t stream) {
    using Sm = TileSmem<D, FMT, PAIR>;
    static_assert(sizeof(Sm) + 1024 <= 227 * 1024, "shared memory of one CTA");
    TilePlan pl;
    pl.tpt = TM / p.G;
    pl.tpi = PAIR ? 2 * pl.tpt : pl.tpt;
    pl.rows = pl.tpt * p.G;
    alignas(64) CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, p, a, p.G, pl.tpt)) return cudaErrorInvalidValue;
    mk = mv = mq;                      // not used by integer caches
    const uint64_t rows = (uint64_t)p.n_pages * p.page;
    if (FMT == TGVKV_CACHE_BF16 &&
        (!make_pool_map(&mk, pool.k, rows, 2 * D, 128, p.page < TN ? p.page : TN) ||
         !make_pool_map(&mv, pool.v, rows, 2 * D, 128, p.page < TN ? p.page : TN)))
        return cudaErrorInvalidValue;
    const size_t smem = sizeof(Sm) + 1024;
    cudaError_t e = cudaFuncSetAttribute(chunk_tile_kernel<D, FMT, PAIR>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    // the register split needs what the launch bounds ask the compiler for
    cudaFuncAttributes at;
    if ((e = cudaFuncGetAttributes(&at, chunk_tile_kernel<D, FMT, PAIR>)) != cudaSuccess) return e;
    if (at.numRegs < TileGeom<D, FMT, PAIR>::LAUNCH_REGS) return cudaErrorInvalidConfiguration;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int ctas = sms < kTileMaxCtas ? sms : kTileMaxCtas;
    e = launch_dependent(chunk_tile_kernel<D, FMT, PAIR>, dim3((unsigned)ctas),
                         dim3(TileGeom<D, FMT, PAIR>::THREADS), smem, stream, mq, mk, mv, p, pool, a, pl,
                         part, split, sync, status);
    if (e != cudaSuccess) return e;
    return launch_tile_merge(p, a, pl, ctas, part, split, stream);
}

}  // namespace tgvkv
