// Writing rows into the paged cache, quantising on the way, and reading them
// back as bf16 (cache.cuh has the layout and the formats).
//
//   write:  slot lens[s] + i of set s  <-  quantised row i of the set's new rows
//           lens_out[s] = lens[s] + rows of s
//   read:   out row offsets[s] + i     <-  slot first[s] + i of set s, exactly
//
// Both move each row once and are bound by HBM: 2 d bytes of bf16 plus the
// stored row per row of K and of V.  A CTA takes RowGeom::ROWS consecutive rows;
// one thread per row finds its set (a search over the offsets, by a warp first for
// the CTA's span) and its pool row, for writes while the row data's loads, whose
// addresses do not depend on it, are already in flight.  A row is spread over d / 8
// lanes of 8 values (16 bytes of bf16), so a scale's 32 values sit in 4 neighbouring
// lanes.  Five CTAs an SM: the searches and barriers of one run under the loads of
// the others.
//
// Measured (of 6790 GB/s): the evicted rows of 32 x 32 sets into int8 pages and back
// 43 us (88%), 28 layers' prompts of 8704 tokens into int4 pages and back 204 us (91%),
// 32 x 32 sets of 1505 .. 3009 slots read back from int4 pages 226 us (98%); one token of 28
// layers 4 us on the GPU, which is the launch and three dependent reads.
//
// Loads are never of the read-only kind: a kernel may start while the one that writes
// its inputs is still at work (griddep_wait).
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowUnroll = 4;          // rows of K and of V a thread has in flight

template <int D>
struct RowGeom {
    static constexpr int LPR = D / 8;                          // lanes a row
    static constexpr int RPI = kRowThreads / LPR;              // rows at a time
    static constexpr int ROWS = RPI * kRowUnroll;              // rows a CTA
};

// The largest i in [lo, hi] with off[i] <= x, given off[lo] <= x.
template <typename T>
__device__ __forceinline__ int find_last(const T* off, int lo, int hi, long long x) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((long long)off[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The same by a whole warp, 32 probes at a time: two loads in a row for 1024
// entries where a binary search has ten.
template <typename T>
__device__ __forceinline__ int find_last_warp(const T* off, int hi, long long x, int lane) {
    int lo = 0;
    while (lo < hi) {
        const int step = (hi - lo + 32) / 32;    // candidates lo, lo + step, ..: the span is hi - lo + 1
        const int at = lo + lane * step;
        const bool le = at <= hi && (long long)off[at] <= x;
        const uint32_t m = __ballot_sync(~0u, le);
        lo += max(__popc(m) - 1, 0) * step;      // offsets ascend: the lanes that hold come first
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// The first and last set (or sequence) of a CTA's rows, by two of its warps.
template <typename T>
__device__ __forceinline__ void find_span(const T* off, int last, long long x0, long long x1,
                                          int (&span)[2]) {
    const int warp = threadIdx.x >> 5;
    if (warp < 2) {
        const int i = find_last_warp(off, last, warp ? x1 : x0, threadIdx.x & 31);
        if ((threadIdx.x & 31) == 0) span[warp] = i;
    }
}

// Pool row of (set, slot), or -1 (with the status bit) when there is none.
__device__ __forceinline__ int pool_row(const CacheProblem& p, const int32_t* page_table,
                                              int s, long long slot, uint32_t* status) {
    if (slot < 0 || slot >= p.cap) {
        raise_status(status, TGVKV_STATUS_INDEX);
        return -1;
    }
    const int page = page_table[(size_t)s * p.max_pages + (int)(slot >> p.page_shift)];
    if (page < 0 || page >= p.n_pages) {
        raise_status(status, TGVKV_STATUS_INDEX);
        return -1;
    }
    return page * p.page + ((int)slot & (p.page - 1));
}

// ---- 8 values to their stored form -------------------------------------------
// The scale byte of a group from the largest magnitude among its values, as
// bf16 bits (15 bits).  With bits = 2^X' (1 + f / 128): Q = 127 needs
// e = X' - 6, one more when f > 126 (the value is above 127 * 2^(X' - 6));
// Q = 7 needs e = X' - 2, one more when f > 96.
template <int FMT>
__device__ __forceinline__ int group_byte(uint32_t bits) {
    const int x = (int)(bits >> 7), f = (int)(bits & 127u);
    if (x == 255) return 255;
    if (FMT == TGVKV_CACHE_INT8) return max(x - 6 + (f > 126 ? 1 : 0), 1);
    return min(max(x - 2 + (f > 96 ? 1 : 0), 1), 247);
}

// Quantise this lane's 8 values (the group's other 24 are in the 3
// neighbouring lanes; the whole warp takes part) and, where `on`, store them
// with the group's scale byte.
template <int FMT>
__device__ __forceinline__ void store_row(uint4 w, uint8_t* row, uint8_t* scales, int unit,
                                          bool on) {
    // magnitudes as bf16 bits order like the values; NaN sorts above infinity
    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, words[i] & 0x7FFF7FFFu);
    top = max(top & 0xFFFFu, top >> 16);
    top = max(top, __shfl_xor_sync(~0u, top, 1));
    top = max(top, __shfl_xor_sync(~0u, top, 2));
    const int byte = group_byte<FMT>(top);
    if (!on) return;
    if (FMT == TGVKV_CACHE_INT8) {
        // x 2^-e + 1.5 * 2^23 rounds x 2^-e to an integer (ties to even) and leaves it, in two's
        // complement, in the low bits; |x 2^-e| <= 127 by the choice of e
        const float inv = __uint_as_float((uint32_t)(254 - min(byte, 253)) << 23);
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[2 * i] = __float_as_uint(fmaf(__uint_as_float(words[i] << 16), inv, 12582912.f));
            q[2 * i + 1] = __float_as_uint(fmaf(__uint_as_float(words[i] & 0xFFFF0000u), inv, 12582912.f));
        }
        uint32_t c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            c[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040),
                               __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
            if (byte == 255) c[i] = 0u;
        }
        reinterpret_cast<uint2*>(row)[unit] = make_uint2(c[0], c[1]);
    } else {
        // in bf16, whose step is 1 from 128 to 256: x 2^-e + 136 rounds to 128 + (q + 8)
        const uint32_t inv = both((uint32_t)(254 - min(byte, 253)) << 7);
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (byte == 247) {         // e at its cap: the values may be beyond 7 * 2^e
                const uint32_t v = bf16x2_min(bf16x2_max(bf16x2_mul(words[i], inv), 0xC0E0C0E0u), 0x40E040E0u);
                q[i] = bf16x2_fma(v, 0x3F803F80u, 0x43084308u);
            } else {
                q[i] = bf16x2_fma(words[i], inv, 0x43084308u);
            }
        }
        // the nibbles: elements 0, 2, 1, 3 (and 4, 6, 5, 7) a byte apart, then the odd ones
        // beside the even ones
        const uint32_t a = (q[0] & 0x000F000Fu) | ((q[1] & 0x000F000Fu) << 8);
        const uint32_t b = (q[2] & 0x000F000Fu) | ((q[3] & 0x000F000Fu) << 8);
        const uint32_t c = __byte_perm(a, b, 0x5410) | (__byte_perm(a, b, 0x7632) << 4);
        reinterpret_cast<uint32_t*>(row)[unit] = byte == 255 ? 0x88888888u : c;
    }
    if ((unit & 3) == 0) scales[unit >> 2] = (uint8_t)byte;
}

// ---- write -------------------------------------------------------------------
// The rows to write: of the CSR form, row u of [0, offsets[S]) belongs to the
// set its offsets say; of the token form, row u = token * H_kv + head.
struct WriteSource {
    const uint16_t* k;
    const uint16_t* v;
    long long k_tok, k_head, v_tok, v_head;   // element strides (token form)
    const int64_t* row_offsets;               // CSR form: [S + 1]
    const int32_t* tok_offsets;               // token form: [B + 1]
    long long rows;                           // rows the tensors hold (< 2^31)
};

template <int D, int FMT, bool TOKENS>
__global__ void __launch_bounds__(kRowThreads, 5)
cache_write_kernel(const CacheProblem p, const WriteSource src, const CachePools pool,
                   const int32_t* page_table, const int32_t* lens,
                   int32_t* __restrict__ lens_out, uint32_t* __restrict__ status) {
    using Gm = RowGeom<D>;
    __shared__ int dst[Gm::ROWS];
    __shared__ int span[2];
    const int tid = threadIdx.x;
    const unsigned u0 = blockIdx.x * (unsigned)Gm::ROWS;
    const int unit = tid % Gm::LPR, sub = tid / Gm::LPR;

    griddep_launch_dependents();       // the next call's set-up may overlap this one's end
    griddep_wait();
    // the lengths after the write, and the check of the offsets
    for (int s = blockIdx.x * kRowThreads + tid; s < p.S; s += gridDim.x * kRowThreads) {
        long long lo, hi, most;
        if (TOKENS) {
            const int b = s / p.H_kv;
            lo = src.tok_offsets[b];
            hi = src.tok_offsets[b + 1];
            most = src.rows / p.H_kv;
            if (b == 0 && lo != 0) raise_status(status, TGVKV_STATUS_INDEX);
        } else {
            lo = src.row_offsets[s];
            hi = src.row_offsets[s + 1];
            most = src.rows;
            if (s == 0 && lo != 0) raise_status(status, TGVKV_STATUS_INDEX);
        }
        const int len = lens[s];
        if (lo < 0 || hi < lo || hi > most || len < 0 || len > p.cap || hi - lo > p.cap - len) {
            raise_status(status, TGVKV_STATUS_INDEX);
            const long long n = max(min(hi, most) - max(lo, 0ll), 0ll);
            lens_out[s] = (int)min((long long)clamp_len(len, p.cap) + n, (long long)p.cap);
        } else {
            lens_out[s] = len + (int)(hi - lo);
        }
    }

    // the rows' data, in flight while their places are looked up
    const unsigned n_rows = (unsigned)src.rows;
    uint4 kw[kRowUnroll], vw[kRowUnroll];
#pragma unroll
    for (int i = 0; i < kRowUnroll; ++i) {
        const unsigned u = u0 + i * Gm::RPI + sub;
        kw[i] = vw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (u >= n_rows) continue;
        size_t ko, vo;
        if (TOKENS) {
            const unsigned t = u / (unsigned)p.H_kv, g = u - t * p.H_kv;
            ko = t * src.k_tok + g * src.k_head;
            vo = t * src.v_tok + g * src.v_head;
        } else {
            ko = vo = (size_t)u * D;
        }
        kw[i] = __ldcs(reinterpret_cast<const uint4*>(src.k + ko) + unit);
        vw[i] = __ldcs(reinterpret_cast<const uint4*>(src.v + vo) + unit);
    }
    const unsigned u_last = max(min(u0 + Gm::ROWS, n_rows), 1u) - 1u;
    if (TOKENS)
        find_span(src.tok_offsets, p.B - 1, u0 / (unsigned)p.H_kv, u_last / (unsigned)p.H_kv, span);
    else
        find_span(src.row_offsets, p.S - 1, u0, u_last, span);
    __syncthreads();
    if (tid < Gm::ROWS) {
        const unsigned u = u0 + tid;
        int row = -1;
        if (u < n_rows) {
            int s = -1;
            long long at = 0;
            if (TOKENS) {
                const int t = (int)(u / (unsigned)p.H_kv);
                if (t >= src.tok_offsets[0] && t < src.tok_offsets[p.B]) {
                    const int b = find_last(src.tok_offsets, span[0], span[1], t);
                    s = b * p.H_kv + (int)(u - (unsigned)t * p.H_kv);
                    at = t - src.tok_offsets[b];
                }
            } else if (u >= src.row_offsets[0] && u < src.row_offsets[p.S]) {
                s = find_last(src.row_offsets, span[0], span[1], u);
                at = u - src.row_offsets[s];
            }
            if (s >= 0 && at >= 0)
                row = pool_row(p, page_table, s, clamp_len(lens[s], p.cap) + at, status);
        }
        dst[tid] = row;
    }
    __syncthreads();
    constexpr int RB = FMT == TGVKV_CACHE_BF16 ? 2 * D : FMT == TGVKV_CACHE_INT8 ? D : D / 2;
#pragma unroll
    for (int i = 0; i < kRowUnroll; ++i) {
        const int row = dst[i * Gm::RPI + sub];
        const bool on = row >= 0;
        const size_t at = on ? row : 0;
        if (FMT == TGVKV_CACHE_BF16) {
            if (!on) continue;
            reinterpret_cast<uint4*>(pool.k + at * RB)[unit] = kw[i];
            reinterpret_cast<uint4*>(pool.v + at * RB)[unit] = vw[i];
        } else {
            // lanes without a row take part in the group's maximum and store nothing
            store_row<FMT>(kw[i], pool.k + at * RB, pool.ks + at * (D / kGroup), unit, on);
            store_row<FMT>(vw[i], pool.v + at * RB, pool.vs + at * (D / kGroup), unit, on);
        }
    }
}

// ---- read --------------------------------------------------------------------
template <int D, int FMT>
__global__ void __launch_bounds__(kRowThreads, 5)
cache_read_kernel(const CacheProblem p, const CachePools pool,
                  const int32_t* page_table, const int32_t* first,
                  const int64_t* offsets, uint16_t* __restrict__ k_out,
                  uint16_t* __restrict__ v_out, long long rows, uint32_t* __restrict__ status) {
    using Gm = RowGeom<D>;
    __shared__ int from[Gm::ROWS];
    __shared__ int span[2];
    const int tid = threadIdx.x;
    const unsigned u0 = blockIdx.x * (unsigned)Gm::ROWS;
    const int unit = tid % Gm::LPR, sub = tid / Gm::LPR;
    griddep_launch_dependents();
    griddep_wait();
    for (int s = blockIdx.x * kRowThreads + tid; s < p.S; s += gridDim.x * kRowThreads) {
        const long long lo = offsets[s], hi = offsets[s + 1];
        if (lo < 0 || hi < lo || hi > rows || (s == 0 && lo != 0))
            raise_status(status, TGVKV_STATUS_INDEX);
    }
    const unsigned n_rows = (unsigned)rows;
    find_span(offsets, p.S - 1, u0, (long long)min(u0 + Gm::ROWS, n_rows) - 1, span);
    __syncthreads();
    if (tid < Gm::ROWS) {
        const unsigned u = u0 + tid;
        int row = -1;
        if (u < n_rows && u >= offsets[0] && u < offsets[p.S]) {
            const int s = find_last(offsets, span[0], span[1], u);
            const long long at = u - offsets[s];
            if (at >= 0)
                row = pool_row(p, page_table, s, at + (first ? (long long)first[s] : 0ll), status);
        }
        from[tid] = row;
    }
    __syncthreads();
    uint4 kw[kRowUnroll], vw[kRowUnroll];
    uint32_t kb[kRowUnroll], vb[kRowUnroll];
#pragma unroll
    for (int i = 0; i < kRowUnroll; ++i) {
        const int row = from[sub + i * Gm::RPI];
        kw[i] = vw[i] = make_uint4(0u, 0u, 0u, 0u);
        kb[i] = vb[i] = 0u;
        if (row < 0) continue;
        const size_t at = row;
        if (FMT == TGVKV_CACHE_BF16) {
            kw[i] = __ldcs(reinterpret_cast<const uint4*>(pool.k + at * (2 * D)) + unit);
            vw[i] = __ldcs(reinterpret_cast<const uint4*>(pool.v + at * (2 * D)) + unit);
        } else {
            if (FMT == TGVKV_CACHE_INT8) {
                const uint2 a = __ldcs(reinterpret_cast<const uint2*>(pool.k + at * D) + unit);
                const uint2 b = __ldcs(reinterpret_cast<const uint2*>(pool.v + at * D) + unit);
                kw[i].x = a.x, kw[i].y = a.y, vw[i].x = b.x, vw[i].y = b.y;
            } else {
                kw[i].x = __ldcs(reinterpret_cast<const uint32_t*>(pool.k + at * (D / 2)) + unit);
                vw[i].x = __ldcs(reinterpret_cast<const uint32_t*>(pool.v + at * (D / 2)) + unit);
            }
            kb[i] = pool.ks[at * (D / kGroup) + (unit >> 2)];
            vb[i] = pool.vs[at * (D / kGroup) + (unit >> 2)];
        }
    }
#pragma unroll
    for (int i = 0; i < kRowUnroll; ++i) {
        if (from[sub + i * Gm::RPI] < 0) continue;
        const size_t u = u0 + sub + i * Gm::RPI;
        if (FMT != TGVKV_CACHE_BF16) {
            kw[i] = codes_to_bf16<FMT>(make_uint2(kw[i].x, kw[i].y), kb[i], p.magic);
            vw[i] = codes_to_bf16<FMT>(make_uint2(vw[i].x, vw[i].y), vb[i], p.magic);
        }
        __stcs(reinterpret_cast<uint4*>(k_out + u * D) + unit, kw[i]);
        __stcs(reinterpret_cast<uint4*>(v_out + u * D) + unit, vw[i]);
    }
}

// Calls f with the head dimension and the format as compile-time constants.
template <int N>
struct Int {
    static constexpr int value = N;
};
template <typename F>
cudaError_t by_shape(const CacheProblem& p, F&& f) {
    auto fmt = [&](auto d) {
        if (p.format == TGVKV_CACHE_BF16) return f(d, Int<TGVKV_CACHE_BF16>());
        if (p.format == TGVKV_CACHE_INT8) return f(d, Int<TGVKV_CACHE_INT8>());
        return f(d, Int<TGVKV_CACHE_INT4>());
    };
    return p.d == 64 ? fmt(Int<64>()) : fmt(Int<128>());
}

unsigned row_blocks(long long rows, int per) {
    return rows <= 0 ? 1u : (unsigned)((rows + per - 1) / per);
}

}  // namespace

cudaError_t launch_cache_write(const CacheProblem& p, const CachePools& pool, const uint16_t* k,
                               const uint16_t* v, const long long (&strides)[4], long long rows,
                               const int64_t* row_offsets, const int32_t* tok_offsets,
                               const int32_t* page_table, const int32_t* lens, int32_t* lens_out,
                               uint32_t* status, cudaStream_t stream) {
    const WriteSource src{k, v, strides[0], strides[1], strides[2], strides[3], row_offsets,
                          tok_offsets, rows};
    return by_shape(p, [&](auto d, auto fmt) {
        constexpr int D = decltype(d)::value, FMT = decltype(fmt)::value;
        const unsigned blocks = row_blocks(rows, RowGeom<D>::ROWS);
        return launch_dependent(tok_offsets ? cache_write_kernel<D, FMT, true> : cache_write_kernel<D, FMT, false>,
                                dim3(blocks), dim3(kRowThreads), 0, stream, p, src, pool, page_table, lens,
                                lens_out, status);
    });
}

cudaError_t launch_cache_read(const CacheProblem& p, const CachePools& pool,
                              const int32_t* page_table, const int32_t* first,
                              const int64_t* offsets, uint16_t* k_out, uint16_t* v_out,
                              long long rows, uint32_t* status, cudaStream_t stream) {
    return by_shape(p, [&](auto d, auto fmt) {
        constexpr int D = decltype(d)::value, FMT = decltype(fmt)::value;
        return launch_dependent(cache_read_kernel<D, FMT>, dim3(row_blocks(rows, RowGeom<D>::ROWS)),
                                dim3(kRowThreads), 0, stream, p, pool, page_table, first, offsets, k_out,
                                v_out, rows, status);
    });
}

}  // namespace tgvkv
