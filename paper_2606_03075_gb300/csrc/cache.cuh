// The paged cache (cache_rows.cu writes and reads it, rope.cu writes it too,
// chunk_stream.cu and chunk_tile.cuh attend to it): its geometry, its formats and
// the conversions from and to bf16.
//
// Set s = b * H_kv + g (sequence b, KV head g) owns page_table[s][0..max_pages)
// of a shared pool; its slot j is pool row page_table[s][j / page] * page +
// j % page.  A pool row holds the d values of one token of one KV head, row
// after row; K and V have a pool each, addressed by the same rows.
//
// Formats.  bf16: 2 d bytes a row.  The integer formats hold, per 32
// consecutive values x, codes q = rint(x / 2^e) (ties to even) and the byte
// E = e + 127, e being the smallest integer >= -126 with max |x| <= Q 2^e:
//   int8  Q = 127, d bytes a row, two's complement;
//   int4  Q = 7, d / 2 bytes a row, q + 8 in 4 bits, the even element in the
//         low half of a byte; e <= 120 (larger values saturate at 7 * 2^120).
// The 4-bit floats (fp4) hold codes of 1 sign, 2 exponent and 1 mantissa bits,
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} 2^e (nearest, ties to the even code), packed like
// int4, e the smallest integer in [-60, 56] with max |x| <= 6 2^e (larger values
// saturate at 6 * 2^56).
// A group with an infinity or a NaN has codes of 0 and E = 255, and reads back as
// NaN.  The scale is a power of two so that code * 2^e is exact in bf16 (a code has
// at most 7 significant bits): reading back, and the attention kernels' bf16
// operands, add no rounding to the quantisation's own.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace tgvkv {

constexpr int kGroup = 32;             // values that share a scale
constexpr int kMinPage = 16, kMaxPage = 256;
constexpr int kMaxGroupHeads = 128;    // query heads per KV head
constexpr int kFp4MinByte = 127 - 60, kFp4MaxByte = 127 + 56;   // fp4's scale bytes

struct CacheProblem {
    int B, H_q, H_kv, G, d;
    int S;                   // sets: B * H_kv
    int page, page_shift;
    int n_pages, max_pages;
    int cap;                 // slots of a set: max_pages * page
    int format;              // TGVKV_CACHE_*
    float scale_log2;        // softmax_scale * log2(e)
    uint32_t magic;          // 0x43004300, the int8 conversions' offset: as a parameter it
                             // stays in a register, so that and-or is one instruction (it
                             // is two with two immediates)
};

__host__ __device__ inline int cache_row_bytes(int d, int format) {
    return format == TGVKV_CACHE_BF16 ? 2 * d : format == TGVKV_CACHE_INT8 ? d : d / 2;
}

// One pool pair as the kernels take it.
struct CachePools {
    uint8_t* k;
    uint8_t* v;
    uint8_t* ks;             // scale bytes, d / 32 a row (null for bf16)
    uint8_t* vs;
};

__device__ __forceinline__ int clamp_len(int len, int cap) { return min(max(len, 0), cap); }

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

// ---- integer codes to bf16 ---------------------------------------------------
// With 0x4300 = 128.0 and its mantissa step 1, a code's low bits or-ed into
// the mantissa give 128 + bits exactly, and a subtraction takes the offset off
// again: no int-to-float conversion, two values an instruction.

__device__ __forceinline__ uint32_t bf16x2_sub(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_min(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_max(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two int8 codes in the low bytes of x's halves (the high bytes are ignored):
// bits 0-6 give 128 + low, bit 7 is the exponent's lowest bit, so or-ing it in
// gives 128 or 256; the difference is the two's complement value.
__device__ __forceinline__ uint32_t int8x2_to_bf16(uint32_t x, uint32_t magic) {
    return bf16x2_sub((x & 0x007F007Fu) | magic, (x & 0x00800080u) | magic);
}

// Two int4 codes (q + 8) in the low 4 bits of x's halves, times the scales
// whose `base` = int4_base(): (2^e (128 + u)) - 2^e 136 = 2^e q.
__device__ __forceinline__ uint32_t int4x2_to_bf16(uint32_t x, uint32_t base) {
    return bf16x2_sub((x & 0x000F000Fu) | base, base | 0x00080008u);
}

// bf16 bits of 2^e from the scale byte (255: infinity, which times q = 0 is NaN).
__device__ __forceinline__ uint32_t scale_bf16(uint32_t byte) { return byte << 7; }
// bf16 bits of 128 * 2^e (255: a NaN's exponent).
__device__ __forceinline__ uint32_t int4_base(uint32_t byte) { return min(byte + 7u, 255u) << 7; }

// ---- 4-bit floats to bf16 ------------------------------------------------------
// A code's exponent and mantissa bits at the low end of bf16's exponent field are
// the code's value times 2^-126, the subnormal 0.5 (bits 1) included; its sign goes
// to the top.  Codes of bits SH .. SH + 3 of x's halves.  Two shifts and two logic operations a
// pair.  The hardware's conversion gives fp16 only (and a third of the instructions): P V in
// fp16 would need a scale for P's range, and S in fp16 took as long (see chunk_stream.cu).
template <int SH>
__device__ __forceinline__ uint32_t fp4x2_small(uint32_t x) {
    const uint32_t sign = SH < 12 ? x << (12 - SH) : x;
    const uint32_t rest = SH < 6 ? x << (6 - SH) : x >> (SH > 6 ? SH - 6 : 0);
    return (sign & 0x80008000u) | (rest & 0x01C001C0u);
}
constexpr uint32_t kBf16x2Up126 = 0x7E807E80u;   // 2^126, which takes the codes to their values
constexpr uint32_t kBf16x2Up62 = 0x5E805E80u;    // 2^62

__device__ __forceinline__ uint32_t both(uint32_t half) { return half | (half << 16); }

// Eight consecutive stored codes (4 bits: in raw.x) of a group as bf16, in order.
template <int FMT>
__device__ __forceinline__ uint4 codes_to_bf16(uint2 raw, uint32_t byte, uint32_t magic) {
    uint32_t r[4];
    if (FMT == TGVKV_CACHE_INT8) {
        const uint32_t sc = both(scale_bf16(byte));
        const uint32_t words[2] = {raw.x, raw.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r[2 * i] = bf16x2_mul(int8x2_to_bf16(__byte_perm(words[i], 0, 0x4140), magic), sc);
            r[2 * i + 1] = bf16x2_mul(int8x2_to_bf16(__byte_perm(words[i], 0, 0x4342), magic), sc);
        }
    } else {
        uint32_t t[4];   // (element j, element j + 4)
        if (FMT == TGVKV_CACHE_INT4) {
            const uint32_t base = both(int4_base(byte));
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = int4x2_to_bf16(raw.x >> (4 * j), base);
        } else {
            const uint32_t sc = both(scale_bf16(byte));
            t[0] = fp4x2_small<0>(raw.x), t[1] = fp4x2_small<4>(raw.x);
            t[2] = fp4x2_small<8>(raw.x), t[3] = fp4x2_small<12>(raw.x);
#pragma unroll
            // (two factors, as 2^(126 + e) is beyond bf16; as K and V 2^-64 in one product, with the
            // factor on S and O, chunks of 0 .. 500 tokens took 369.5 us, so 368)
            for (int j = 0; j < 4; ++j) t[j] = bf16x2_mul(bf16x2_mul(t[j], kBf16x2Up126), sc);
        }
        r[0] = __byte_perm(t[0], t[1], 0x5410);
        r[1] = __byte_perm(t[2], t[3], 0x5410);
        r[2] = __byte_perm(t[0], t[1], 0x7632);
        r[3] = __byte_perm(t[2], t[3], 0x7632);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// ---- 8 values to their stored form -------------------------------------------
// The scale byte of a group from the largest magnitude among its values, as
// bf16 bits (15 bits).  With bits = 2^X' (1 + f / 128): Q = 127 needs
// e = X' - 6, one more when f > 126 (the value is above 127 * 2^(X' - 6));
// Q = 7 needs e = X' - 2, one more when f > 96; 6 needs e = X' - 2, one more when
// f > 64.
template <int FMT>
__device__ __forceinline__ int group_byte(uint32_t bits) {
    const int x = (int)(bits >> 7), f = (int)(bits & 127u);
    if (x == 255) return 255;
    if (FMT == TGVKV_CACHE_INT8) return max(x - 6 + (f > 126 ? 1 : 0), 1);
    if (FMT == TGVKV_CACHE_INT4) return min(max(x - 2 + (f > 96 ? 1 : 0), 1), 247);
    return min(max(x - 2 + (f > 64 ? 1 : 0), kFp4MinByte), kFp4MaxByte);
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
    } else if (FMT == TGVKV_CACHE_FP4) {
        // x 2^-e is exact, the conversion rounds to the nearest code (ties to even) and
        // saturates at 6
        const float inv = __uint_as_float((uint32_t)(254 - min(byte, kFp4MaxByte)) << 23);
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[2 * i] = __uint_as_float(words[i] << 16) * inv;
            y[2 * i + 1] = __uint_as_float(words[i] & 0xFFFF0000u) * inv;
        }
        uint32_t c;
        asm("{ .reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3}; }"
            : "=r"(c)
            : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
        reinterpret_cast<uint32_t*>(row)[unit] = byte == 255 ? 0u : c;
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

}  // namespace tgvkv
