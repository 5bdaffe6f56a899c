// The paged cache (cache_rows.cu writes and reads it, chunk_stream.cu and
// chunk_tile.cuh attend to it): its geometry, its integer formats and the
// conversions back to bf16.
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
// A group with an infinity or a NaN has q = 0 and E = 255, and reads back as
// NaN.  The scale is a power of two so that q 2^e is exact in bf16 (a code has
// at most 7 significant bits): reading back, and the attention kernels' bf16
// operands, add no rounding to the quantisation's own.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace tgvkv {

constexpr int kGroup = 32;             // values that share a scale
constexpr int kMinPage = 16, kMaxPage = 256;
constexpr int kMaxGroupHeads = 128;    // query heads per KV head

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

__device__ __forceinline__ uint32_t both(uint32_t half) { return half | (half << 16); }

// Eight consecutive stored codes (int4: in raw.x) of a group as bf16, in order.
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
        const uint32_t base = both(int4_base(byte));
        uint32_t t[4];   // (element j, element j + 4)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = int4x2_to_bf16(raw.x >> (4 * j), base);
        r[0] = __byte_perm(t[0], t[1], 0x5410);
        r[1] = __byte_perm(t[2], t[3], 0x5410);
        r[2] = __byte_perm(t[0], t[1], 0x7632);
        r[3] = __byte_perm(t[2], t[3], 0x7632);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

}  // namespace tgvkv
