// Rotary positions (rope.cu): the angle of a pair at a position, and rows turned by it.
#pragma once

#include "chunk.cuh"

namespace tgvkv {

constexpr int kPlanReady = 0x524F5045;   // of a plan that tgvkv_rope_init has filled

// The turns p f mod 1 of position p, as a 32-bit fraction: with f = F / 2^64 the low 64
// bits of p F are the fraction, of which the upper half is enough.  As u = p + 2^31 is not
// negative, the upper half of u F - 2^31 F takes two products; the borrow between the halves
// is left out (2^-32 turns, as the bits below are).
__device__ __forceinline__ uint32_t turn_of(int p, uint64_t f) {
    const uint32_t u = (uint32_t)p ^ 0x80000000u;
    return __umulhi(u, (uint32_t)f) + (u * (uint32_t)(f >> 32) - (uint32_t)(f >> 1));
}

// A factor in two floats.
struct Factor {
    float hi, lo;
    __host__ __device__ __forceinline__ bool one() const { return hi == 1.f && lo == 0.f; }
};

// cos and sin of t / 2^32 turns.  The nearest quarter turn is taken off, which leaves an
// angle of at most pi / 4, x + rest with rest what fp32 loses in 2 pi / 2^32 and in the
// product; there the Taylor series to x^9 and x^8 are within 2^-28 and 2^-25.  No library
// call, whose reduction of large arguments is not needed here.  (Two angles an instruction, in
// f32x2: 28.6 us against 23.4 for 220161 moved rows, as the constants need register pairs.)
// A factor a (ONE: of 1) multiplies the sums' parts, before the rounding to one float.
template <bool ONE>
__device__ __forceinline__ void cos_sin_of_turn(uint32_t t, const Factor& a, float& c, float& s) {
    const uint32_t quarter = t + 0x20000000u;                // in its top two bits
    const float r = (float)(int)(t << 2);                    // the other 30, signed: 4 / 2^32 turns
    constexpr float kStep = 3.6572953e-10f, kStepLost = -1.0177351e-17f;   // 2 pi / 2^34
    const float x = r * kStep, rest = fmaf(r, kStepLost, fmaf(r, kStep, -x));
    const float z = x * x;
    float sn = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
    sn = fmaf(sn, z, 1.f / 120.f);
    sn = fmaf(sn, z, -1.f / 6.f);
    sn = fmaf(sn * z, x, rest);            // without x
    float cs = fmaf(z, 1.f / 40320.f, -1.f / 720.f);
    cs = fmaf(cs, z, 1.f / 24.f);
    cs = fmaf(cs, z, -0.5f);               // without 1, of z
    if (ONE) {
        sn += x;
        cs = fmaf(cs, z, 1.f);
    } else {
        sn = fmaf(x, a.hi, fmaf(sn, a.hi, x * a.lo));
        cs = a.hi + fmaf(cs * z, a.hi, a.lo);
    }
    const bool odd = quarter & 0x40000000u;
    // quarters 0 .. 3: (c, s), (-s, c), (-c, -s), (s, -c)
    c = __uint_as_float(__float_as_uint(odd ? sn : cs) ^ ((quarter + 0x40000000u) & 0x80000000u));
    s = __uint_as_float(__float_as_uint(odd ? cs : sn) ^ (quarter & 0x80000000u));
}

// One tensor of a rotary call, [T][heads][d] with element strides, and where it goes.
struct RopeTensor {
    const uint16_t* x;
    long long x_tok, x_head;
    uint16_t* y;
    long long y_tok, y_head;
    int heads;
};

}  // namespace tgvkv
