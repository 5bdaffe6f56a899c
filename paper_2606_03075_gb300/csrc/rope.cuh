// Rotary positions (rope.cu): the angle of a pair at a position, and rows turned by it.
#pragma once

#include "chunk.cuh"

namespace tgvkv {

constexpr int kPlanReady = 0x524F5045;   // of a plan that tgvkv_rope_init has filled

// The turns p f mod 1 of position p, as a 32-bit fraction: with f = F / 2^64 the low 64
// bits of p F are the fraction, of which the upper half is enough (2^-32 turns).
// Wrapping arithmetic makes it right for negative positions too.
__device__ __forceinline__ uint32_t turn_of(int p, uint64_t f) {
    return (uint32_t)(((uint64_t)(int64_t)p * f) >> 32);
}

// cos and sin of t / 2^32 turns.  The nearest quarter turn is taken off, which leaves an
// angle x of at most pi / 4, where the Taylor series to x^9 and x^8 are within 2^-28 and
// 2^-25; no library call, whose reduction of large arguments is not needed here.
__device__ __forceinline__ void cos_sin_of_turn(uint32_t t, float& c, float& s) {
    const uint32_t quarter = (t + 0x20000000u) >> 30;
    const float x = (float)(int)(t - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float z = x * x;
    float sn = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
    sn = fmaf(sn, z, 1.f / 120.f);
    sn = fmaf(sn, z, -1.f / 6.f);
    sn = fmaf(sn * z, x, x);
    float cs = fmaf(z, 1.f / 40320.f, -1.f / 720.f);
    cs = fmaf(cs, z, 1.f / 24.f);
    cs = fmaf(cs, z, -0.5f);
    cs = fmaf(cs, z, 1.f);
    const bool odd = quarter & 1u;
    // quarters 0 .. 3: (c, s), (-s, c), (-c, -s), (s, -c)
    c = __uint_as_float(__float_as_uint(odd ? sn : cs) ^ (((quarter + 1u) & 2u) << 30));
    s = __uint_as_float(__float_as_uint(odd ? cs : sn) ^ ((quarter & 2u) << 30));
}

// A plan's pair i at token t: cos and sin times the attention factor.
__device__ __forceinline__ void pair_at(const tgvkv_rope_plan& plan, int i, const int32_t* positions,
                                        long long pos_stride, int t, float& c, float& s) {
    const int p = plan.axes == 1 ? positions[t] : positions[plan.axis[i] * pos_stride + t];
    cos_sin_of_turn(turn_of(p, plan.turns[i]), c, s);
    c *= plan.attention;
    s *= plan.attention;
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
