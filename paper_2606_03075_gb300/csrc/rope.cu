// Rotary positions: rows turned by their tokens' positions (rope_kernel), and a serving
// step's queries, keys and values in one pass, the keys turned and stored in the paged
// cache's format (rope_write_kernel).
//
//   (y1, y2) = a (x1 c - x2 s, x2 c + x1 s),   c, s = cos, sin(p f_i)
//
// Both move each row once and are bound by HBM for long prompts, by the launch for a few
// tokens.  The rows of a token share their angles: a thread computes those of its pairs
// once and goes through heads, as many as leave the GPU filled.
#include "cache_launch.h"
#include "launch.h"
#include "rope.cuh"

namespace tgvkv {
namespace {

constexpr int kRopeThreads = 256;

// W values of bf16 as they are loaded and stored.
template <int W>
struct Words;
template <> struct Words<8> { using type = uint4; };
template <> struct Words<4> { using type = uint2; };
template <> struct Words<2> { using type = uint32_t; };
template <> struct Words<1> { using type = uint16_t; };

template <int W>
union Values {
    typename Words<W>::type w;
    uint16_t h[W];
};

__device__ __forceinline__ float bf16_value(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ uint16_t bf16_round(float x) {
    return __bfloat16_as_ushort(__float2bfloat16_rn(x));
}

// A row's units: of W pairs (values i and i + half of a turned part in halves), of W
// values (W / 2 neighbouring pairs), and of W values that are copied.
struct RopeShape {
    int units;               // of a row
    int turned;              // units that turn, the first ones
    int chunks;              // slots (groups of `units` threads) that share a token's heads
    int T;
    int heads;               // of both tensors
    bool copy_q, copy_k;     // copied values have somewhere else to go
};

// Slot (token t, chunk c) takes heads c, c + chunks, ..: neighbouring slots are at
// neighbouring rows at any moment.
template <int LAYOUT, int W>
__global__ void __launch_bounds__(kRopeThreads)
rope_kernel(const __grid_constant__ tgvkv_rope_plan plan, const RopeShape sh, const float sign,
            const int32_t* positions, const long long pos_stride, const RopeTensor q,
            const RopeTensor k) {
    constexpr bool HALF = LAYOUT == TGVKV_ROPE_HALF;
    constexpr int P = HALF ? W : W / 2;              // pairs of a unit
    constexpr int BATCH = 4;
    const int per_block = kRopeThreads / sh.units;   // slots
    const int sub = threadIdx.x / sh.units, unit = threadIdx.x - sub * sh.units;
    const unsigned slot = blockIdx.x * (unsigned)per_block + sub;
    const int t = (int)(slot / (unsigned)sh.chunks), c0 = (int)(slot - (unsigned)t * sh.chunks);
    if (sub >= per_block || t >= sh.T) return;
    const int half = plan.rot_dim >> 1;
    const bool turns = unit < sh.turned;
    // the unit's first value, and for pairs of two halves their second ones' distance
    const int at = HALF && !turns ? plan.rot_dim + (unit - sh.turned) * W : unit * W;
    float c[P], s[P];
    if (turns) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            pair_at(plan, unit * P + i, positions, pos_stride, t, c[i], s[i]);
            s[i] *= sign;
        }
    }
    for (int h0 = c0; h0 < sh.heads; h0 += BATCH * sh.chunks) {
        Values<W> a[BATCH], b[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int h = h0 + u * sh.chunks;
            if (h >= sh.heads) break;
            const RopeTensor& x = h < q.heads ? q : k;
            const uint16_t* row = x.x + t * x.x_tok + (h < q.heads ? h : h - q.heads) * x.x_head + at;
            a[u].w = *reinterpret_cast<const typename Words<W>::type*>(row);
            if (HALF && turns) b[u].w = *reinterpret_cast<const typename Words<W>::type*>(row + half);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int h = h0 + u * sh.chunks;
            if (h >= sh.heads) break;
            const bool is_q = h < q.heads;
            const RopeTensor& x = is_q ? q : k;
            uint16_t* row = x.y + t * x.y_tok + (is_q ? h : h - q.heads) * x.y_head + at;
            if (turns) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    uint16_t& h1 = a[u].h[HALF ? i : 2 * i];
                    uint16_t& h2 = HALF ? b[u].h[i] : a[u].h[(2 * i + 1) % W];
                    const float x1 = bf16_value(h1), x2 = bf16_value(h2);
                    h1 = bf16_round(fmaf(x1, c[i], -(x2 * s[i])));
                    h2 = bf16_round(fmaf(x2, c[i], x1 * s[i]));
                }
                if (HALF) *reinterpret_cast<typename Words<W>::type*>(row + half) = b[u].w;
            } else if (!(is_q ? sh.copy_q : sh.copy_k)) {
                continue;
            }
            *reinterpret_cast<typename Words<W>::type*>(row) = a[u].w;
        }
    }
}

// Slots that share a token's rows, so that few tokens fill the GPU (2048 threads an SM)
// and many compute their angles once.
int chunks_of(long long tokens, int threads_a_slot, int rows, int sms) {
    const long long want = (long long)sms * 2048, have = tokens * threads_a_slot;
    return (int)std::min<long long>(std::max<long long>((want + have - 1) / have, 1), rows);
}

template <int LAYOUT, int W>
cudaError_t launch_rope_w(const tgvkv_rope_plan& plan, RopeShape sh, float sign,
                          const int32_t* positions, long long pos_stride, const RopeTensor& q,
                          const RopeTensor& k, cudaStream_t stream) {
    const int rot = plan.rot_dim;
    sh.turned = LAYOUT == TGVKV_ROPE_HALF ? rot / 2 / W : rot / W;
    sh.units = sh.turned + (plan.d - rot) / W;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    sh.chunks = chunks_of(sh.T, sh.units, sh.heads, sms);
    const long long slots = (long long)sh.T * sh.chunks;
    const int per_block = kRopeThreads / sh.units;
    rope_kernel<LAYOUT, W><<<(unsigned)((slots + per_block - 1) / per_block), kRopeThreads, 0, stream>>>(
        plan, sh, sign, positions, pos_stride, q, k);
    return cudaGetLastError();
}

// ---- turned and stored -------------------------------------------------------------
struct RopeWrite {
    RopeTensor q;                             // y: q_out
    const uint16_t *k, *v;
    long long k_tok, k_head, v_tok, v_head;
    const int32_t* slots;                     // [T][H_kv]
    int T, rows;                              // rows of a token: H_q (0 without q) + 2 H_kv
    int chunks;
};

// Lane `unit` of a slot has values 8 unit .. 8 unit + 7 of its rows (the groups of a scale
// are then 4 neighbouring lanes, as in cache_write_kernel) and loads their partners beside
// them.  EVEN: whole vectors turn, and partners are whole vectors too.
template <int D, int FMT, int LAYOUT, bool EVEN>
__global__ void __launch_bounds__(kRopeThreads)
rope_write_kernel(const __grid_constant__ tgvkv_rope_plan plan, const CacheProblem p,
                  const RopeWrite a, const CachePools pool, const int32_t* positions,
                  const long long pos_stride, uint32_t* __restrict__ status) {
    constexpr bool HALF = LAYOUT == TGVKV_ROPE_HALF;
    constexpr int LPR = D / 8, BATCH = 2;
    constexpr int RB = FMT == TGVKV_CACHE_BF16 ? 2 * D : FMT == TGVKV_CACHE_INT8 ? D : D / 2;
    const int unit = threadIdx.x % LPR;
    const unsigned slot = blockIdx.x * (unsigned)(kRopeThreads / LPR) + threadIdx.x / LPR;
    const int t = (int)(slot / (unsigned)a.chunks), c0 = (int)(slot - (unsigned)t * a.chunks);
    const bool live = t < a.T;                // all lanes stay: the groups' maxima need them
    const int half = plan.rot_dim >> 1, e0 = 8 * unit;
    float c[8], s[8];                         // of each value; s with the sign its partner takes
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = 1.f, s[j] = 0.f;
    if (live && e0 < plan.rot_dim) {
        if (HALF) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = e0 + j;
                if (!EVEN && e >= plan.rot_dim) break;
                pair_at(plan, e < half ? e : e - half, positions, pos_stride, t, c[j], s[j]);
                if (e < half) s[j] = -s[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                if (!EVEN && e0 + j >= plan.rot_dim) break;
                pair_at(plan, (e0 + j) >> 1, positions, pos_stride, t, c[j], s[j + 1]);
                c[j + 1] = c[j];
                s[j] = -s[j + 1];
            }
        }
    }
    const long long pool_rows = (long long)p.n_pages * p.page;
    const int n_q = a.q.heads;
    for (int r0 = 0; r0 < a.rows; r0 += BATCH * a.chunks) {
        Values<8> x[BATCH], y[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int r = r0 + u * a.chunks + c0;
            x[u].w = y[u].w = make_uint4(0u, 0u, 0u, 0u);
            if (!live || r >= a.rows) continue;
            const bool is_v = r >= n_q + p.H_kv;
            const uint16_t* row = r < n_q ? a.q.x + t * a.q.x_tok + r * a.q.x_head
                                  : is_v  ? a.v + t * a.v_tok + (r - n_q - p.H_kv) * a.v_head
                                          : a.k + t * a.k_tok + (r - n_q) * a.k_head;
            x[u].w = *reinterpret_cast<const uint4*>(row + e0);
            if (HALF && !is_v && e0 < plan.rot_dim) {
                if (EVEN) {
                    y[u].w = *reinterpret_cast<const uint4*>(row + (e0 < half ? e0 + half : e0 - half));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = e0 + j;
                        if (e < plan.rot_dim) y[u].h[j] = row[e < half ? e + half : e - half];
                    }
                }
            }
        }
        __syncwarp();                          // q_out may be q: every partner is read by now
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int r = r0 + u * a.chunks + c0;
            const bool mine = live && r < a.rows, is_q = r < n_q, is_v = r >= n_q + p.H_kv;
            if (mine && !is_v && e0 < plan.rot_dim) {
                Values<8> z;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint16_t other = HALF ? y[u].h[j] : x[u].h[j ^ 1];
                    z.h[j] = bf16_round(fmaf(bf16_value(x[u].h[j]), c[j], bf16_value(other) * s[j]));
                    if (!EVEN && e0 + j >= plan.rot_dim) z.h[j] = x[u].h[j];
                }
                x[u] = z;
            }
            if (mine && is_q)
                reinterpret_cast<uint4*>(a.q.y + t * a.q.y_tok + r * a.q.y_head)[unit] = x[u].w;
            const bool stores = mine && !is_q;
            int at = -1;
            if (stores) {
                at = a.slots[(size_t)t * p.H_kv + (is_v ? r - n_q - p.H_kv : r - n_q)];
                if (at >= pool_rows) {
                    if (unit == 0) raise_status(status, TGVKV_STATUS_INDEX);
                    at = -1;
                }
            }
            const bool on = at >= 0;
            const size_t row = on ? at : 0;
            uint8_t* to = is_v ? pool.v : pool.k;
            if (FMT == TGVKV_CACHE_BF16) {
                if (on) reinterpret_cast<uint4*>(to + row * RB)[unit] = x[u].w;
            } else if (__any_sync(~0u, on)) {
                store_row<FMT>(x[u].w, to + row * RB, (is_v ? pool.vs : pool.ks) + row * (D / kGroup), unit, on);
            }
        }
    }
}

template <int D, int FMT, int LAYOUT, bool EVEN>
cudaError_t launch_write(const CacheProblem& p, const CachePools& pool, const tgvkv_rope_plan& plan,
                         RopeWrite a, const int32_t* positions, long long pos_stride, uint32_t* status,
                         cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    a.chunks = chunks_of(a.T, D / 8, a.rows, sms);
    constexpr int per_block = kRopeThreads / (D / 8);
    const long long slots = (long long)a.T * a.chunks;
    rope_write_kernel<D, FMT, LAYOUT, EVEN>
        <<<(unsigned)((slots + per_block - 1) / per_block), kRopeThreads, 0, stream>>>(
            plan, p, a, pool, positions, pos_stride, status);
    return cudaGetLastError();
}

template <int D, int FMT>
cudaError_t launch_write_by_layout(const CacheProblem& p, const CachePools& pool,
                                   const tgvkv_rope_plan& plan, const RopeWrite& a,
                                   const int32_t* positions, long long pos_stride, uint32_t* status,
                                   cudaStream_t stream) {
    if (plan.layout == TGVKV_ROPE_HALF)
        return plan.rot_dim % 16 == 0
                   ? launch_write<D, FMT, TGVKV_ROPE_HALF, true>(p, pool, plan, a, positions, pos_stride, status, stream)
                   : launch_write<D, FMT, TGVKV_ROPE_HALF, false>(p, pool, plan, a, positions, pos_stride, status, stream);
    return plan.rot_dim % 8 == 0
               ? launch_write<D, FMT, TGVKV_ROPE_INTERLEAVED, true>(p, pool, plan, a, positions, pos_stride, status, stream)
               : launch_write<D, FMT, TGVKV_ROPE_INTERLEAVED, false>(p, pool, plan, a, positions, pos_stride, status, stream);
}

template <int D>
cudaError_t launch_write_by_format(const CacheProblem& p, const CachePools& pool,
                                   const tgvkv_rope_plan& plan, const RopeWrite& a,
                                   const int32_t* positions, long long pos_stride, uint32_t* status,
                                   cudaStream_t stream) {
    switch (p.format) {
        case TGVKV_CACHE_BF16: return launch_write_by_layout<D, TGVKV_CACHE_BF16>(p, pool, plan, a, positions, pos_stride, status, stream);
        case TGVKV_CACHE_INT8: return launch_write_by_layout<D, TGVKV_CACHE_INT8>(p, pool, plan, a, positions, pos_stride, status, stream);
        case TGVKV_CACHE_INT4: return launch_write_by_layout<D, TGVKV_CACHE_INT4>(p, pool, plan, a, positions, pos_stride, status, stream);
        default: return launch_write_by_layout<D, TGVKV_CACHE_FP4>(p, pool, plan, a, positions, pos_stride, status, stream);
    }
}

}  // namespace

cudaError_t launch_rope(const tgvkv_rope_plan& plan, int mode, const int32_t* positions,
                        long long pos_stride, int T, const RopeTensor& q, const RopeTensor& k,
                        cudaStream_t stream) {
    tgvkv_rope_plan used = plan;
    if (mode == TGVKV_ROPE_MOVE) used.attention = 1.f;
    const float sign = mode == TGVKV_ROPE_GRADIENT ? -1.f : 1.f;
    RopeShape sh{};
    sh.T = T;
    sh.heads = q.heads + k.heads;
    sh.copy_q = q.x != q.y;
    sh.copy_k = k.x != k.y;
    // the widest load that pairs and their partners allow (rows are 16-byte aligned)
    const int step = plan.layout == TGVKV_ROPE_HALF ? plan.rot_dim / 2 : plan.rot_dim;
    if (plan.layout == TGVKV_ROPE_HALF) {
        if (step % 8 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 8>(used, sh, sign, positions, pos_stride, q, k, stream);
        if (step % 4 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 4>(used, sh, sign, positions, pos_stride, q, k, stream);
        if (step % 2 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 2>(used, sh, sign, positions, pos_stride, q, k, stream);
        return launch_rope_w<TGVKV_ROPE_HALF, 1>(used, sh, sign, positions, pos_stride, q, k, stream);
    }
    if (step % 8 == 0) return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 8>(used, sh, sign, positions, pos_stride, q, k, stream);
    if (step % 4 == 0) return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 4>(used, sh, sign, positions, pos_stride, q, k, stream);
    return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 2>(used, sh, sign, positions, pos_stride, q, k, stream);
}

cudaError_t launch_rope_write(const CacheProblem& p, const CachePools& pool,
                              const tgvkv_rope_plan& plan, const int32_t* positions,
                              long long pos_stride, const int32_t* slots, int T, const RopeTensor& q,
                              const uint16_t* k, const uint16_t* v, const long long (&strides)[4],
                              uint32_t* status, cudaStream_t stream) {
    RopeWrite a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.k_tok = strides[0], a.k_head = strides[1], a.v_tok = strides[2], a.v_head = strides[3];
    a.slots = slots;
    a.T = T;
    a.rows = q.heads + 2 * p.H_kv;
    return p.d == 64 ? launch_write_by_format<64>(p, pool, plan, a, positions, pos_stride, status, stream)
                     : launch_write_by_format<128>(p, pool, plan, a, positions, pos_stride, status, stream);
}

}  // namespace tgvkv
