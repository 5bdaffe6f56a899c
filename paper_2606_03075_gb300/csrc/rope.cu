// Rotary positions: rows turned by their tokens' positions (rope_kernel, and rope_one_kernel
// for tensors of one row a token), and a serving step's queries, keys and values in one pass,
// the keys turned and stored in the paged cache's format (rope_write_kernel).
//
//   (y1, y2) = a (x1 c - x2 s, x2 c + x1 s),   c, s = cos, sin(p f_i)
//
// All move each row once and are bound by HBM for long prompts, by the launch for a few
// tokens.  An angle's c and s take about 30 instructions, a pair itself 4, so the rows of a
// token share them: a CTA goes through tiles of a tensor's tokens, starts a tile's first
// loads, computes its angles into shared memory meanwhile, and turns the rows, kRopeRows in
// flight a thread.  What a row needs beside its arithmetic counts, too (of some 60
// instructions a 16-byte vector): a thread keeps to one tensor and to one row of its
// tokens, so that addresses go on by constants.
//
// Measured, calls one after another (us; the bytes alone at a copy's rate in brackets): queries
// and keys of 8704 tokens, 28 + 4 rows of 128 on three axes 26.0 (21.1); gradients of 16381
// tokens, 32 + 8 rows of which 64 values are turned 53.2 (49.7); 220161 rows moved 22.6 (16.8),
// which have an angle of their own for every pair; sixteen prompts of 2049 .. 4099 tokens,
// 32 + 8 + 8 rows, into int8 pages and read back 236 (211); one token 2.5, 64 tokens into
// bf16 pages 3.5, the launch.
#include "cache_launch.h"
#include "launch.h"
#include "rope.cuh"

namespace tgvkv {
namespace {

constexpr int kRopeThreads = 256;
// Rows a thread has in flight and CTAs of an SM.  Gradients / sixteen prompts (us): 3 and 4
// 53.8 / 237; 2 and 4 59.2 / 235; 4 and 4 54.2 / 242; 3 and 3 59.3 / 236; 3 and 5 (the registers
// end) 56.8 / 241.
constexpr int kRopeRows = 3;
constexpr int kRopeResident = 4;
// CTAs of rope_one_kernel: 220161 rows 23.5 us at 3, 25.5 at 2, 35 at 4 (which spills).
constexpr int kOneResident = 3;
// Angles of a tile (32 KB for two tables); no difference from 1024 to 4096.
constexpr int kTableAngles = 2048;
// Tiles of a CTA at least where a token's rows are cut into parts for the groups' sake.
constexpr int kTilesEach = 2;

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
    uint32_t two[W > 1 ? W / 2 : 1];
    uint16_t h[W];
};

__device__ __forceinline__ float low_value(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float high_value(uint32_t two) { return __uint_as_float(two & 0xFFFF0000u); }
// y1 and y2 of a pair
__device__ __forceinline__ float first_of(float x1, float x2, float c, float s) { return fmaf(x1, c, -(x2 * s)); }
__device__ __forceinline__ float second_of(float x1, float x2, float c, float s) { return fmaf(x2, c, x1 * s); }

// What angles are made of.
struct Angles {
    const int32_t* positions;
    long long pos_stride;
    Factor attention;
    int axes;
    int pairs;                                // of a row
    int T;                                    // tokens
};

// A plan's pairs in shared memory: lanes that read different ones of a parameter wait for one
// another.
struct PlanPairs {
    uint64_t turns[TGVKV_ROPE_MAX_DIM / 2];
    uint8_t axis[TGVKV_ROPE_MAX_DIM / 2];

    __device__ __forceinline__ void take(const tgvkv_rope_plan& plan, int pairs) {
        for (int i = threadIdx.x; i < pairs; i += kRopeThreads) turns[i] = plan.turns[i], axis[i] = plan.axis[i];
        __syncthreads();
    }
};

// Where pair i's (c, s) lies among a token's: the P pairs of a unit are read two at a time,
// by neighbouring units from neighbouring places.
template <int P>
__device__ __forceinline__ int angle_place(int i, int pairs) {
    if (P == 1) return i;
    const int unit = i / P, j = i % P;
    return ((j >> 1) * (pairs / P) + unit) * 2 + (j & 1);
}

// The angles of n tokens from t0 on into `table`, [token][pairs], by the CTA.
template <int P>
__device__ __forceinline__ void make_angles(const Angles& an, const PlanPairs& pp, int t0, int n, float2* table) {
    int t = threadIdx.x / an.pairs, i = threadIdx.x - t * an.pairs;
    const int dt = kRopeThreads / an.pairs, di = kRopeThreads - dt * an.pairs;
    while (t < n) {
        const int32_t* of_token = an.positions + t0 + t;
        const int p = an.axes == 1 ? *of_token : of_token[pp.axis[i] * an.pos_stride];
        float c, s;
        if (an.attention.one()) cos_sin_of_turn<true>(turn_of(p, pp.turns[i]), an.attention, c, s);
        else cos_sin_of_turn<false>(turn_of(p, pp.turns[i]), an.attention, c, s);
        table[t * an.pairs + angle_place<P>(i, an.pairs)] = make_float2(c, s);
        t += dt, i += di;
        if (i >= an.pairs) i -= an.pairs, ++t;
    }
}

// The P pairs of unit `unit` of one token.
template <int P>
__device__ __forceinline__ void take_angles(const float2* of_token, int unit, int pairs, float (&c)[P], float (&s)[P]) {
    if constexpr (P == 1) {
        c[0] = of_token[unit].x, s[0] = of_token[unit].y;
    } else {
#pragma unroll
        for (int j = 0; j < P; j += 2) {
            const float4 two = reinterpret_cast<const float4*>(of_token)[(j >> 1) * (pairs / P) + unit];
            c[j] = two.x, s[j] = two.y, c[j + 1] = two.z, s[j + 1] = two.w;
        }
    }
}

// A tensor's rows cut into tiles of `tokens` tokens: groups of threads take `rows` of a token's
// rows at a time, `parts` times, of `side` tokens side by side, and of the `deep` tokens that
// are `side` apart.  The tiles of a call's tensors, one tensor after another, go round the
// CTAs, so that each has as many as any other.
struct Tiles {
    int before;                               // tiles of the tensors before
    int count;
    int side, deep, tokens, rows, parts;
    unsigned magic;                           // n / rows = n * magic >> 16 for n < 256
};

// Where a CTA is among its tiles and their parts.
struct Step {
    int tile, part;

    __device__ __forceinline__ explicit Step(const Tiles& ti)
        : tile((int)((blockIdx.x + gridDim.x - ti.before % gridDim.x) % gridDim.x)), part(0) {}

    __device__ __forceinline__ void next(const Tiles& ti) {
        if (++part == ti.parts) part = 0, tile += gridDim.x;
    }
    // every token of the tile is there, kRopeRows deep
    __device__ __forceinline__ bool full(const Tiles& ti, int T) const {
        return ti.deep == kRopeRows && (long long)tile * ti.tokens + ti.tokens <= T;
    }
};

// A group's place in every tile: row r of a part, token `of` of those side by side.
struct Place {
    int of, r;

    __device__ __forceinline__ Place(const Tiles& ti, int group) {
        of = (int)(group * ti.magic >> 16);
        r = group - of * ti.rows;
    }
    // how many of the tokens of, of + side, .. it has rows of: the row u is u * side < left
    __device__ __forceinline__ int left(const Tiles& ti, const Step& st, int heads, int T) const {
        if (of >= ti.side || st.part * ti.rows + r >= heads || st.tile >= ti.count) return 0;
        return min(T - st.tile * ti.tokens, ti.tokens) - of;
    }
};

// A thread's address in a tensor, which goes on by constants: `side` to the next of its rows
// in a tile, then on to the next part or tile.
template <typename T>
struct Walk {
    T* at;
    long long side, part, tile;

    __device__ __forceinline__ Walk(const Tiles& ti, const Step& st, const Place& pl, T* base, long long tok,
                                    long long head, int value) {
        at = base + ((long long)st.tile * ti.tokens + pl.of) * tok + pl.r * head + value;
        side = ti.side * tok;
        part = ti.rows * head;
        tile = (long long)gridDim.x * ti.tokens * tok - (ti.parts - 1) * part;
    }
    __device__ __forceinline__ void next(const Tiles& ti, const Step& st) {
        at += st.part + 1 < ti.parts ? part : tile;
    }
};

// Calls f(u, address) for the rows of a part that the thread has, without a test a row where
// the tile is full.
template <typename T, typename F>
__device__ __forceinline__ void for_rows(const Tiles& ti, const Step& st, int left, int tokens,
                                         const Walk<T>& walk, F&& f) {
    T* at = walk.at;
    if (st.full(ti, tokens)) {
        if (left > 0) {
#pragma unroll
            for (int u = 0; u < kRopeRows; ++u, at += walk.side) f(u, at);
        }
    } else {
#pragma unroll
        for (int u = 0; u < kRopeRows; ++u, at += walk.side)
            if (u * ti.side < left) f(u, at);
    }
}

// Host: the tiles of the tokens' `heads` rows for CTAs of `groups` groups: kRopeRows tokens deep,
// less where that would leave SMs without one, or where their angles would exceed
// kTableAngles.
Tiles make_tiles(const Angles& an, int heads, int groups, int busy, int sms) {
    Tiles ti{};
    if (heads == 0) return ti;
    ti.parts = (heads + groups - 1) / groups;
    ti.rows = (heads + ti.parts - 1) / ti.parts;
    ti.side = groups / ti.rows;
    // Smaller parts of more tokens while less than busy / 16 of the groups are busy and there are
    // tiles enough.  200 MB in halves (12), us: 28 rows of 64 values, 32 turned (42 groups) 77.6, so
    // 65.5; 12 rows of 128, 64 turned (21 groups) 88.6, so 74.3; 28 rows of 96 (42 groups) 65.3, so 73.6;
    // at 13, 12 rows of 128 (32 groups) 67.5, so 74.7.  Neighbouring pairs, whose threads hold half as
    // many bytes (13): 12 rows of 128 (16 groups) 77.8, so 66.8; at 15, 28 rows 65.3, so 70.
    for (int parts = ti.parts + 1;
         16LL * heads * ti.side < (long long)busy * groups * ti.parts && parts <= std::min(heads, 16); ++parts) {
        const int rows = (heads + parts - 1) / parts, side = groups / rows, deep = side * kRopeRows;
        if ((long long)kTilesEach * deep * sms * kRopeResident > an.T || deep * an.pairs > kTableAngles) break;
        if (side * ti.parts > ti.side * parts) ti.parts = parts, ti.rows = rows, ti.side = side;
    }
    ti.deep = std::min(std::min(an.T / (ti.side * sms), kTableAngles / (ti.side * an.pairs)), kRopeRows);
    ti.deep = std::max(ti.deep, 1);
    ti.tokens = ti.side * ti.deep;
    ti.count = (int)(((long long)an.T + ti.tokens - 1) / ti.tokens);
    ti.magic = (65536u + ti.rows - 1) / ti.rows;
    return ti;
}

// Host: CTAs for tensors' tiles, as many as are resident at a time; *table: angles of the
// largest tile.
template <int N>
unsigned count_blocks(Tiles* (&ti)[N], int pairs, int sms, int* table) {
    long long all = 0;
    *table = 0;
    for (Tiles* t : ti) {
        t->before = (int)(all % ((long long)sms * kRopeResident));    // only its place among them counts
        all += t->count;
        *table = std::max(*table, t->tokens * pairs);
    }
    return (unsigned)std::min<long long>(all, (long long)sms * kRopeResident);
}

// How a row is cut into units, a thread each: `turned` of W pairs (halves) or W values
// (neighbouring pairs), `narrow` of W values that are copied, up to a multiple of 8, and the rest
// of 8 values that are copied.  (Copies as narrow as the pairs, 200 MB of 8 rows a token in halves:
// 20 of 80 values turned 231 us, so 106; 24 of 96 130, so 97.)
struct Cut {
    int turned, narrow, units;

    template <int LAYOUT, int W>
    static Cut of(int d, int rot) {
        const int wide = (rot + 7) / 8 * 8, turned = LAYOUT == TGVKV_ROPE_HALF ? rot / 2 / W : rot / W;
        const int narrow = (wide - rot) / W;
        return Cut{turned, narrow, turned + narrow + (d - wide) / 8};
    }
};

// A unit of a row: what it holds between its load and its store.
template <int LAYOUT, int W>
struct Unit {
    using Word = typename Words<W>::type;
    static constexpr bool HALF = LAYOUT == TGVKV_ROPE_HALF;
    static constexpr int P = HALF ? W : W / 2;
    Values<W> x, y;                           // values; second halves
    uint4 z;                                  // of a wide copy (W = 8: in x)

    // a thread's kind of unit, and where it begins
    struct Kind {
        bool turns, wide;
        int first;

        __device__ __forceinline__ Kind(const Cut& cut, int unit, int rot) {
            turns = unit < cut.turned;
            wide = W < 8 && unit >= cut.turned + cut.narrow;
            first = HALF && !turns ? rot + (unit - cut.turned) * W : unit * W;
            if (wide) first = (rot + 7) / 8 * 8 + (unit - cut.turned - cut.narrow) * 8;
        }
    };
    __device__ __forceinline__ void load(const uint16_t* row, const Kind& kind, int half) {
        if (kind.wide) {
            z = *reinterpret_cast<const uint4*>(row);
        } else {
            x.w = *reinterpret_cast<const Word*>(row);
            if (HALF && kind.turns) y.w = *reinterpret_cast<const Word*>(row + half);
        }
    }
    // (of a turned unit in halves: the first one, the second is stored where it was turned)
    __device__ __forceinline__ void store(uint16_t* row, const Kind& kind, bool moves) const {
        if (kind.wide) {
            if (moves) *reinterpret_cast<uint4*>(row) = z;
        } else if (kind.turns || moves) {
            *reinterpret_cast<Word*>(row) = x.w;
        }
    }
    __device__ __forceinline__ void store_second(uint16_t* row, int half) const {
        if (HALF) *reinterpret_cast<Word*>(row + half) = y.w;
    }

    __device__ __forceinline__ void turn(const float (&c)[P], const float (&s)[P]) {
        if constexpr (!HALF) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float x1 = low_value(x.two[i]), x2 = high_value(x.two[i]);
                x.two[i] = pack_bf16x2(first_of(x1, x2, c[i], s[i]), second_of(x1, x2, c[i], s[i]));
            }
        } else if constexpr (W > 1) {
#pragma unroll
            for (int i = 0; i < P; i += 2) {
                uint32_t &f = x.two[i / 2], &g = y.two[i / 2];
                const float x1 = low_value(f), x2 = low_value(g), z1 = high_value(f), z2 = high_value(g);
                f = pack_bf16x2(first_of(x1, x2, c[i], s[i]), first_of(z1, z2, c[i + 1], s[i + 1]));
                g = pack_bf16x2(second_of(x1, x2, c[i], s[i]), second_of(z1, z2, c[i + 1], s[i + 1]));
            }
        } else {
            const float x1 = low_value(x.h[0]), x2 = low_value(y.h[0]);
            const uint32_t two = pack_bf16x2(first_of(x1, x2, c[0], s[0]), second_of(x1, x2, c[0], s[0]));
            x.h[0] = (uint16_t)two;
            y.h[0] = (uint16_t)(two >> 16);
        }
    }
};

// A call's rows.
struct RopeCall {
    RopeTensor q, k;
    Tiles q_tiles, k_tiles;
    int table;                                // angles of the largest tile
    Cut cut;
};

template <int LAYOUT, int W>
__global__ void __launch_bounds__(kRopeThreads, kRopeResident)
rope_kernel(const __grid_constant__ tgvkv_rope_plan plan, const __grid_constant__ RopeCall a,
            const __grid_constant__ Angles an) {
    using U = Unit<LAYOUT, W>;
    constexpr int P = U::P;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ PlanPairs pp;
    const int group = threadIdx.x / a.cut.units, unit = threadIdx.x - group * a.cut.units;
    const int half = plan.rot_dim >> 1;
    const typename U::Kind kind(a.cut, unit, plan.rot_dim);
    pp.take(plan, an.pairs);
    griddep_launch_dependents();       // the next call's set-up may overlap this one
    griddep_wait();
    float2* table = reinterpret_cast<float2*>(smem);           // two, in turn
    int flip = 0;
    for (int tensor = 0; tensor < 2; ++tensor) {
        const RopeTensor x = tensor ? a.k : a.q;
        const Tiles ti = tensor ? a.k_tiles : a.q_tiles;
        Step st(ti);
        if (st.tile >= ti.count) continue;
        const bool moves = x.x != x.y;
        const Place place(ti, group);
        Walk<const uint16_t> from(ti, st, place, x.x, x.x_tok, x.x_head, kind.first);
        Walk<uint16_t> to(ti, st, place, x.y, x.y_tok, x.y_head, kind.first);
        U v[kRopeRows];
        auto load = [&](const Step& of) {
            for_rows(ti, of, place.left(ti, of, x.heads, an.T), an.T, from,
                     [&](int u, const uint16_t* row) { v[u].load(row, kind, half); });
        };
        load(st);
        for (; st.tile < ti.count; flip ^= 1) {
            float2* angles = table + flip * a.table;
            const int t0 = st.tile * ti.tokens;
            make_angles<P>(an, pp, t0, min(ti.tokens, an.T - t0), angles);
            __syncthreads();       // (and all are done with the other table, the next tile's)
            angles += place.of * an.pairs;
            const int deeper = ti.side * an.pairs;
            for (int part = 0; part < ti.parts; ++part) {
                for_rows(ti, st, place.left(ti, st, x.heads, an.T), an.T, to, [&](int u, uint16_t* row) {
                    if (kind.turns) {
                        float c[P], s[P];
                        take_angles<P>(angles + u * deeper, unit, an.pairs, c, s);
                        v[u].turn(c, s);
                        v[u].store_second(row, half);
                    }
                    v[u].store(row, kind, moves);
                });
                from.next(ti, st);
                to.next(ti, st);
                st.next(ti);
                load(st);
            }
        }
    }
}

// One row a token, of every tensor: there is nothing to share, every thread computes the angles of
// its rows.  ONE: the attention factor is 1 (220161 rows 22.6 us, with a branch 27).
template <int LAYOUT, int W, bool ONE>
__global__ void __launch_bounds__(kRopeThreads, kOneResident)
rope_one_kernel(const __grid_constant__ tgvkv_rope_plan plan, const RopeTensor x, const __grid_constant__ Cut cut,
                const __grid_constant__ Angles an) {
    using U = Unit<LAYOUT, W>;
    constexpr int P = U::P, N = 2;
    const int units = cut.units;
    const int groups = kRopeThreads / units, group = threadIdx.x / units, unit = threadIdx.x - group * units;
    if (group >= groups) return;
    const int half = plan.rot_dim >> 1;
    const bool moves = x.x != x.y;
    const typename U::Kind kind(cut, unit, plan.rot_dim);
    uint64_t f[P];
#pragma unroll
    for (int i = 0; i < P; ++i) f[i] = plan.turns[kind.turns ? unit * P + i : 0];
    const long long step = (long long)gridDim.x * groups;
    long long t = (long long)blockIdx.x * groups + group, loads = t;
    const uint16_t* from = x.x + t * x.x_tok + kind.first;
    uint16_t* to = x.y + t * x.y_tok + kind.first;
    const long long from_step = step * x.x_tok, to_step = step * x.y_tok;
    U v[N];
    int p[N];
    auto load = [&](int u) {
        if (loads < an.T) {
            v[u].load(from, kind, half);
            p[u] = an.positions[loads];
        }
        loads += step;
        from += from_step;
    };
    griddep_launch_dependents();
    griddep_wait();
#pragma unroll
    for (int u = 0; u < N; ++u) load(u);
    while (t < an.T) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (t >= an.T) break;
            if (kind.turns) {
                float c[P], s[P];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int pi = an.axes == 1 ? p[u] : an.positions[plan.axis[unit * P + i] * an.pos_stride + t];
                    cos_sin_of_turn<ONE>(turn_of(pi, f[i]), an.attention, c[i], s[i]);
                }
                v[u].turn(c, s);
                v[u].store_second(to, half);
            }
            v[u].store(to, kind, moves);
            to += to_step;
            t += step;
            load(u);
        }
    }
}

template <int LAYOUT, int W>
cudaError_t launch_rope_w(const tgvkv_rope_plan& plan, RopeCall a, const Angles& an, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    a.cut = Cut::of<LAYOUT, W>(plan.d, plan.rot_dim);
    const int groups = kRopeThreads / a.cut.units;
    // Rows of one head go with another tensor's of more: one launch, and 200 MB of 12 + 1 rows of
    // 96 values, 64 turned, 73.5 us, not 94 in two that overlap (of 128, all turned, 70 and 67).
    for (RopeTensor* x : {&a.q, &a.k}) {
        if (x->heads != 1 || a.q.heads > 1 || a.k.heads > 1) continue;
        const unsigned blocks = (unsigned)std::min<long long>(((long long)an.T + groups - 1) / groups,
                                                              (long long)sms * kOneResident);
        auto kernel = rope_one_kernel<LAYOUT, W, false>;
        if (an.attention.one()) kernel = rope_one_kernel<LAYOUT, W, true>;
        const cudaError_t e = launch_early(kernel, dim3(blocks), dim3(kRopeThreads), 0, stream, plan, *x, a.cut, an);
        if (e != cudaSuccess) return e;
        x->heads = 0;
    }
    if (a.q.heads + a.k.heads == 0) return cudaSuccess;
    constexpr int busy = LAYOUT == TGVKV_ROPE_HALF ? 12 : 13;
    a.q_tiles = make_tiles(an, a.q.heads, groups, busy, sms);
    a.k_tiles = make_tiles(an, a.k.heads, groups, busy, sms);
    Tiles* tiles[2] = {&a.q_tiles, &a.k_tiles};
    const unsigned blocks = count_blocks(tiles, an.pairs, sms, &a.table);
    const size_t smem = 2 * sizeof(float2) * a.table;
    return launch_early(rope_kernel<LAYOUT, W>, dim3(blocks), dim3(kRopeThreads), smem, stream, plan, a, an);
}

// ---- turned and stored -------------------------------------------------------------
struct RopeWrite {
    RopeTensor q;                             // y: q_out; no heads where there are no queries
    RopeTensor k, v;                          // y: none
    Tiles q_tiles, k_tiles, v_tiles;
    int table;                                // angles of the largest tile
    const int32_t* slots;                     // [T][H_kv]
    bool early;                               // lets the next call's set-up overlap
};

// One vector of 8 values into row `row` of a pool (-1: none), `unit` being the vector's number
// in its row; 4 neighbouring lanes have 4 neighbouring vectors.
template <int D, int FMT>
__device__ __forceinline__ void store_vector(uint4 w, uint8_t* rows, uint8_t* scales, int row, int unit) {
    constexpr int RB = FMT == TGVKV_CACHE_BF16 ? 2 * D : FMT == TGVKV_CACHE_INT8 ? D : D / 2;
    const size_t at = row >= 0 ? row : 0;
    if (FMT == TGVKV_CACHE_BF16) {
        if (row >= 0) reinterpret_cast<uint4*>(rows + at * RB)[unit] = w;
    } else {                           // lanes without a row take part in the maxima
        store_row<FMT>(w, rows + at * RB, scales + at * (D / kGroup), unit, row >= 0);
    }
}

// The lanes of a group hold a row's vectors of 8 values so that a scale's 4 vectors are in 4
// neighbouring lanes.
enum Hold {
    // lane i has vectors i and i + D / 16, which are each other's partners in halves (whole heads
    // in halves, and neighbouring pairs)
    kTwo,
    // lane i has vector i, and loads beside it the vector of its partners (a part of a head in
    // halves that is a multiple of 16)
    kPartners,
    // lane i has vector i, and loads the partners one by one (parts that end inside a vector.
    // For every part of a head, 200 MB of 32 + 8 + 8 rows, 64 of 128 values turned: bf16 117 us, as
    // partner vectors 69.5; int8 126, so 74)
    kSingly
};
template <int D, int FMT, int LAYOUT, int HOLD>
__global__ void __launch_bounds__(kRopeThreads, kRopeResident)
rope_write_kernel(const __grid_constant__ tgvkv_rope_plan plan, const __grid_constant__ RopeWrite a,
                  const __grid_constant__ Angles an, const CacheProblem p, const CachePools pool,
                  uint32_t* __restrict__ status) {
    constexpr bool HALF = LAYOUT == TGVKV_ROPE_HALF;
    constexpr bool TWO = HOLD == kTwo;
    constexpr int LPR = TWO ? D / 16 : D / 8, P = HALF ? 8 : 4;
    constexpr int PLACED = HOLD == kSingly ? 1 : P;            // how the angles lie in their table
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ PlanPairs pp;
    const int unit = threadIdx.x % LPR, half = plan.rot_dim >> 1, e0 = 8 * unit;
    const int pool_rows = p.n_pages * p.page;          // below 2^31
    pp.take(plan, an.pairs);
    if (a.early) griddep_launch_dependents();
    griddep_wait();
    float2* table = reinterpret_cast<float2*>(smem);           // two, in turn
    int flip = 0;
    // Queries, keys and values, from a tensor on that differs by CTA, as one is bound by
    // arithmetic and another by memory.
    for (int i = 0, tensor = blockIdx.x % 3; i < 3; ++i, tensor = tensor == 2 ? 0 : tensor + 1) {
        const bool is_q = tensor == 0, is_v = tensor == 2;
        const RopeTensor x = is_q ? a.q : is_v ? a.v : a.k;
        const Tiles ti = is_q ? a.q_tiles : is_v ? a.v_tiles : a.k_tiles;
        Step st(ti);
        if (st.tile >= ti.count) continue;
        uint8_t* rows = is_v ? pool.v : pool.k;
        uint8_t* scales = is_v ? pool.vs : pool.ks;
        const Place place(ti, threadIdx.x / LPR);
        Walk<const uint16_t> from(ti, st, place, x.x, x.x_tok, x.x_head, e0);
        Walk<uint16_t> to(ti, st, place, x.y, x.y_tok, x.y_head, e0);          // of queries
        Values<8> v[kRopeRows], w[kRopeRows];     // the values; the other vector, or the partners
        int row_of[kRopeRows];                    // pool rows
        auto load = [&](const Step& of) {
            const int left = place.left(ti, of, x.heads, an.T);
#pragma unroll
            for (int u = 0; u < kRopeRows; ++u) row_of[u] = -1;
            if (!is_q) {
                const int at = (of.tile * ti.tokens + place.of) * p.H_kv + of.part * ti.rows + place.r;   // below 2^31
#pragma unroll
                for (int u = 0; u < kRopeRows; ++u)
                    if (u * ti.side < left) row_of[u] = a.slots[at + u * ti.side * p.H_kv];
            }
            for_rows(ti, of, left, an.T, from, [&](int u, const uint16_t* row) {
                v[u].w = *reinterpret_cast<const uint4*>(row);
                if (TWO) {
                    w[u].w = *reinterpret_cast<const uint4*>(row + D / 2);
                } else if (HOLD == kPartners) {
                    if (!is_v && e0 < plan.rot_dim)
                        w[u].w = *reinterpret_cast<const uint4*>(e0 < half ? row + half : row - half);
                } else if (HALF && !is_v) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = e0 + j;
                        w[u].h[j] = e < plan.rot_dim ? row[e < half ? j + half : j - half] : 0;
                    }
                }
            });
        };
#pragma unroll
        for (int u = 0; u < kRopeRows; ++u) v[u].w = w[u].w = make_uint4(0u, 0u, 0u, 0u);
        load(st);
        while (st.tile < ti.count) {
            float2* angles = table + flip * a.table;
            if (!is_v) {
                flip ^= 1;
                const int t0 = st.tile * ti.tokens;
                make_angles<PLACED>(an, pp, t0, min(ti.tokens, an.T - t0), angles);
                __syncthreads();   // (and all are done with the other table, the next tile's)
            }
            angles += place.of * an.pairs;
            const int deeper = ti.side * an.pairs;
            for (int part = 0; part < ti.parts; ++part) {
                const int left = place.left(ti, st, x.heads, an.T);
                if (!TWO) __syncwarp();            // q_out may be q: a group's rows have been loaded before one is stored
                for_rows(ti, st, is_v ? 0 : left, an.T, to, [&](int u, uint16_t* row) {
                    const float2* of_token = angles + u * deeper;
                    float c[P], s[P];
                    if constexpr (TWO && HALF) {
                        take_angles<P>(of_token, unit, an.pairs, c, s);
                        Unit<LAYOUT, 8> both{v[u], w[u]};
                        both.turn(c, s);
                        v[u] = both.x, w[u] = both.y;
                    } else if constexpr (TWO) {
                        Unit<LAYOUT, 8> one{v[u], v[u]}, two{w[u], w[u]};
                        if (e0 < plan.rot_dim) {
                            take_angles<P>(of_token, unit, an.pairs, c, s);
                            one.turn(c, s);
                        }
                        if (e0 + D / 2 < plan.rot_dim) {
                            take_angles<P>(of_token, unit + D / 16, an.pairs, c, s);
                            two.turn(c, s);
                        }
                        v[u] = one.x, w[u] = two.x;
                    } else if constexpr (HOLD == kPartners) {
                        if (e0 < plan.rot_dim) {
                            take_angles<P>(of_token, (e0 < half ? e0 : e0 - half) >> 3, an.pairs, c, s);
                            const uint32_t sign = e0 < half ? 0x80008000u : 0u;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                // y1 takes the partner's product off, y2 adds it
                                const uint32_t own = v[u].two[j], other = w[u].two[j] ^ sign;
                                v[u].two[j] = pack_bf16x2(
                                    fmaf(low_value(own), c[2 * j], low_value(other) * s[2 * j]),
                                    fmaf(high_value(own), c[(2 * j + 1) % P], high_value(other) * s[(2 * j + 1) % P]));
                            }
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < P; ++j) {
                            const int e = HALF ? e0 + j : e0 + 2 * j;
                            const float2 cs = of_token[e >= plan.rot_dim ? 0 : !HALF ? e >> 1 : e < half ? e : e - half];
                            c[j] = cs.x, s[j] = cs.y;
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t own = v[u].two[j];
                            uint32_t z;
                            if constexpr (HALF) {
                                // y1 takes the partner's product off, y2 adds it
                                uint32_t other = w[u].two[j];
                                if (e0 + 2 * j < half) other ^= 0x00008000u;
                                if (e0 + 2 * j + 1 < half) other ^= 0x80000000u;
                                z = pack_bf16x2(fmaf(low_value(own), c[2 * j], low_value(other) * s[2 * j]),
                                                fmaf(high_value(own), c[(2 * j + 1) % P],
                                                     high_value(other) * s[(2 * j + 1) % P]));
                            } else {
                                const float x1 = low_value(own), x2 = high_value(own);
                                z = pack_bf16x2(first_of(x1, x2, c[j % P], s[j % P]), second_of(x1, x2, c[j % P], s[j % P]));
                            }
                            v[u].two[j] = e0 + 2 * j < plan.rot_dim ? z : own;
                        }
                    }
                    if (is_q) {
                        *reinterpret_cast<uint4*>(row) = v[u].w;
                        if (TWO) *reinterpret_cast<uint4*>(row + D / 2) = w[u].w;
                    }
                });
                if (!is_q) {
#pragma unroll
                    for (int u = 0; u < kRopeRows; ++u) {
                        if (row_of[u] >= pool_rows) {
                            if (unit == 0) raise_status(status, TGVKV_STATUS_INDEX);
                            row_of[u] = -1;
                        }
                        store_vector<D, FMT>(v[u].w, rows, scales, row_of[u], unit);
                        if (TWO) store_vector<D, FMT>(w[u].w, rows, scales, row_of[u], unit + D / 16);
                    }
                }
                from.next(ti, st);
                to.next(ti, st);
                st.next(ti);
                load(st);
            }
        }
    }
}

template <int D, int FMT, int LAYOUT, int HOLD>
cudaError_t launch_write(const CacheProblem& p, const CachePools& pool, const tgvkv_rope_plan& plan,
                         RopeWrite a, const Angles& an, uint32_t* status, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    constexpr int groups = kRopeThreads / (HOLD == kTwo ? D / 16 : D / 8);
    a.q_tiles = make_tiles(an, a.q.heads, groups, 12, sms);
    a.k_tiles = a.v_tiles = make_tiles(an, p.H_kv, groups, 12, sms);
    Tiles* tiles[3] = {&a.q_tiles, &a.k_tiles, &a.v_tiles};
    const unsigned blocks = count_blocks(tiles, an.pairs, sms, &a.table);
    const size_t smem = 2 * sizeof(float2) * a.table;
    const auto kernel = rope_write_kernel<D, FMT, LAYOUT, HOLD>;
    // Overlap with the calls before and after pays where the CTAs have one tile each (64 tokens
    // 5.6 -> 3.5 us, call after call), and costs beside long ones: sixteen prompts stored and
    // read back 282 us against 255.
    a.early = a.q_tiles.count + a.k_tiles.count + a.v_tiles.count <= (int)blocks;
    if (a.early)
        return launch_early(kernel, dim3(blocks), dim3(kRopeThreads), smem, stream, plan, a, an, p, pool, status);
    kernel<<<blocks, kRopeThreads, smem, stream>>>(plan, a, an, p, pool, status);
    return cudaGetLastError();
}

template <int D, int FMT>
cudaError_t launch_write_by_layout(const CacheProblem& p, const CachePools& pool, const tgvkv_rope_plan& plan,
                                   const RopeWrite& a, const Angles& an, uint32_t* status, cudaStream_t stream) {
    if (plan.layout == TGVKV_ROPE_HALF) {
        if (plan.rot_dim == D) return launch_write<D, FMT, TGVKV_ROPE_HALF, kTwo>(p, pool, plan, a, an, status, stream);
        return plan.rot_dim % 16 == 0
                   ? launch_write<D, FMT, TGVKV_ROPE_HALF, kPartners>(p, pool, plan, a, an, status, stream)
                   : launch_write<D, FMT, TGVKV_ROPE_HALF, kSingly>(p, pool, plan, a, an, status, stream);
    }
    return plan.rot_dim % 8 == 0
               ? launch_write<D, FMT, TGVKV_ROPE_INTERLEAVED, kTwo>(p, pool, plan, a, an, status, stream)
               : launch_write<D, FMT, TGVKV_ROPE_INTERLEAVED, kSingly>(p, pool, plan, a, an, status, stream);
}

template <int D>
cudaError_t launch_write_by_format(const CacheProblem& p, const CachePools& pool, const tgvkv_rope_plan& plan,
                                   const RopeWrite& a, const Angles& an, uint32_t* status, cudaStream_t stream) {
    switch (p.format) {
        case TGVKV_CACHE_BF16: return launch_write_by_layout<D, TGVKV_CACHE_BF16>(p, pool, plan, a, an, status, stream);
        case TGVKV_CACHE_INT8: return launch_write_by_layout<D, TGVKV_CACHE_INT8>(p, pool, plan, a, an, status, stream);
        case TGVKV_CACHE_INT4: return launch_write_by_layout<D, TGVKV_CACHE_INT4>(p, pool, plan, a, an, status, stream);
        default: return launch_write_by_layout<D, TGVKV_CACHE_FP4>(p, pool, plan, a, an, status, stream);
    }
}

// A plan's angles; its attention factor is 1 for rows that are only moved.
Angles angles_of(const tgvkv_rope_plan& plan, int mode, const int32_t* positions, long long pos_stride, int T) {
    const double x = mode == TGVKV_ROPE_MOVE ? 1.0 : plan.attention;
    return Angles{positions, pos_stride, Factor{(float)x, (float)(x - (float)x)}, plan.axes, plan.rot_dim / 2, T};
}

}  // namespace

cudaError_t launch_rope(const tgvkv_rope_plan& plan, int mode, const int32_t* positions,
                        long long pos_stride, int T, const RopeTensor& q, const RopeTensor& k,
                        cudaStream_t stream) {
    const Angles an = angles_of(plan, mode, positions, pos_stride, T);
    RopeCall a{};
    a.q = q;
    a.k = k;
    tgvkv_rope_plan used = plan;
    if (mode == TGVKV_ROPE_GRADIENT)         // turned the other way
        for (int i = 0; i < an.pairs; ++i) used.turns[i] = 0u - plan.turns[i];
    // the widest load that pairs and their partners allow (rows are 16-byte aligned)
    if (plan.layout == TGVKV_ROPE_HALF) {
        if (an.pairs % 8 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 8>(used, a, an, stream);
        if (an.pairs % 4 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 4>(used, a, an, stream);
        if (an.pairs % 2 == 0) return launch_rope_w<TGVKV_ROPE_HALF, 2>(used, a, an, stream);
        return launch_rope_w<TGVKV_ROPE_HALF, 1>(used, a, an, stream);
    }
    if (plan.rot_dim % 8 == 0) return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 8>(used, a, an, stream);
    if (plan.rot_dim % 4 == 0) return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 4>(used, a, an, stream);
    return launch_rope_w<TGVKV_ROPE_INTERLEAVED, 2>(used, a, an, stream);
}

cudaError_t launch_rope_write(const CacheProblem& p, const CachePools& pool,
                              const tgvkv_rope_plan& plan, const int32_t* positions,
                              long long pos_stride, const int32_t* slots, int T, const RopeTensor& q,
                              const uint16_t* k, const uint16_t* v, const long long (&strides)[4],
                              uint32_t* status, cudaStream_t stream) {
    const Angles an = angles_of(plan, TGVKV_ROPE_FORWARD, positions, pos_stride, T);
    RopeWrite a{};
    a.q = q;
    a.k = RopeTensor{k, strides[0], strides[1], nullptr, 0, 0, p.H_kv};
    a.v = RopeTensor{v, strides[2], strides[3], nullptr, 0, 0, p.H_kv};
    a.slots = slots;
    return p.d == 64 ? launch_write_by_format<64>(p, pool, plan, a, an, status, stream)
                     : launch_write_by_format<128>(p, pool, plan, a, an, status, stream);
}

}  // namespace tgvkv
