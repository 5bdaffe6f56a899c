// Page tables and slot maps from lengths (the page list of include/tgvkv.h).
//
//   need_s = pages set s takes (or gives back), prefix_s = need_0 + .. + need_{s-1}
//   take:  table[s][held_s + i] = free[F - 1 - (prefix_s + i)],   F -> F - K
//   give:  free[F + R - 1 - (prefix_s + i)] = table[s][keep_s + i],  F -> F + R
//   slot(t, g) = table[s][j / page] * page + j % page,  j = lens[s] + t - tok_offsets[b]
//
// A few bytes a set, an entry or a token: latency for a decode step, the slots' stores
// for long prompts.  Every CTA makes the prefix sums of all sets for itself (8 bytes a set
// from L2), so that none waits for another; the one that ends last writes n_free, which
// all have read by then.  Prefixes are kept of granules of 1, 2, 4 or 8 sets, at most
// kGranules of them (32 KB).  Entries and tokens are shared out flat, so that one long set
// is spread as well as many short ones; where sequences have few new tokens (a decode step) a
// warp does its sets' entries and slots instead, without a search (BY_SET).
//
// Measured, tokens appended and taken back, two calls in a graph (us): 64 sequences of 4 heads,
// one token each, 6.2 (flat 11.9); 256 sequences 8.5 (21.1); 1024 sequences 13.5; one of 64 with
// 256 tokens 9.3; 64 prompts of 4352 .. 8704 tokens, 1.7 million slots, 14.4.
// Followers are not let in early: with that the prompts took 41 against 25.
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

constexpr int kPageThreads = 256;
constexpr int kGranules = 8192;
constexpr int kSlotUnroll = 4;                           // slots a thread has in flight
constexpr int kSlotRun = 512;                            // slots in a row that a warp makes
constexpr int kSlotTile = kPageThreads * kSlotUnroll;    // of page_slots_kernel
constexpr int kSetBatch = 4;                             // sets a thread looks at together
constexpr int kManySets = 2048;
constexpr int kHeldOffsets = 2048;                       // sequences whose offsets a CTA holds
// BY_SET: up to this many new tokens a sequence, on average, and in all.  Appended and taken back,
// heads of 4, in a graph, by set / flat (us): a token each, 64 sequences 6.8 / 13.7, 1024 13.3 /
// 27.9, 4096 30.2 / 54.5; four each, 1024 sequences 14.1 / 24.9.  But a warp has its sequence's
// tokens to itself: all of them in one of 1024 sequences, 256 16.9 / 19.9, 1024 28.2 / 20.5, 2048
// 43.6 / 20.3, 4096 71.8 / 19.8 (which the host cannot know: the bound in all is for that).
constexpr int kFewTokens = 4, kFewInAll = 2048;

__device__ __forceinline__ int pages_of(const CacheProblem& p, int len) {
    return (int)(((long long)len + p.page - 1) >> p.page_shift);
}

// What a call says of a set: its length, and its new one, or its sequence's offsets.
struct SetInput {
    int len, lo, hi;

    // A length, and (of new tokens) offsets, that may be; first: the offsets are those of the
    // first sequence.
    __device__ __forceinline__ bool sound(const CacheProblem& p, const PagesArgs& a, bool first) const {
        return len >= 0 & len <= p.cap & lo >= 0 & hi >= lo & hi <= a.T & (!first | lo == 0);
    }
    // The lengths before and after; both 0 and false where they are nonsense.
    template <int MODE>
    __device__ __forceinline__ bool lengths(const CacheProblem& p, const PagesArgs& a, bool first, int& before,
                                            int& after) const {
        bool fine;
        if (MODE == kPagesAppend) {
            fine = sound(p, a, first) & (long long)hi - lo <= (long long)p.cap - len;
            after = fine ? len + (hi - lo) : 0;
        } else {
            fine = len >= 0 & len <= p.cap & hi >= 0 & hi <= p.cap;
            after = fine ? hi : 0;
        }
        before = fine ? len : 0;
        return fine;
    }
};
template <int MODE>
__device__ __forceinline__ SetInput set_input(const CacheProblem& p, const PagesArgs& a, int s, int b) {
    if (MODE == kPagesAppend) return SetInput{a.lens[s], a.tok_offsets[b], a.tok_offsets[b + 1]};
    return SetInput{a.lens[s], 0, a.lens_new[s]};
}

// Pages that a set of these lengths takes (gives back: MODE kPagesShrink), and the first of
// its entries that changes.
template <int MODE>
__device__ __forceinline__ int need_of(const CacheProblem& p, int len, int now) {
    const int before = pages_of(p, len), after = pages_of(p, now);
    return max(MODE == kPagesShrink ? before - after : after - before, 0);
}
template <int MODE>
__device__ __forceinline__ int set_need(const CacheProblem& p, const PagesArgs& a, int s, int& held) {
    int len, now;
    const int b = MODE == kPagesAppend ? s / p.H_kv : 0;
    set_input<MODE>(p, a, s, b).template lengths<MODE>(p, a, b == 0, len, now);
    held = pages_of(p, MODE == kPagesShrink ? now : len);
    return need_of<MODE>(p, len, now);
}

// A page number of the list or of a table, or -1 (with the status bit) where it names none.
__device__ __forceinline__ int valid_entry(const CacheProblem& p, int page, uint32_t* status) {
    if (page >= 0 && page < p.n_pages) return page;
    raise_status(status, TGVKV_STATUS_INDEX);
    return -1;
}

template <int MODE, bool BY_SET>
__global__ void __launch_bounds__(kPageThreads)
pages_kernel(const CacheProblem p, const PagesArgs a, uint32_t* __restrict__ ticket,
             uint32_t* __restrict__ status) {
    extern __shared__ int prefix[];                      // of every granule
    __shared__ int offsets[MODE == kPagesAppend && !BY_SET ? kHeldOffsets + 1 : 1];
    __shared__ int warp_sum[kPageThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int shift = a.granule_shift, size = 1 << shift, n_gran = (p.S + size - 1) >> shift;
    griddep_wait();
    const int free_now = *a.n_free;
    const bool held_offsets = MODE == kPagesAppend && !BY_SET && p.B <= kHeldOffsets;
    if (held_offsets)
        for (int b = tid; b <= p.B; b += kPageThreads) offsets[b] = a.tok_offsets[b];
    // ---- what every set needs, of granules side by side; then a thread sums a run of them (an
    // odd number: in other banks than its neighbours')
    bool bad = free_now < 0 || free_now > p.n_pages;
    for (int g0 = tid; g0 < n_gran; g0 += kSetBatch * kPageThreads) {
        int need[kSetBatch];
#pragma unroll
        for (int k = 0; k < kSetBatch; ++k) need[k] = 0;
        for (int x = 0; x < size; ++x) {
            SetInput in[kSetBatch];                      // loads in flight
#pragma unroll
            for (int k = 0; k < kSetBatch; ++k) {
                const int s = ((g0 + k * kPageThreads) << shift) + x;
                if (s < p.S) in[k] = set_input<MODE>(p, a, s, MODE == kPagesAppend ? s / p.H_kv : 0);
            }
#pragma unroll
            for (int k = 0; k < kSetBatch; ++k) {
                const int s = ((g0 + k * kPageThreads) << shift) + x;
                if (s >= p.S) continue;
                int len, now;
                bad |= !in[k].template lengths<MODE>(p, a, MODE == kPagesAppend && s < p.H_kv, len, now);
                need[k] += need_of<MODE>(p, len, now);
            }
        }
#pragma unroll
        for (int k = 0; k < kSetBatch; ++k)
            if (g0 + k * kPageThreads < n_gran) prefix[g0 + k * kPageThreads] = need[k];
    }
    __syncthreads();
    const int run = ((n_gran + kPageThreads - 1) / kPageThreads) | 1, g0 = min(tid * run, n_gran);
    const int g1 = min(g0 + run, n_gran);
    int sum = 0;
    for (int g = g0; g < g1; ++g) sum += prefix[g];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int base = incl - sum, carry = 0;
#pragma unroll
    for (int w = 0; w < kPageThreads / 32; ++w) {
        if (w < warp) base += warp_sum[w];
        carry += warp_sum[w];
    }
    for (int g = g0; g < g1; ++g) {
        const int need = prefix[g];
        prefix[g] = base;
        base += need;
    }
    bad = __syncthreads_or(bad);
    const int total = carry;
    const bool room = MODE == kPagesShrink ? total <= p.n_pages - free_now : total <= free_now;
    const bool go = !bad && room;
    if (!go && blockIdx.x == 0 && tid == 0)
        raise_status(status, bad || MODE == kPagesShrink ? TGVKV_STATUS_INDEX : TGVKV_STATUS_PAGES);
    const int threads = gridDim.x * kPageThreads, thread = blockIdx.x * kPageThreads + tid;
    // the page that the list's i-th taking gets
    const auto taken = [&](int i) { return a.free_pages[free_now - 1 - i]; };
    // pages taken by the sets before s
    const auto before = [&](int s) {
        int i = prefix[s >> shift], h;
        for (int e = s >> shift << shift; e < s; ++e) i += set_need<MODE>(p, a, e, h);
        return i;
    };

    if constexpr (BY_SET) {
        for (int s0 = thread - lane; s0 < p.S; s0 += threads) {          // 32 sets a warp
            const int s = s0 + lane, b = min(s, p.S - 1) / p.H_kv, g = s - b * p.H_kv;
            const int lo = a.tok_offsets[b], n = s < p.S ? a.tok_offsets[b + 1] - lo : 0;
            const int len = s < p.S ? a.lens[s] : 0;
            if (s < p.S) a.lens_out[s] = go ? len + n : len;
            if (!go) continue;
            const int held = pages_of(p, len), i0 = s < p.S ? before(s) - held : 0;
            // the i-th new token of set x: its page, entered with the page's first token
            const auto place = [&](int x, int xlen, int xheld, int xi0, int i, int t, int head) {
                const int j = xlen + i, at = j >> p.page_shift;
                int32_t* entry = a.table + (size_t)x * p.max_pages + at;
                const int page = valid_entry(p, at < xheld ? *entry : taken(xi0 + at), status);
                if (at >= xheld && (i == 0 || (j & (p.page - 1)) == 0)) *entry = page;
                if (a.slots) a.slots[(size_t)t * p.H_kv + head] = page < 0 ? -1 : page * p.page + (j & (p.page - 1));
            };
            if (n <= kFewTokens)
                for (int i = 0; i < n; ++i) place(s, len, held, i0, i, lo + i, g);
            // sets of more tokens, by all lanes
            for (uint32_t many = __ballot_sync(~0u, n > kFewTokens); many; many &= many - 1) {
                const int from = __ffs(many) - 1;
                const int xn = __shfl_sync(~0u, n, from), xlen = __shfl_sync(~0u, len, from);
                const int xheld = __shfl_sync(~0u, held, from), xi0 = __shfl_sync(~0u, i0, from);
                const int xlo = __shfl_sync(~0u, lo, from), xg = __shfl_sync(~0u, g, from);
#pragma unroll 4
                for (int i = lane; i < xn; i += 32) place(s0 + from, xlen, xheld, xi0, i, xlo + i, xg);
            }
        }
        if (a.slots)                                     // tokens that are no sequence's, or all
            for (long long u = (long long)(go ? a.tok_offsets[p.B] : 0) * p.H_kv + thread;
                 u < (long long)a.T * p.H_kv; u += threads)
                a.slots[u] = -1;
    } else {
        // ---- the entries that change
        for (int i = thread; go && i < total; i += threads) {
            const int g = find_last(prefix, 0, n_gran - 1, i);
            int s = g << shift, at = i - prefix[g], held, need;
            while ((need = set_need<MODE>(p, a, s, held)) <= at) at -= need, ++s;
            int32_t* entry = a.table + (size_t)s * p.max_pages + held + at;
            if (MODE == kPagesShrink) {
                a.free_pages[free_now + total - 1 - i] = valid_entry(p, *entry, status);
                *entry = -1;
            } else {
                *entry = valid_entry(p, taken(i), status);
            }
        }
    }
    if constexpr (MODE == kPagesAppend && !BY_SET) {
        for (int s = thread; s < p.S; s += threads) {
            const int b = s / p.H_kv, len = a.lens[s];
            a.lens_out[s] = go ? len + a.tok_offsets[b + 1] - a.tok_offsets[b] : len;
        }
        // ---- the tokens' slots: a warp takes kSlotRun in a row, which have few sequences
        const unsigned n_slots = a.slots ? (unsigned)a.T * p.H_kv : 0u, H = p.H_kv;
        const int end = go ? a.tok_offsets[p.B] : 0;
        const int32_t* off = held_offsets ? offsets : a.tok_offsets;
        for (unsigned u0 = (thread >> 5) * kSlotRun; u0 < n_slots; u0 += (threads >> 5) * kSlotRun) {
            unsigned t = (u0 + lane) / H, g = u0 + lane - t * H;
            const unsigned dt = 32u / H, dg = 32u - dt * H;
            int b = (int)t < end ? find_last(off, 0, p.B - 1, t) : 0;
#pragma unroll 2
            for (unsigned u = u0 + lane; u < min(u0 + kSlotRun, n_slots); u += 32 * kSlotUnroll) {
                int page[kSlotUnroll], in_page[kSlotUnroll];
#pragma unroll
                for (int x = 0; x < kSlotUnroll; ++x) {
                    page[x] = -1;
                    in_page[x] = 0;
                    if ((int)t < end && u + 32 * x < n_slots) {
                        while ((int)t >= off[b + 1]) ++b;
                        const int s = b * H + g, len = a.lens[s], j = len + (int)t - off[b];
                        const int at = j >> p.page_shift, held = pages_of(p, len);
                        in_page[x] = j & (p.page - 1);
                        page[x] = at >= held ? taken(before(s) + at - held) : a.table[(size_t)s * p.max_pages + at];
                        if (page[x] < 0 || page[x] >= p.n_pages) page[x] = -2;
                    }
                    t += dt, g += dg;
                    if (g >= H) g -= H, ++t;
                }
#pragma unroll
                for (int x = 0; x < kSlotUnroll; ++x) {
                    if (u + 32 * x >= n_slots) break;
                    if (page[x] == -2) raise_status(status, TGVKV_STATUS_INDEX);
                    a.slots[u + 32 * x] = page[x] < 0 ? -1 : page[x] * p.page + in_page[x];
                }
            }
        }
    }
    // ---- the list's size, by the CTA that ends last
    if (gridDim.x > 1) __syncthreads();
    if (tid == 0) {
        if (gridDim.x > 1) {
            __threadfence();
            const uint32_t t = atomicAdd(ticket, 1u);
            if (t >= gridDim.x) raise_status(status, TGVKV_STATUS_TIMEOUT);   // not at zero
            if (t != gridDim.x - 1) return;
            *ticket = 0u;
        }
        if (go) *a.n_free = MODE == kPagesShrink ? free_now + total : free_now - total;
    }
}

// The slots of sets that hold their pages.
__global__ void __launch_bounds__(kPageThreads)
page_slots_kernel(const CacheProblem p, const PagesArgs a, uint32_t* __restrict__ status) {
    __shared__ int span[2];
    const int tid = threadIdx.x;
    griddep_wait();
    if (blockIdx.x == 0)
        for (int s = tid; s < p.S; s += kPageThreads) {
            int len, now;
            if (!set_input<kPagesAppend>(p, a, s, s / p.H_kv).lengths<kPagesAppend>(p, a, s < p.H_kv, len, now))
                raise_status(status, TGVKV_STATUS_INDEX);
        }
    const unsigned n_slots = (unsigned)a.T * p.H_kv, u0 = blockIdx.x * kSlotTile;
    if (u0 >= n_slots) return;
    const unsigned u1 = min(u0 + kSlotTile, n_slots) - 1;
    find_span(a.tok_offsets, p.B - 1, u0 / (unsigned)p.H_kv, u1 / (unsigned)p.H_kv, span);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kSlotUnroll; ++x) {
        const unsigned u = u0 + x * kPageThreads + tid;
        if (u > u1) break;
        int slot = -1;
        const int t = (int)(u / (unsigned)p.H_kv);
        if (t >= a.tok_offsets[0] && t < a.tok_offsets[p.B]) {
            const int b = find_last(a.tok_offsets, span[0], span[1], t);
            const int s = b * p.H_kv + (int)(u - (unsigned)t * p.H_kv);
            const SetInput in = set_input<kPagesAppend>(p, a, s, b);
            // (nonsense is reported by the first CTA; a set that would outgrow its row has the slots in it)
            if (in.sound(p, a, b == 0) && t >= in.lo && t < in.hi)
                slot = pool_row(p, a.table, s, (long long)in.len + t - in.lo, status);
        }
        a.slots[u] = slot;
    }
}

__global__ void __launch_bounds__(kPageThreads)
pages_init_kernel(const CacheProblem p, const PagesArgs a) {
    const long long entries = (long long)p.S * p.max_pages;
    const long long step = (long long)gridDim.x * kPageThreads;
    const long long i0 = (long long)blockIdx.x * kPageThreads + threadIdx.x;
    griddep_wait();
    for (long long i = i0; i < entries; i += step) a.table[i] = -1;
    for (long long i = i0; i < p.n_pages; i += step) a.free_pages[i] = p.n_pages - 1 - (int)i;
    if (i0 == 0) *a.n_free = p.n_pages;
}

// `work`: entries or slots, of which a thread does `each`.
template <int MODE, bool BY_SET>
cudaError_t launch_mode(const CacheProblem& p, PagesArgs a, long long work, int each, uint32_t* ticket,
                        uint32_t* status, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    a.granule_shift = 0;
    while ((p.S - 1) >> a.granule_shift >= kGranules) ++a.granule_shift;
    const int granules = ((p.S - 1) >> a.granule_shift) + 1, tile = kPageThreads * each;
    // every CTA reads all lengths: one an SM where that is more than its share of the work (a
    // token each appended and taken back, one and four an SM, us: 4096 sets 13.5 / 15.1, 32768
    // sets 97 / 111)
    const int most = p.S > kManySets ? sms : 4 * sms;
    const long long blocks = std::min<long long>(std::max<long long>((work + tile - 1) / tile, 1), most);
    return launch_early(pages_kernel<MODE, BY_SET>, dim3((unsigned)blocks), dim3(kPageThreads),
                        sizeof(int) * granules, stream, p, a, ticket, status);
}

}  // namespace

cudaError_t launch_pages(const CacheProblem& p, int mode, const PagesArgs& a, uint32_t* ticket,
                         uint32_t* status, cudaStream_t stream) {
    const long long entries = (long long)p.S * p.max_pages, slots = (long long)a.T * p.H_kv;
    if (mode == kPagesGrow) return launch_mode<kPagesGrow, false>(p, a, entries, 1, ticket, status, stream);
    if (mode == kPagesShrink) return launch_mode<kPagesShrink, false>(p, a, entries, 1, ticket, status, stream);
    if (a.T <= (long long)kFewTokens * p.B && a.T <= kFewInAll)
        return launch_mode<kPagesAppend, true>(p, a, p.S, 1, ticket, status, stream);
    return launch_mode<kPagesAppend, false>(p, a, std::max<long long>(slots, p.S), kSlotRun / 32, ticket, status, stream);
}

cudaError_t launch_page_slots(const CacheProblem& p, const PagesArgs& a, uint32_t* status,
                              cudaStream_t stream) {
    const long long n = (long long)a.T * p.H_kv;
    const unsigned blocks = (unsigned)std::max<long long>((n + kSlotTile - 1) / kSlotTile, 1);
    return launch_early(page_slots_kernel, dim3(blocks), dim3(kPageThreads), 0, stream, p, a, status);
}

cudaError_t launch_pages_init(const CacheProblem& p, const PagesArgs& a, cudaStream_t stream) {
    const long long work = std::max<long long>((long long)p.S * p.max_pages, p.n_pages);
    const unsigned blocks = (unsigned)std::min<long long>((work + 1023) / 1024, 4096);
    return launch_early(pages_init_kernel, dim3(blocks), dim3(kPageThreads), 0, stream, p, a);
}

}  // namespace tgvkv
