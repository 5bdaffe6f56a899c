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
// thread does all of its sets instead, without a search (BY_SET).
// Followers are not let in early: with that, two calls for 64 prompts took 41 us against 25.
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

constexpr int kPageThreads = 256;
constexpr int kGranules = 8192;
constexpr int kSlotUnroll = 4;                           // slots a thread has in flight
constexpr int kSlotRun = 512;                            // slots in a row that a warp makes
constexpr int kSlotTile = kPageThreads * kSlotUnroll;    // of page_slots_kernel
constexpr int kHeldOffsets = 2048;                       // sequences whose offsets a CTA holds
constexpr int kFewTokens = 4;                            // new tokens a sequence, on average, up to which BY_SET

__device__ __forceinline__ int pages_of(const CacheProblem& p, int len) {
    return (int)(((long long)len + p.page - 1) >> p.page_shift);
}

// Set s: its length before and after; false where the call's input says nonsense.
template <int MODE>
__device__ __forceinline__ bool set_lengths(const CacheProblem& p, const PagesArgs& a, int s, int& len,
                                            int& now) {
    len = now = a.lens[s];
    if (len < 0 || len > p.cap) return false;
    if (MODE == kPagesAppend) {
        const int b = s / p.H_kv, lo = a.tok_offsets[b], hi = a.tok_offsets[b + 1];
        if (lo < 0 || hi < lo || hi > a.T || (b == 0 && lo != 0) || hi - lo > p.cap - len) return false;
        now = len + (hi - lo);
        return true;
    }
    now = a.lens_new[s];
    return now >= 0 && now <= p.cap;
}

// Pages that set s takes (give back: MODE kPagesShrink), of valid input.
template <int MODE>
__device__ __forceinline__ int set_need(const CacheProblem& p, const PagesArgs& a, int s, int& held) {
    int len, now;
    if (!set_lengths<MODE>(p, a, s, len, now)) {
        held = 0;
        return 0;
    }
    const int before = pages_of(p, len), after = pages_of(p, now);
    held = MODE == kPagesShrink ? after : before;        // the first entry that changes
    return max(MODE == kPagesShrink ? before - after : after - before, 0);
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
    // ---- what every set needs
    int carry = 0;
    bool bad = free_now < 0 || free_now > p.n_pages;
    for (int g0 = 0; g0 < n_gran; g0 += kPageThreads) {
        const int g = g0 + tid;
        int sum = 0;
        if (g < n_gran)
            for (int s = g << shift; s < min((g + 1) << shift, p.S); ++s) {
                int len, now, held;
                bad |= !set_lengths<MODE>(p, a, s, len, now);
                sum += set_need<MODE>(p, a, s, held);
            }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int base = carry;
#pragma unroll
        for (int w = 0; w < kPageThreads / 32; ++w) {
            if (w < warp) base += warp_sum[w];
            carry += warp_sum[w];
        }
        if (g < n_gran) prefix[g] = base + incl - sum;
        if (g0 + kPageThreads < n_gran) __syncthreads();
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
        for (int s = thread; s < p.S; s += threads) {
            const int b = s / p.H_kv, g = s - b * p.H_kv;
            const int len = a.lens[s], lo = a.tok_offsets[b], hi = a.tok_offsets[b + 1];
            a.lens_out[s] = go ? len + hi - lo : len;
            if (!go) continue;
            int32_t* entries = a.table + (size_t)s * p.max_pages;
            const int held = pages_of(p, len), i0 = before(s) - held;
            int at = -1, page = -1;                      // the page of the token before
            for (int t = lo; t < hi; ++t) {
                const int j = len + t - lo;
                if (j >> p.page_shift != at) {
                    at = j >> p.page_shift;
                    page = at < held ? entries[at] : taken(i0 + at);
                    page = valid_entry(p, page, status);
                    if (at >= held) entries[at] = page;
                }
                if (a.slots) a.slots[(size_t)t * p.H_kv + g] = page < 0 ? -1 : page * p.page + (j & (p.page - 1));
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
            int len, now;
            set_lengths<MODE>(p, a, s, len, now);
            a.lens_out[s] = go ? now : a.lens[s];
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
            if (!set_lengths<kPagesAppend>(p, a, s, len, now)) raise_status(status, TGVKV_STATUS_INDEX);
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
            const long long j = (long long)clamp_len(a.lens[s], p.cap) + t - a.tok_offsets[b];
            slot = pool_row(p, a.table, s, j, status);
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
    const long long blocks = std::min<long long>(std::max<long long>((work + tile - 1) / tile, 1), 4 * sms);
    return launch_early(pages_kernel<MODE, BY_SET>, dim3((unsigned)blocks), dim3(kPageThreads),
                        sizeof(int) * granules, stream, p, a, ticket, status);
}

}  // namespace

cudaError_t launch_pages(const CacheProblem& p, int mode, const PagesArgs& a, uint32_t* ticket,
                         uint32_t* status, cudaStream_t stream) {
    const long long entries = (long long)p.S * p.max_pages, slots = (long long)a.T * p.H_kv;
    if (mode == kPagesGrow) return launch_mode<kPagesGrow, false>(p, a, entries, 1, ticket, status, stream);
    if (mode == kPagesShrink) return launch_mode<kPagesShrink, false>(p, a, entries, 1, ticket, status, stream);
    if (a.T <= (long long)kFewTokens * p.B)
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
