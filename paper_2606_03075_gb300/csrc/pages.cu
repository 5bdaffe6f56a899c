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
// kGranules of them (32 KB); entries and tokens are shared out flat, so that one long set
// is spread as well as many short ones.
#include "cache_launch.h"
#include "launch.h"

namespace tgvkv {
namespace {

constexpr int kPageThreads = 256;
constexpr int kGranules = 8192;
constexpr int kSlotUnroll = 4;
constexpr int kSlotTile = kPageThreads * kSlotUnroll;    // slots a CTA makes at a time

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

template <int MODE>
__global__ void __launch_bounds__(kPageThreads)
pages_kernel(const CacheProblem p, const PagesArgs a, uint32_t* __restrict__ ticket,
             uint32_t* __restrict__ status) {
    extern __shared__ int prefix[];                      // of every granule, then the total
    __shared__ int warp_sum[kPageThreads / 32];
    __shared__ int span[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int size = a.granule, n_gran = (p.S + size - 1) / size;
    const int free_now = *a.n_free;
    // ---- what every set needs
    int carry = 0;
    bool bad = free_now < 0 || free_now > p.n_pages;
    for (int g0 = 0; g0 < n_gran; g0 += kPageThreads) {
        const int g = g0 + tid;
        int sum = 0;
        if (g < n_gran)
            for (int s = g * size; s < min((g + 1) * size, p.S); ++s) {
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
        __syncthreads();
    }
    bad = __syncthreads_or(bad);
    const int total = carry;
    const bool room = MODE == kPagesShrink ? total <= p.n_pages - free_now : total <= free_now;
    const bool go = !bad && room;
    if (!go && blockIdx.x == 0 && tid == 0)
        raise_status(status, bad || MODE == kPagesShrink ? TGVKV_STATUS_INDEX : TGVKV_STATUS_PAGES);

    // ---- the entries that change
    if (go) {
        for (int i = blockIdx.x * kPageThreads + tid; i < total; i += gridDim.x * kPageThreads) {
            const int g = find_last(prefix, 0, n_gran - 1, i);
            int s = g * size, at = i - prefix[g], held, need;
            while ((need = set_need<MODE>(p, a, s, held)) <= at) at -= need, ++s;
            int32_t* entry = a.table + (size_t)s * p.max_pages + held + at;
            int page;
            if (MODE == kPagesShrink) {
                page = *entry;
                *entry = -1;
            } else {
                page = a.free_pages[free_now - 1 - i];
            }
            if (page < 0 || page >= p.n_pages) {
                raise_status(status, TGVKV_STATUS_INDEX);
                page = -1;
            }
            if (MODE == kPagesShrink) a.free_pages[free_now + total - 1 - i] = page;
            else *entry = page;
        }
    }
    if (MODE == kPagesAppend) {
        for (int s = blockIdx.x * kPageThreads + tid; s < p.S; s += gridDim.x * kPageThreads) {
            int len, now;
            set_lengths<MODE>(p, a, s, len, now);
            a.lens_out[s] = go ? now : a.lens[s];
        }
        // ---- the tokens' slots
        const unsigned n_slots = a.slots ? (unsigned)a.T * p.H_kv : 0u;
        for (unsigned u0 = blockIdx.x * kSlotTile; u0 < n_slots; u0 += gridDim.x * kSlotTile) {
            const unsigned u1 = min(u0 + kSlotTile, n_slots) - 1;
            __syncthreads();
            if (go) find_span(a.tok_offsets, p.B - 1, u0 / (unsigned)p.H_kv, u1 / (unsigned)p.H_kv, span);
            __syncthreads();
#pragma unroll
            for (int x = 0; x < kSlotUnroll; ++x) {
                const unsigned u = u0 + x * kPageThreads + tid;
                if (u > u1) break;
                int slot = -1;
                const int t = (int)(u / (unsigned)p.H_kv);
                if (go && t < a.tok_offsets[p.B]) {
                    const int b = find_last(a.tok_offsets, span[0], span[1], t);
                    const int s = b * p.H_kv + (int)(u - (unsigned)t * p.H_kv);
                    const int len = a.lens[s], j = len + t - a.tok_offsets[b];
                    const int at = j >> p.page_shift, held = pages_of(p, len);
                    int page;
                    if (at >= held) {                    // a page taken just now
                        int i = prefix[s / size] + at - held, h;
                        for (int e = s / size * size; e < s; ++e) i += set_need<MODE>(p, a, e, h);
                        page = a.free_pages[free_now - 1 - i];
                    } else {
                        page = a.table[(size_t)s * p.max_pages + at];
                    }
                    if (page >= 0 && page < p.n_pages) slot = page * p.page + (j & (p.page - 1));
                    else raise_status(status, TGVKV_STATUS_INDEX);
                }
                a.slots[u] = slot;
            }
        }
    }
    // ---- the list's size, by the CTA that ends last
    __syncthreads();
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
    for (long long i = i0; i < entries; i += step) a.table[i] = -1;
    for (long long i = i0; i < p.n_pages; i += step) a.free_pages[i] = p.n_pages - 1 - (int)i;
    if (i0 == 0) *a.n_free = p.n_pages;
}

template <int MODE>
cudaError_t launch_mode(const CacheProblem& p, PagesArgs a, long long work, uint32_t* ticket,
                        uint32_t* status, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    a.granule = 1;
    while ((p.S + a.granule - 1) / a.granule > kGranules) a.granule *= 2;
    const int granules = (p.S + a.granule - 1) / a.granule;
    const long long blocks = std::min<long long>(std::max<long long>((work + kSlotTile - 1) / kSlotTile, 1), 2 * sms);
    pages_kernel<MODE><<<(unsigned)blocks, kPageThreads, sizeof(int) * granules, stream>>>(p, a, ticket, status);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pages(const CacheProblem& p, int mode, const PagesArgs& a, uint32_t* ticket,
                         uint32_t* status, cudaStream_t stream) {
    const long long entries = (long long)p.S * p.max_pages;
    if (mode == kPagesGrow) return launch_mode<kPagesGrow>(p, a, entries, ticket, status, stream);
    if (mode == kPagesShrink) return launch_mode<kPagesShrink>(p, a, entries, ticket, status, stream);
    // an entry for every `page` tokens and set at most, and one
    return launch_mode<kPagesAppend>(p, a, std::max<long long>((long long)a.T * p.H_kv, p.S), ticket, status,
                                     stream);
}

cudaError_t launch_page_slots(const CacheProblem& p, const PagesArgs& a, uint32_t* status,
                              cudaStream_t stream) {
    const long long n = (long long)a.T * p.H_kv;
    const unsigned blocks = (unsigned)std::max<long long>((n + kSlotTile - 1) / kSlotTile, 1);
    page_slots_kernel<<<blocks, kPageThreads, 0, stream>>>(p, a, status);
    return cudaGetLastError();
}

cudaError_t launch_pages_init(const CacheProblem& p, const PagesArgs& a, cudaStream_t stream) {
    const long long work = std::max<long long>((long long)p.S * p.max_pages, p.n_pages);
    const unsigned blocks = (unsigned)std::min<long long>((work + 1023) / 1024, 4096);
    pages_init_kernel<<<blocks, kPageThreads, 0, stream>>>(p, a);
    return cudaGetLastError();
}

}  // namespace tgvkv
