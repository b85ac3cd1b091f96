// The page table of a paged cache on the device (gfx950): reserving, forking, freeing and compacting.  Whole numbers only, bound by latency:
// what has to be in order -- which free page goes to whom -- is one workgroup's scan of the reference counts, 4 or 16 a thread and round;
// what has not, the tables' rows, is one workgroup per slot.
#include "sage_paged.h"

namespace sage {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Counts that a thread looks at per round: few for small pools, whose free pages are then spread over the threads, more for large ones,
// where there are to be few rounds (a round's free pages go through a list in LDS: one a thread).  Measured in a graph, us: fork of 64 slots, 220
// pages, 7.7 with 4, 14.0 with 16 and each thread on its own free pages; reserve of 248, 16661 pages, 6.9 with 16 and the list, 8.8 with
// 32 without.
constexpr int kFew = 4, kMany = 16, kSmallPool = kThreads * kFew;

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Exclusive prefix sum of x over the workgroup, and its total.  Two barriers.
__device__ __forceinline__ int scan(int x, int &total, int *shared) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int incl = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(incl, d);
        if (lane >= d) incl += y;
    }
    __syncthreads();
    if (lane == 63) shared[wave] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int s = shared[w];
        all += s;
        if (w < wave) before += s;
    }
    total = all;
    return before + incl - x;
}

// The counts of pages p0 + EACH * thread .. (behind the last page: 1, neither free nor counted as live by the callers' bounds).
template <int EACH>
__device__ __forceinline__ void load_refs(const sage_page_table &pt, int p0, int (&r)[EACH]) {
    const int p = p0 + EACH * (int)threadIdx.x;
    if (p + EACH <= pt.n_pages) {
#pragma unroll
        for (int i = 0; i < EACH / 4; ++i) {
            const int4 v = *reinterpret_cast<const int4 *>(pt.refs + p + 4 * i);
            r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) r[i] = p + i < pt.n_pages ? pt.refs[p + i] : 1;
    }
}

// Which entry of a list needs the k-th page: the last one whose first page is at or before k (entries that need none share their
// first page with the next and are passed over).
__device__ __forceinline__ int entry_of(const int *first, int n, int k) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= k) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Entry w of the row that a fork gives to dst, and the count of the page that it shares.
__device__ __forceinline__ void fork_entry(const sage_page_table &pt, int src, int dst, int own, int len, int w) {
    const int full = len / pt.page_tokens;
    int page = -1;
    if (w < full) {
        page = pt.table[(size_t)src * pt.width + w];
        if (page >= 0 && page < pt.n_pages) atomicAdd(pt.refs + page, 1);
    } else if (w == full && len % pt.page_tokens) {
        page = own;
    }
    pt.table[(size_t)dst * pt.width + w] = page;
    if (w == 0) pt.lens[dst] = len;
}

// The second half of a fork where that is more than one workgroup's work: a workgroup per entry.
__global__ __launch_bounds__(256) void fork_rows_kernel(const sage_page_table pt, const int32_t *__restrict__ page_moves,
                                                        const int32_t *__restrict__ slot_moves) {
    const int i = blockIdx.x, src = slot_moves[2 * i], dst = slot_moves[2 * i + 1];
    if (dst < 0) return;
    const int len = pt.lens[src];
    for (int w = threadIdx.x; w < pt.width; w += 256) fork_entry(pt, src, dst, page_moves[2 * i + 1], len, w);
}

// Reserve (slots, n_new) and the first half of a fork (src, dst): one workgroup.  FORK: entry i needs one page if src's last page is not
// full; its page and the moves are written here, tables and shared counts too where rows_here, or by fork_rows_kernel.
// Dynamic LDS: claim[slots] (the first entry that names a slot, of dst for forks), first[n + 1] (the pages needed before an entry), have[n]
// (the pages that its row has, -1: refused).
template <bool FORK, int EACH>
__global__ __launch_bounds__(kThreads) void assign_kernel(const sage_page_table pt, const int32_t *__restrict__ slots,
                                                         const int32_t *__restrict__ n_new, const int32_t *__restrict__ src, int n,
                                                         int32_t *__restrict__ status, int32_t *__restrict__ page_moves,
                                                         int32_t *__restrict__ slot_moves, bool rows_here) {
    constexpr int ROUND = kThreads * EACH;
    extern __shared__ int lds[];
    __shared__ int shared[kWaves];
    __shared__ uint16_t list[ROUND];  // a round's free pages, in order
    int *claim = lds, *first = lds + pt.slots, *have = first + n + 1;
    const int tid = threadIdx.x;
    int r[EACH];
    load_refs(pt, 0, r);  // (under way while the list is looked at)
    for (int i = tid; i < pt.slots; i += kThreads) claim[i] = n;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const int s = slots[i];
        if (s >= 0 && s < pt.slots) atomicMin(&claim[s], i);
    }
    __syncthreads();
    // what entry i's row has (-1: it cannot be served whatever is free) and needs
    const auto entry = [&](int i, int &need) {
        need = 0;
        const int s = slots[i];
        if (s < 0 || s >= pt.slots || claim[s] != i) return -1;
        const int32_t *row = pt.table + (size_t)s * pt.width;
        const int64_t room = (int64_t)pt.width * pt.page_tokens;
        if constexpr (FORK) {
            const int from = src[i];
            if (from < 0 || from >= pt.slots || claim[from] < n || pt.lens[s] != 0 || row[0] >= 0) return -1;
            const int len = pt.lens[from];
            if (len < 0 || len > room) return -1;
            need = len % pt.page_tokens != 0;
            return len / pt.page_tokens;
        } else {
            const int old = pt.lens[s], more = n_new ? n_new[i] : 1;
            if (old < 0 || more < 0 || old + (int64_t)more > room) return -1;
            int has = ceil_div(old, pt.page_tokens);
            while (has < pt.width && row[has] >= 0) ++has;  // (a sequence that was shortened kept its pages)
            need = max(0, ceil_div(old + more, pt.page_tokens) - has);
            return has;
        }
    };
    int wanted = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + tid;
        int need = 0, total;
        if (i < n) have[i] = entry(i, need);
        const int before = wanted + scan(need, total, shared);
        if (i < n) first[i] = before;
        wanted += total;
    }
    if (tid == 0) first[n] = wanted;
    __syncthreads();
    // the free pages in order; an entry whose pages turn out not to be all there gives them back below
    int found = 0;
    for (int p0 = 0; p0 < pt.n_pages && found < wanted; p0 += ROUND) {
        uint32_t is_free = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) is_free |= (uint32_t)(r[e] == 0) << e;
        if (p0 + ROUND < pt.n_pages) load_refs(pt, p0 + ROUND, r);  // the next round's, under way
        int total, k = scan(__popc(is_free), total, shared);
        for (; is_free; is_free &= is_free - 1) list[k++] = (uint16_t)(EACH * tid + __ffs(is_free) - 1);
        __syncthreads();
        for (k = tid; k < min(total, wanted - found); k += kThreads) {
            const int page = p0 + list[k], i = entry_of(first, n, found + k);
            pt.refs[page] = 1;
            if constexpr (FORK) page_moves[2 * i + 1] = page;
            else pt.table[(size_t)slots[i] * pt.width + have[i] + found + k - first[i]] = page;
        }
        found += total;  // (the next round's scan has the barrier that the list needs)
    }
    __syncthreads();  // (and the pages written above are seen below)
    for (int i = tid; i < n; i += kThreads) {
        const int need = first[i + 1] - first[i];
        bool ok = have[i] >= 0;
        if (ok && need && first[i + 1] > found) {
            ok = false;
            for (int w = 0; w < need && first[i] + w < found; ++w) {
                if constexpr (FORK) {
                    pt.refs[page_moves[2 * i + 1]] = 0;
                } else {
                    int32_t *t = pt.table + (size_t)slots[i] * pt.width + have[i] + w;
                    pt.refs[*t] = 0;
                    *t = -1;
                }
            }
        }
        status[i] = ok ? 0 : -1;
        if constexpr (FORK) {
            const bool part = ok && need;
            page_moves[2 * i] = part ? pt.table[(size_t)src[i] * pt.width + have[i]] : -1;
            if (!part) page_moves[2 * i + 1] = -1;
            slot_moves[2 * i] = ok ? src[i] : -1;
            slot_moves[2 * i + 1] = ok ? slots[i] : -1;
        } else if (ok) {
            pt.lens[slots[i]] += n_new ? n_new[i] : 1;  // (a slot is served once: nobody else looks at this length any more)
        }
    }
    if constexpr (FORK) {
        if (!rows_here) return;
        __syncthreads();
        for (int e = tid; e < n * pt.width; e += kThreads) {
            const int i = e / pt.width, s = slot_moves[2 * i], d = slot_moves[2 * i + 1];
            if (d >= 0) fork_entry(pt, s, d, page_moves[2 * i + 1], pt.lens[s], e - i * pt.width);
        }
    }
}

// A workgroup per listed slot.  Entries are taken out by exchange, so a slot that is listed twice gives its pages back once.
__global__ __launch_bounds__(256) void free_kernel(const sage_page_table pt, const int32_t *__restrict__ slots) {
    const int s = slots[blockIdx.x];
    if (s < 0 || s >= pt.slots) return;
    for (int w = threadIdx.x; w < pt.width; w += 256) {
        int32_t *t = pt.table + (size_t)s * pt.width + w;
        if (*t < 0) continue;
        const int page = atomicExch(t, -1);
        if (page >= 0 && page < pt.n_pages) atomicSub(pt.refs + page, 1);
    }
    if (threadIdx.x == 0) pt.lens[s] = 0;
}

// One workgroup: the live pages at and behind M = number of live pages, in order, and the free ones before M, in order: as many.  The k-th
// moves to the k-th.  remap[p] for p >= M: where page p is now.
template <int EACH>
__global__ __launch_bounds__(kThreads) void compact_kernel(const sage_page_table pt, int32_t *__restrict__ moves, int max_moves,
                                                           int32_t *__restrict__ counts, int32_t *__restrict__ remap) {
    __shared__ int shared[kWaves];
    const int tid = threadIdx.x;
    constexpr int ROUND = kThreads * EACH;
    int mine = 0, live = 0, r[EACH];
    for (int p0 = 0; p0 < pt.n_pages; p0 += ROUND) {
        load_refs(pt, p0, r);
#pragma unroll
        for (int e = 0; e < EACH; ++e) mine += r[e] > 0 && p0 + EACH * tid + e < pt.n_pages;
    }
    scan(mine, live, shared);
    int movers = 0, holes = 0;
    for (int p0 = 0; p0 < pt.n_pages; p0 += ROUND) {
        load_refs(pt, p0, r);
        int m = 0, f = 0, total;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int p = p0 + EACH * tid + e;
            m += p < pt.n_pages && p >= live && r[e] > 0;
            f += p < live && r[e] <= 0;
        }
        // (both sums in one scan: at most 2^14 of either in a round)
        const int before = scan(m << 16 | f, total, shared);
        int km = movers + (int)((uint32_t)before >> 16), kf = holes + (before & 0xffff);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int p = p0 + EACH * tid + e;
            if (p >= pt.n_pages) continue;
            if (p < live) {
                if (r[e] > 0) continue;
                if (kf < max_moves) moves[2 * kf + 1] = p;
                ++kf;
            } else {
                remap[p] = p;
                if (r[e] <= 0) continue;
                if (km < max_moves) moves[2 * km] = p;
                ++km;
            }
        }
        movers += (int)((uint32_t)total >> 16), holes += total & 0xffff;
    }
    __syncthreads();
    const int n = min(movers, max_moves);
    for (int k = tid; k < max_moves; k += kThreads) {
        if (k < n) {
            const int from = moves[2 * k], to = moves[2 * k + 1];
            remap[from] = to;
            pt.refs[to] = pt.refs[from];
            pt.refs[from] = 0;
        } else {
            moves[2 * k] = moves[2 * k + 1] = -1;
        }
    }
    if (tid == 0) counts[0] = live, counts[1] = n;
}

__global__ __launch_bounds__(256) void rename_kernel(const sage_page_table pt, const int32_t *__restrict__ counts,
                                                     const int32_t *__restrict__ remap) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)pt.slots * pt.width) return;
    const int page = pt.table[i];
    if (page >= counts[0] && page < pt.n_pages) pt.table[i] = remap[page];
}

size_t lds_bytes(const sage_page_table &pt, int n) { return ((size_t)pt.slots + 2 * (size_t)n + 1) * sizeof(int); }

}  // namespace

hipError_t launch_pages_reserve(const sage_page_table &pt, const int32_t *slots, const int32_t *n_new, int n, int32_t *status,
                                hipStream_t stream) {
    (pt.n_pages <= kSmallPool ? assign_kernel<false, kFew> : assign_kernel<false, kMany>)<<<dim3(1), dim3(kThreads), lds_bytes(pt, n), stream>>>(pt, slots, n_new, nullptr, n, status, nullptr, nullptr, false);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const sage_page_table &pt, const int32_t *src, const int32_t *dst, int n, int32_t *status, int32_t *page_moves,
                             int32_t *slot_moves, hipStream_t stream) {
    const bool rows_here = (int64_t)n * pt.width <= 8 * kThreads;  // a few rounds of one workgroup against a launch
    (pt.n_pages <= kSmallPool ? assign_kernel<true, kFew> : assign_kernel<true, kMany>)<<<dim3(1), dim3(kThreads), lds_bytes(pt, n), stream>>>(pt, dst, nullptr, src, n, status, page_moves, slot_moves, rows_here);
    if (!rows_here) fork_rows_kernel<<<dim3(n), dim3(256), 0, stream>>>(pt, page_moves, slot_moves);
    return hipGetLastError();
}

hipError_t launch_pages_free(const sage_page_table &pt, const int32_t *slots, int n, hipStream_t stream) {
    free_kernel<<<dim3(n), dim3(256), 0, stream>>>(pt, slots);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const sage_page_table &pt, int32_t *moves, int max_moves, int32_t *counts, int32_t *remap,
                                hipStream_t stream) {
    (pt.n_pages <= kSmallPool ? compact_kernel<kFew> : compact_kernel<kMany>)<<<dim3(1), dim3(kThreads), 0, stream>>>(pt, moves, max_moves, counts, remap);
    const int64_t entries = (int64_t)pt.slots * pt.width;
    rename_kernel<<<dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, stream>>>(pt, counts, remap);
    return hipGetLastError();
}

}  // namespace sage
