// Page tables of the 8-bit cache: growing, forking, freeing, compacting, on the device and in a fixed order.
//
// All of it is integer bookkeeping over refs [n_pages], a few requests and table rows: one workgroup of 16 wavefronts, so that
// "the lowest free page first, in the order of the list" needs no hand-over between workgroups.  Requests become ranges of
// ranks by a prefix sum of what they need; a free page's rank is the number of free pages in front of it (each wavefront
// counts its own stretch of refs, then ranks it with ballots), and the request that gets a page is found by bisection of the
// prefix sums.  Bound by latency: refs is read twice (once where no page is needed), 256 KiB of it for
// 65536 pages.
#include "hgf_kv8.h"

#include <limits.h>

namespace hgf {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

struct Pages {
    int n_pages, n_seqs, max_pages, page_log2;
    int32_t *table, *lens, *refs;

    __device__ int len(int s) const { return min(max(lens[s], 0), max_pages << page_log2); }
    __device__ int pages_for(int len) const { return (len + (1 << page_log2) - 1) >> page_log2; }
};

Pages pages_of(const hgf_kv8_pages &p)
{
    return {p.n_pages, p.n_seqs, p.max_pages, __builtin_ctz((unsigned)p.page), p.table, p.lens, p.refs};
}

// The stretch of pages that a wavefront counts and ranks, in steps of 256 (four to a lane).
__device__ inline void stretch_of(int n_pages, int w, int &from, int &to)
{
    const int each = ((n_pages + kWaves - 1) / kWaves + 255) & ~255;
    from = min(w * each, n_pages);
    to = min(from + each, n_pages);
}
// refs of the lane's four pages from `at` on (at: a multiple of four); behind the end `none`.
__device__ inline v4i four_refs(const int32_t *refs, int at, int to, int none)
{
    if (at + 4 <= to) return *reinterpret_cast<const v4i *>(refs + at);
    v4i r = {none, none, none, none};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + j < to) r[j] = refs[at + j];
    return r;
}
__device__ inline int lanes_below(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}
// Pages of [from, to) for which `is` holds, in all lanes.
template <class Is>
__device__ inline int count_pages(const int32_t *refs, int from, int to, int none, Is is)
{
    const int l = threadIdx.x & 63;
    int c = 0;
#pragma unroll 4
    for (int at = from + 4 * l; at < to; at += 256) {
        const v4i r = four_refs(refs, at, to, none);
#pragma unroll
        for (int j = 0; j < 4; ++j) c += is(at + j, r[j]) ? 1 : 0;
    }
    return wave_sum(c);
}
// Calls f(page, ref, rank) for the pages of [from, to) for which `is` holds, ranks rising from `rank`.
template <class Is, class F>
__device__ inline void rank_pages(const int32_t *refs, int from, int to, int none, int rank, Is is, F f)
{
    const int l = threadIdx.x & 63;
    for (int base = from; base < to; base += 256) {
        const int at = base + 4 * l;
        const v4i r = four_refs(refs, at, to, none);
        bool hit[4];
        int below = 0, all = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            hit[j] = is(at + j, r[j]);
            const unsigned long long m = __ballot(hit[j]);
            below += lanes_below(m);
            all += (int)__popcll(m);
        }
        int mine = rank + below;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (hit[j]) f(at + j, r[j], mine++);
        rank += all;
    }
}
// Sum of the counts of the wavefronts in front of this one, and of all; `box` [kWaves] in LDS.
__device__ inline void sum_waves(int *box, int c, int &before, int &all)
{
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) box[w] = c;
    __syncthreads();
    before = all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const int x = box[i];
        before += i < w ? x : 0;
        all += x;
    }
}
// Exclusive prefix sum over the workgroup's threads.
__device__ inline int scan_threads(int *box, int v, int &all)
{
    const int l = threadIdx.x & 63;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (l >= o) x += y;
    }
    int before;
    sum_waves(box, __shfl(x, 63, 64), before, all);
    return before + x - v;
}
// Marks in first[] (LDS, n_seqs) where the list names each sequence first.
__device__ inline void mark_first(int *first, int n_seqs, const int32_t *list, int n)
{
    for (int i = threadIdx.x; i < n_seqs; i += kThreads) first[i] = INT_MAX;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads)
        if ((unsigned)list[i] < (unsigned)n_seqs) atomicMin(&first[list[i]], i);
    __syncthreads();
}

struct Request {
    int need;           // fresh pages; 0 where the request is refused
    bool valid;
};

// The common part of grow and fork: request i (need(i)) gets the free pages of ranks upto[i-1] .. upto[i]-1, if there are
// that many; take(i, k, page) for its k-th page.  Returns the number of free pages; upto [n] stays in LDS.
template <class Need, class Take>
__device__ inline int hand_out(const Pages &p, int *upto, int *box, int n, Need need, Take take)
{
    int total = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + threadIdx.x;
        const int v = i < n ? need(i).need : 0;
        int all;
        const int before = scan_threads(box, v, all);
        // (sums beyond the pages that exist are all the same: too many)
        if (i < n) upto[i] = min(total + before + v, p.n_pages + 1);
        total = min(total + all, p.n_pages + 1);
    }
    const bool any = total > 0;
    if (!any) {
        __syncthreads();
        return 0;
    }
    int from, to, before, n_free;
    stretch_of(p.n_pages, threadIdx.x >> 6, from, to);
    auto is_free = [](int, int ref) { return ref <= 0; };
    const int mine = count_pages(p.refs, from, to, 1, is_free);
    sum_waves(box, mine, before, n_free);
    // what is granted: everything up to the first request that the free pages do not reach
    int lo = 0, hi = n;                             // first i with upto[i] > n_free
    while (lo < hi) {
        const int m = (lo + hi) >> 1;
        if (upto[m] > n_free) hi = m;
        else lo = m + 1;
    }
    const int granted = lo > 0 ? upto[lo - 1] : 0;
    if (before < granted) {
        rank_pages(p.refs, from, to, 1, before, is_free, [&](int page, int, int rank) {
            if (rank >= granted) return;
            int a = 0, b = n - 1;                   // first i with upto[i] > rank
            while (a < b) {
                const int m = (a + b) >> 1;
                if (upto[m] > rank) b = m;
                else a = m + 1;
            }
            p.refs[page] = 1;
            take(a, rank - (a > 0 ? upto[a - 1] : 0), page);
        });
    }
    __syncthreads();
    return n_free;
}

__global__ __launch_bounds__(kThreads) void pages_grow_kernel(Pages p, const int32_t *seqs, const int32_t *add, int n, int32_t *ok)
{
    extern __shared__ int lds[];
    __shared__ int box[kWaves];
    int *first = lds, *upto = lds + p.n_seqs;
    mark_first(first, p.n_seqs, seqs, n);
    auto need = [&](int i) -> Request {
        const int s = seqs[i];
        if ((unsigned)s >= (unsigned)p.n_seqs || first[s] != i) return {0, false};
        const int len = p.len(s), more = add[i];
        if (more < 0 || more > (p.max_pages << p.page_log2) - len) return {0, false};
        return {p.pages_for(len + more) - p.pages_for(len), true};
    };
    const int n_free = hand_out(p, upto, box, n, need, [&](int i, int k, int page) {
        const int s = seqs[i];
        p.table[(size_t)s * p.max_pages + p.pages_for(p.len(s)) + k] = page;
    });
    for (int i = threadIdx.x; i < n; i += kThreads) {               // (each sequence belongs to one thread by now)
        const Request r = need(i);
        const bool yes = r.valid && (r.need == 0 || upto[i] <= n_free);
        ok[i] = yes ? 1 : 0;
        if (yes) p.lens[seqs[i]] = p.len(seqs[i]) + add[i];
    }
}

__global__ __launch_bounds__(kThreads) void pages_fork_kernel(Pages p, const int32_t *src, const int32_t *dst, int n, int32_t *pairs,
                                                               int32_t *ok)
{
    extern __shared__ int lds[];
    __shared__ int box[kWaves];
    int *first = lds, *upto = lds + p.n_seqs;
    mark_first(first, p.n_seqs, dst, n);
    const int in_page = (1 << p.page_log2) - 1;
    auto need = [&](int i) -> Request {
        const int s = src[i], d = dst[i];
        if ((unsigned)s >= (unsigned)p.n_seqs || (unsigned)d >= (unsigned)p.n_seqs || s == d || first[d] != i) return {0, false};
        if (p.lens[d] != 0) return {0, false};
        return {(p.len(s) & in_page) != 0 ? 1 : 0, true};
    };
    for (int i = threadIdx.x; i < n; i += kThreads) pairs[2 * i] = pairs[2 * i + 1] = -1;
    const int n_free = hand_out(p, upto, box, n, need, [&](int i, int, int page) {
        const int last = p.len(src[i]) >> p.page_log2;
        p.table[(size_t)dst[i] * p.max_pages + last] = page;
        pairs[2 * i] = p.table[(size_t)src[i] * p.max_pages + last];
        pairs[2 * i + 1] = page;
    });
    // full pages, a wavefront to a request; upto[] turns into the new lengths, which are written when every length has
    // been read
    const int l = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < n; i += kWaves) {
        const Request r = need(i);
        const bool yes = r.valid && (r.need == 0 || upto[i] <= n_free);
        const int len = yes ? p.len(src[i]) : 0, full = len >> p.page_log2;
        if (yes) {
            const int32_t *from = p.table + (size_t)src[i] * p.max_pages;
            int32_t *to = p.table + (size_t)dst[i] * p.max_pages;
            for (int j = l; j < full; j += 64) {
                const int page = from[j];
                to[j] = page;
                if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(&p.refs[page], 1);
            }
        }
        if (l == 0) {
            ok[i] = yes ? 1 : 0;
            upto[i] = len;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (upto[i] > 0) p.lens[dst[i]] = upto[i];
}

__global__ __launch_bounds__(kThreads) void pages_free_kernel(Pages p, const int32_t *seqs, int n)
{
    extern __shared__ int lds[];
    mark_first(lds, p.n_seqs, seqs, n);
    const int l = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < n; i += kWaves) {
        const int s = seqs[i];
        if ((unsigned)s >= (unsigned)p.n_seqs || lds[s] != i) continue;
        const int used = p.pages_for(p.len(s));
        int32_t *row = p.table + (size_t)s * p.max_pages;
        for (int j = l; j < used; j += 64) {
            const int page = row[j];
            if ((unsigned)page < (unsigned)p.n_pages) atomicSub(&p.refs[page], 1);
            row[j] = -1;
        }
        if (l == 0) p.lens[s] = 0;                  // (this wavefront has read it)
    }
}

__global__ __launch_bounds__(kThreads) void pages_compact_kernel(Pages p, int32_t *pairs, int32_t *count, int32_t *moved)
{
    __shared__ int box[kWaves];
    int from, to, live_before, live, holes_before, holes;
    stretch_of(p.n_pages, threadIdx.x >> 6, from, to);
    auto is_live = [](int, int ref) { return ref > 0; };
    const int mine = count_pages(p.refs, from, to, 0, is_live);
    sum_waves(box, mine, live_before, live);
    auto is_hole = [&](int page, int ref) { return page < live && ref <= 0; };
    const int my_holes = count_pages(p.refs, from, min(to, live), 1, is_hole);
    sum_waves(box, my_holes, holes_before, holes);
    // (as many pages in use lie behind the first `live` places as there are holes in them)
    const int room = max(1, p.n_pages / 2);
    rank_pages(p.refs, from, min(to, live), 1, holes_before, is_hole, [&](int page, int, int rank) { pairs[2 * rank + 1] = page; });
    rank_pages(p.refs, from, to, 0, live_before, is_live, [&](int page, int, int rank) {
        if (page >= live) pairs[2 * (rank - (live - holes))] = page;
        else moved[page] = page;
    });
    for (int i = from + (threadIdx.x & 63); i < to; i += 64)
        if (p.refs[i] <= 0) moved[i] = -1;
    for (int i = holes + threadIdx.x; i < room; i += kThreads) pairs[2 * i] = pairs[2 * i + 1] = -1;
    if (threadIdx.x == 0) *count = holes;
    __syncthreads();
    for (int i = threadIdx.x; i < holes; i += kThreads) {
        const int src = pairs[2 * i], dst = pairs[2 * i + 1];
        moved[src] = dst;
        p.refs[dst] = p.refs[src];
        p.refs[src] = 0;
    }
}

// The table's entries in use get their pages' new numbers: a workgroup to a sequence.
__global__ __launch_bounds__(256) void pages_renumber_kernel(Pages p, const int32_t *moved)
{
    const int s = blockIdx.x, used = p.pages_for(p.len(s));
    int32_t *row = p.table + (size_t)s * p.max_pages;
    for (int j = threadIdx.x; j < used; j += 256) {
        const int page = row[j];
        if ((unsigned)page < (unsigned)p.n_pages) row[j] = moved[page];
    }
}

hipError_t allow(const void *kernel, OncePerDevice &once) { return allow_lds(once, kernel, 2 * kMaxSeqs * sizeof(int)); }

}  // namespace

hipError_t launch_pages_grow(const hgf_kv8_pages &p, const int32_t *seqs, const int32_t *add, int n, int32_t *ok, hipStream_t st)
{
    static OncePerDevice once;
    const hipError_t e = allow((const void *)pages_grow_kernel, once);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pages_grow_kernel, dim3(1), dim3(kThreads), (size_t)(p.n_seqs + n) * sizeof(int), st, pages_of(p), seqs, add, n, ok);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const hgf_kv8_pages &p, const int32_t *src, const int32_t *dst, int n, int32_t *pairs, int32_t *ok,
                             hipStream_t st)
{
    static OncePerDevice once;
    const hipError_t e = allow((const void *)pages_fork_kernel, once);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(kThreads), (size_t)(p.n_seqs + n) * sizeof(int), st, pages_of(p), src, dst, n,
                       pairs, ok);
    return hipGetLastError();
}

hipError_t launch_pages_free(const hgf_kv8_pages &p, const int32_t *seqs, int n, hipStream_t st)
{
    static OncePerDevice once;
    const hipError_t e = allow((const void *)pages_free_kernel, once);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pages_free_kernel, dim3(1), dim3(kThreads), (size_t)p.n_seqs * sizeof(int), st, pages_of(p), seqs, n);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const hgf_kv8_pages &p, int32_t *pairs, int32_t *count, int32_t *moved, hipStream_t st)
{
    hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kThreads), 0, st, pages_of(p), pairs, count, moved);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pages_renumber_kernel, dim3(p.n_seqs), dim3(256), 0, st, pages_of(p), moved);
    return hipGetLastError();
}

}  // namespace hgf
