// Shared by the sources of the paged 8-bit cache and of the attention over prompts (not part of the ABI).
#pragma once

#include "hgf_internal.h"

namespace hgf {

constexpr int kKvBlock = 16;                // positions that share a scale
constexpr int kMaxSeqs = 16384;             // rows of a page table (two int32 of LDS each in the page operations)

// What the kernels need of a cache and its table, by value.
struct KvView {
    int8_t *k, *v;
    float *ks, *vs;
    const int32_t *table, *lens, *seqs;     // seqs may be null
    int n_pages, n_seqs, max_pages, n_heads;
    int page_log2;                          // positions per page: 16 << (page_log2 - 4)

    // Sequence of a batch row, or -1.
    __device__ int seq(int b) const
    {
        const int s = seqs ? seqs[b] : b;
        return (unsigned)s < (unsigned)n_seqs ? s : -1;
    }
    __device__ int len(int s) const { return min(max(lens[s], 0), max_pages << page_log2); }
    // Page that holds block `blk` (16 positions) of sequence s, or -1.
    __device__ int page_of(int s, int blk) const
    {
        const int i = blk >> (page_log2 - 4);
        const int p = (unsigned)i < (unsigned)max_pages ? table[(size_t)s * max_pages + i] : -1;
        return (unsigned)p < (unsigned)n_pages ? p : -1;
    }
    // Number of a block among all blocks of `heads` heads' pool (times 16 d_h: its codes, itself: its scale).
    __device__ size_t block(int page, int heads, int head, int blk) const
    {
        return (((size_t)page * heads + head) << (page_log2 - 4)) + (blk & ((1 << (page_log2 - 4)) - 1));
    }
};

KvView kv_view(const hgf_kv8_cache &c, const hgf_kv8_pages &p, const int32_t *seqs);

// Rising offsets cu[0 .. B] clipped to 0 .. T; the rows of batch entry b.
__device__ inline void clipped_rows(const int32_t *cu, int b, int T, int &first, int &n)
{
    first = min(max(cu[b], 0), T);
    n = max(min(max(cu[b + 1], 0), T) - first, 0);
}

// Largest b in 0 .. B-1 whose key(b) is at most `at`, keys rising from key(0) <= at: 64 keys a step, so up to
// 4096 batch entries take two dependent loads.  Any keys give a b inside the range.
template <class Key>
__device__ inline int wave_search(int B, int at, Key key)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = B;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool below = i < n && key(lo + (i < n ? i : 0)) <= at;
        const int c = max(1, (int)__popcll(__ballot(below)));
        const int skip = (c - 1) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    return lo;
}

// Batch entry b that slot `at` of a grid belongs to, where entry b has the slots from row(b) / 2^SHIFT + PER b on (row(b): its first
// row), and its rows.  Up to 64 entries in one trip to memory.
template <int SHIFT, int PER>
__device__ inline int slot_entry(const int32_t *cu, int B, int T, int at, int &first, int &n)
{
    auto clip = [&](int x) { return min(max(x, 0), T); };
    if (B <= 64) {
        const int lane = threadIdx.x & 63, i = min(lane, B - 1);
        const int from = clip(cu[i]), to = clip(cu[i + 1]);
        const bool below = lane < B && (from >> SHIFT) + PER * i <= at;
        const int b = max(1, (int)__popcll(__ballot(below))) - 1;
        first = __builtin_amdgcn_readlane(from, b);
        n = max(__builtin_amdgcn_readlane(to, b) - first, 0);
        return b;
    }
    const int b = wave_search(B, at, [&](int x) { return (clip(cu[x]) >> SHIFT) + PER * x; });
    clipped_rows(cu, b, T, first, n);
    return b;
}

// tanh(y) of a capped score for |y| below kTanhSeries, where 1 - 2 / (e^2y + 1) would cancel: within 4e-8 in fp32 (up to y^7 only it
// was 4.3e-7 at the end, and the other form is within 1.9e-7 there).
constexpr float kTanhSeries = 0.3f;
__device__ inline float tanh_series(float y)
{
    const float y2 = y * y;
    const float p = __builtin_fmaf(y2, __builtin_fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f);
    return y * __builtin_fmaf(y2, __builtin_fmaf(y2, p, -1.0f / 3.0f), 1.0f);
}

hipError_t launch_kv8_append(const void *k, const void *v, const KvView &kv, int d_h, const int32_t *cu, int B, int T,
                             hipStream_t st);
hipError_t launch_kv8_gather(const KvView &kv, int d_h, const int32_t *cu, int B, int T, void *k, void *v, hipStream_t st);
hipError_t launch_kv8_copy_pages(const hgf_kv8_cache &c, const int32_t *pairs, const int32_t *count, int n, hipStream_t st);

hipError_t launch_pages_grow(const hgf_kv8_pages &p, const int32_t *seqs, const int32_t *add, int n, int32_t *ok, hipStream_t st);
hipError_t launch_pages_fork(const hgf_kv8_pages &p, const int32_t *src, const int32_t *dst, int n, int32_t *pairs, int32_t *ok,
                             hipStream_t st);
hipError_t launch_pages_free(const hgf_kv8_pages &p, const int32_t *seqs, int n, hipStream_t st);
hipError_t launch_pages_compact(const hgf_kv8_pages &p, int32_t *pairs, int32_t *count, int32_t *moved, hipStream_t st);

size_t diff_attn_kv8_workspace_bytes(int B, long long capacity, int n_heads, int d_h);
hipError_t launch_diff_attn_kv8(const void *q, const KvView &kv, int B, int d_h, float lambda, float softcap, const float *slopes,
                                void *out, void *workspace, hipStream_t st);

struct PrefillArgs {
    const _Float16 *q, *k, *v;
    const int32_t *cu_q, *cu_k;              // cu_k is cu_q where the caller gave none
    const int32_t *prefix, *doc_q, *doc_k;   // may be null
    const float *slopes;                     // may be null
    _Float16 *out;
    int B, Tq, Tk, n_heads, causal;
    float lambda, softcap;
};
hipError_t launch_diff_attn_prefill(const PrefillArgs &a, int d_h, hipStream_t st);

}  // namespace hgf
