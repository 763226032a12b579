// Differential attention, one decode step over the paged 8-bit cache.
//
// For every head the step reads 3 d_h bytes of codes a position and nothing else of size: bound by HBM.  All products
// run on the int8 matrix cores straight from the codes as they arrive, without a conversion:
//   scores: q is written as a 23-bit fixed-point number, three balanced digits of base 256.  A operand: the digits
//     (rows 4 g + 0..2 for the 16 positions of group g, zeros elsewhere), B operand: 16-byte pieces of K
//     as they lie in memory.  The instructions of 64 positions add up in one accumulator, in which lane l
//     finds the three digit sums of position l: no exchange between lanes.
//   weighted V: the softmax weights (times the scale of their block of V) of 64 positions relative to their largest, again
//     as three digits, rows 0..2 for branch 1 and 4..6 for branch 2, against pieces of V (16 positions of a column): one read of
//     V serves both branches, lane l holds branch (l / 16) mod 2 of columns 16 t + l mod 16.
// The integer sums are exact, a digit sum stays below 2^21, and what is rounded is q and a weight to 23 bits
// each, below fp32's own rounding of the products.  Running maximum, sums and the outputs between tiles are fp32.
// A wavefront takes tiles of 64 positions; a workgroup of four or eight merges its wavefronts in LDS; with more than one part
// of a sequence, a second launch merges the parts.  The parts of a sequence follow from its length on the device, their number
// from the batch and the table's capacity.
#include "hgf_kv8.h"

#include <type_traits>

namespace hgf {

namespace {

constexpr int kTile = 64;
constexpr float kLog2e = 1.44269504088896340736f;

struct Kv8AttnParams {
    KvView kv;
    const _Float16 *q;                  // [B, 2 n_heads, D]
    const float *slopes;                // [2 n_heads] or null
    float *part;                        // [B, n_heads, parts, 2, D + 2]: maximum (base 2), sum, weighted V
    _Float16 *out;                      // [B, n_heads, D]
    int parts;
    float lambda, softcap, scale;
};

// Tiles of each part of a sequence: no fewer than the wavefronts of a workgroup.
__device__ inline int part_tiles(int tiles, int parts) { return max((tiles + parts - 1) / parts, 4); }

// 2^(21 - exponent of v) for positive v: v times it lies in [2^21, 2^22), so its top digit of base 256 fits int8.
__device__ inline float fixed_point(float v)
{
    const int e = (int)(__builtin_bit_cast(uint32_t, v) >> 23) - 127;
    return __builtin_bit_cast(float, (uint32_t)(min(max(21 - e, -126), 127) + 127) << 23);
}
__device__ inline float reciprocal_of_power(float p) { return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, p)); }
// The three balanced digits of base 256 of an integer below 2^22 in magnitude, most significant first.
__device__ inline void digits_of(int n, int (&d)[3])
{
    d[2] = (int)(int8_t)n;
    n = (n - d[2]) >> 8;
    d[1] = (int)(int8_t)n;
    d[0] = (n - d[1]) >> 8;
}
__device__ inline float join_digits(v4i a)
{
    return __builtin_fmaf((float)a[0], 65536.0f, __builtin_fmaf((float)a[1], 256.0f, (float)a[2]));
}
// cap tanh(x / cap)
__device__ inline float soft_cap(float x, float cap, float inv)
{
    const float y = x * inv;
    const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.0f * kLog2e)) + 1.0f);
    return cap * (fabsf(y) < kTanhSeries ? tanh_series(y) : t);
}

// ONE: one part per sequence, eight wavefronts, and no merge afterwards.
template <int D, bool MOD, bool ONE>
__global__ __launch_bounds__(ONE ? 512 : 256) void kv8_attn_kernel(Kv8AttnParams p)
{
    constexpr int WAVES = ONE ? 8 : 4;
    constexpr int LD = D / 16;                      // 16-byte loads per lane of one head of K (or V) for 64 positions
    constexpr int QC = D == 128 ? 2 : 1;            // chunks of 16 columns whose digits a lane holds
    __shared__ __align__(16) unsigned char dig[WAVES][8][kTile], q_dig[2][4][D];
    __shared__ float o_s[WAVES][2][D], m_s[WAVES][2], l_s[WAVES][2];
    const KvView &kv = p.kv;
    const int H = kv.n_heads, h = blockIdx.x, part = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, l = tid & 63, g = l >> 4, r = l & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (q is requested before anything is known of the sequence: fewer trips to memory one after the other)
    _Float16 q_own[2][LD];
#pragma unroll
    for (int br = 0; br < 2; ++br)
#pragma unroll
        for (int c = 0; c < LD; ++c) q_own[br][c] = p.q[((size_t)b * 2 * H + br * H + h) * D + c * 16 + r];
    const int my_br = tid / D & 1;                  // the thread's column of q, for its digits
    const _Float16 q_mine = p.q[((size_t)b * 2 * H + my_br * H + h) * D + tid % D];
    const int seq = kv.seq(b);
    const int len = seq >= 0 ? kv.len(seq) : 0;
    const int tiles = (len + kTile - 1) / kTile, each = part_tiles(tiles, p.parts);
    const int t0 = part * each, t1 = min(t0 + each, tiles);
    _Float16 *out = p.out + ((size_t)b * H + h) * D;
    if (t0 >= t1) {                                 // (the merge reads no such part)
        if (ONE && tid < D) out[tid] = (_Float16)0.0f;
        return;
    }

    int own_next = kv.page_of(seq, (t0 + w) * 4 + g);           // (a tile ahead: of the lane's own block of 16 positions)

    // ---- q as digits: a thread takes a column apart, lane l holds digit r mod 4 of the columns that its k-group g takes in each
    // load (D < 64: the k-groups repeat the columns)
    v4i qd[2][QC];
    float q_scale[2], f[2];
    bool odd = false;
#pragma unroll
    for (int br = 0; br < 2; ++br) {
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < LD; ++c) {
            const float x = fabsf((float)q_own[br][c]);
            odd |= !(x <= 65504.0f);
            amax = x <= 65504.0f ? fmaxf(amax, x) : amax;
        }
        amax = wave_max(amax);
        f[br] = fixed_point(amax);
        q_scale[br] = amax > 0.0f ? reciprocal_of_power(f[br]) * p.scale : 0.0f;
    }
    if (tid < 2 * D) {
        const float x = (float)q_mine;
        int d[3];
        digits_of((int)rintf(fabsf(x) <= 65504.0f ? x * (my_br ? f[1] : f[0]) : 0.0f), d);
#pragma unroll
        for (int i = 0; i < 3; ++i) q_dig[my_br][i][tid % D] = (unsigned char)d[i];
        q_dig[my_br][3][tid % D] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int br = 0; br < 2; ++br)
#pragma unroll
        for (int i = 0; i < QC; ++i) qd[br][i] = *reinterpret_cast<const v4i *>(&q_dig[br][r & 3][(i * 4 + g % LD) * 16]);
    odd = __any(odd);

    float m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f}, o[LD];
#pragma unroll
    for (int t = 0; t < LD; ++t) o[t] = 0.0f;
    const float cap = p.softcap, cap_inv = cap > 0.0f ? 1.0f / cap : 0.0f;
    float slope[2] = {0.0f, 0.0f};
    if (MOD && p.slopes) {
        slope[0] = p.slopes[h];
        slope[1] = p.slopes[H + h];
    }

    for (int tile = t0 + w; tile < t1; tile += WAVES) {
        const int pos = tile * kTile + l;
        const int blk = tile * 4 + g;               // the lane's own block of 16 positions
        const int own = own_next;
        own_next = kv.page_of(seq, blk + 4 * WAVES);
        const bool valid = pos < len && own >= 0;
        const int page = max(own, 0);               // (where there is none: any address inside the pool)
        // block numbers of the lane's own block in the pools of K (both branches) and V
        const size_t kb[2] = {kv.block(page, 2 * H, h, blk), kv.block(page, 2 * H, H + h, blk)};
        const size_t vb = kv.block(page, H, h, blk);
        v4u kx[2][LD], vx[LD];
#pragma unroll
        for (int t = 0; t < LD; ++t) {
            // the piece that this lane takes: block (4 t + g) / LD of the tile, chunk (4 t + g) mod LD, position r
            const int from = (4 * t + g) / LD, chunk = (4 * t + g) % LD;
            const int pg = __shfl(page, from * 16, 64);
#pragma unroll
            for (int br = 0; br < 2; ++br) {
                const size_t at = kv.block(pg, 2 * H, br * H + h, tile * 4 + from);
                kx[br][t] = *reinterpret_cast<const v4u *>(kv.k + at * (16 * D) + (chunk * 16 + r) * 16);
            }
        }
        const float ks[2] = {kv.ks[kb[0]], kv.ks[kb[1]]}, vs = kv.vs[vb];
#pragma unroll
        for (int t = 0; t < LD; ++t) vx[t] = *reinterpret_cast<const v4u *>(kv.v + vb * (16 * D) + (t * 16 + r) * 16);

        float f_inv[2], corr[2];
#pragma unroll
        for (int br = 0; br < 2; ++br) {
            v4i acc = {0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < LD; ++t) {
                const bool mine = (r >> 2) == (4 * t + g) / LD;         // rows of that block's positions
                v4i a = qd[br][QC == 2 ? t & 1 : 0];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = mine ? a[i] : 0;
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, __builtin_bit_cast(v4i, kx[br][t]), acc, 0, 0, 0);
            }
            float x = join_digits(acc) * (q_scale[br] * ks[br]);
            if (MOD) {
                if (cap > 0.0f) x = soft_cap(x, cap, cap_inv);
                x -= slope[br] * (float)(len - 1 - pos);
            }
            x = valid ? x * kLog2e : -INFINITY;
            const float top = fmaxf(m[br], wave_max(x));
            const float base = top == -INFINITY ? 0.0f : top;
            corr[br] = __builtin_amdgcn_exp2f(m[br] - base);
            m[br] = top;
            const float e = __builtin_amdgcn_exp2f(x - base);
            sum[br] = sum[br] * corr[br] + e;
            const float wt = valid ? e * vs : 0.0f;
            const float f = fixed_point(wave_max(wt));
            f_inv[br] = reciprocal_of_power(f);
            int d[3];
            digits_of((int)rintf(wt * f), d);
#pragma unroll
            for (int i = 0; i < 3; ++i) dig[w][br * 4 + i][l] = (unsigned char)d[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const v4i wd = *reinterpret_cast<const v4i *>(&dig[w][r & 7][g * 16]);      // (rows 3 and 7: sums that nothing reads)
        const float my_corr = g & 1 ? corr[1] : corr[0], my_f = g & 1 ? f_inv[1] : f_inv[0];
#pragma unroll
        for (int t = 0; t < LD; ++t) {
            const v4i zero = {0, 0, 0, 0};
            const v4i acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wd, __builtin_bit_cast(v4i, vx[t]), zero, 0, 0, 0);
            o[t] = __builtin_fmaf(o[t], my_corr, join_digits(acc) * my_f);
        }
        __builtin_amdgcn_wave_barrier();            // (the digits are read before the next tile's are written)
    }

    // ---- the wavefronts' results, merged
#pragma unroll
    for (int br = 0; br < 2; ++br)
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) sum[br] += __shfl_xor(sum[br], i, 64);
    if (g < 2) {
#pragma unroll
        for (int t = 0; t < LD; ++t) o_s[w][g][t * 16 + r] = o[t];
    }
    if (l < 2) {
        m_s[w][l] = l == 0 ? m[0] : m[1];
        l_s[w][l] = l == 0 ? sum[0] : sum[1];
    }
    __syncthreads();
    const int br = tid / D, d = tid % D;
    float acc = 0.0f, total = 0.0f, top = -INFINITY;
    if (br < 2) {
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = fmaxf(top, m_s[i][br]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float f = __builtin_amdgcn_exp2f(m_s[i][br] - base);
            acc += o_s[i][br][d] * f;
            total += l_s[i][br] * f;
        }
        if (odd) acc = __builtin_nanf("");
    }
    if (ONE) {
        if (br < 2) o_s[0][br][d] = total > 0.0f ? acc / total : 0.0f;      // (its own element; nothing seen: 0, whatever q is)
        __syncthreads();
        if (br == 0) out[d] = (_Float16)((o_s[0][0][d] - p.lambda * o_s[0][1][d]) * 0.5f);
    } else if (br < 2) {
        float *dst = p.part + ((((size_t)b * H + h) * p.parts + part) * 2 + br) * (D + 2);
        dst[2 + d] = acc;
        if (d == 0) {
            dst[0] = top;
            dst[1] = total;
        }
    }
}

// One workgroup per head and sequence: first the parts' largest maximum and their weighted sums' total, by one wavefront a branch,
// then the columns, groups of threads taking every so many parts.  Bound by latency.
template <int D>
__global__ __launch_bounds__(512) void kv8_merge_kernel(Kv8AttnParams p)
{
    constexpr int GROUPS = 512 / D;
    __shared__ float red[GROUPS][2][D], top_s[2], sum_s[2];
    const int H = p.kv.n_heads, h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int seq = p.kv.seq(b);
    const int tiles = seq >= 0 ? (p.kv.len(seq) + kTile - 1) / kTile : 0, each = part_tiles(tiles, p.parts);
    const int used = tiles > 0 ? (tiles + each - 1) / each : 0;
    const float *part = p.part + ((size_t)b * H + h) * p.parts * 2 * (D + 2);
    if (tid < 128) {
        const int br = tid >> 6, l = tid & 63;
        float top = -INFINITY;
        for (int c = l; c < used; c += 64) top = fmaxf(top, part[(c * 2 + br) * (D + 2)]);
        top = wave_max(top);
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        for (int c = l; c < used; c += 64) {
            const float *q = part + (c * 2 + br) * (D + 2);
            sum += q[1] * __builtin_amdgcn_exp2f(q[0] - base);
        }
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i, 64);
        if (l == 0) {
            top_s[br] = base;
            sum_s[br] = sum;
        }
    }
    __syncthreads();
    const int d = tid % D, grp = tid / D;
    float acc[2] = {0.0f, 0.0f};
#pragma unroll 4
    for (int c = grp; c < used; c += GROUPS) {
#pragma unroll
        for (int br = 0; br < 2; ++br) {
            const float *q = part + (c * 2 + br) * (D + 2);
            acc[br] += q[2 + d] * __builtin_amdgcn_exp2f(q[0] - top_s[br]);
        }
    }
    red[grp][0][d] = acc[0];
    red[grp][1][d] = acc[1];
    __syncthreads();
    if (tid < D) {
        float o[2];
#pragma unroll
        for (int br = 0; br < 2; ++br) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) s += red[i][br][tid];
            o[br] = sum_s[br] > 0.0f ? s / sum_s[br] : 0.0f;        // (nothing seen: 0, whatever q is)
        }
        p.out[((size_t)b * H + h) * D + tid] = (_Float16)((o[0] - p.lambda * o[1]) * 0.5f);
    }
}

// Parts of every sequence.  One, taken by workgroups of eight wavefronts, in tables of up to 1024 positions and, up to 8192, where
// there are so many sequences and heads that their lengths level each other out, 12 positions of capacity or fewer to
// each: no second launch.  (us, one part of eight wavefronts / several of four, caches from memory: 8 sequences of up to 1024, 8 heads of
// 32 6.1 / 7.4, of up to 2048 8.8 / 7.7; 20 of up to 2048, 8 of 32 9.5 / 10.4; 16 of up to 3000, 16 of 32 13.5 / 14.4; 16 of up to 4096,
// 16 of 128 52.3 / 50.2; 32 of up to 4096, 16 of 64 48.4 / 53.1; 16 of up to 8192, 16 of 128 93.5 / 88.4; 32 of up to 8192, 32 of 32
// 85.2 / 90.8.)
// Else the larger of two numbers, and none of fewer than 256 positions:
// - about as many workgroups as the chip holds at a time (1024 of 64 columns).  More of them start and merge for longer than they
//   level out, fewer leave ragged sequences' ends alone.  (us, for 768 / 1024 / 1536 workgroups: 8 ragged of up to 4096, 32 heads of 64
//   28.1 / 26.5 / 27.4, full 42.5 / 41.8 / 43.7; 16 ragged of up to 8192, 16 of 128 104.2 / 94.4 / 96.1.)
// - parts of up to 4096 positions, within 16384 workgroups, for the long sequence among short ones.  (us, without / with, 64 sequences,
//   16 heads of 64, one of 65536 positions and the others below 1200 314 / 78; ragged ones of up to 16384 383 / 351; where none
//   is long after all, 37 / 43.)
int parts_of(int B, long long capacity, int n_heads)
{
    const long long rows = (long long)B * n_heads;
    if (capacity <= 1024 || (capacity <= 8192 && capacity <= 12 * rows)) return 1;
    const long long fill = (1024 + rows - 1) / rows, room = 16384 / rows, cut = (capacity + 4095) / 4096, most = (capacity + 255) / 256;
    const long long parts = fill > room || fill > cut ? fill : room < cut ? room : cut;
    return (int)(parts < most ? parts : most);
}

}  // namespace

size_t diff_attn_kv8_workspace_bytes(int B, long long capacity, int n_heads, int d_h)
{
    const int parts = parts_of(B, capacity, n_heads);
    return parts > 1 ? (size_t)B * n_heads * parts * 2 * (d_h + 2) * sizeof(float) : 0;
}

hipError_t launch_diff_attn_kv8(const void *q, const KvView &kv, int B, int d_h, float lambda, float softcap, const float *slopes,
                                void *out, void *workspace, hipStream_t st)
{
    Kv8AttnParams p;
    p.kv = kv;
    p.q = reinterpret_cast<const _Float16 *>(q);
    p.slopes = slopes;
    p.part = reinterpret_cast<float *>(workspace);
    p.out = reinterpret_cast<_Float16 *>(out);
    p.parts = parts_of(B, (long long)kv.max_pages << kv.page_log2, kv.n_heads);
    p.lambda = lambda;
    p.softcap = softcap;
    p.scale = 1.0f / sqrtf((float)d_h);
    const dim3 grid(kv.n_heads, p.parts, B);
    const bool mod = softcap > 0.0f || slopes, one = p.parts == 1;
    auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (one && mod) hipLaunchKernelGGL((kv8_attn_kernel<D, true, true>), grid, dim3(512), 0, st, p);
        else if (one) hipLaunchKernelGGL((kv8_attn_kernel<D, false, true>), grid, dim3(512), 0, st, p);
        else if (mod) hipLaunchKernelGGL((kv8_attn_kernel<D, true, false>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((kv8_attn_kernel<D, false, false>), grid, dim3(256), 0, st, p);
        if (!one) hipLaunchKernelGGL(kv8_merge_kernel<D>, dim3(kv.n_heads, B), dim3(512), 0, st, p);
    };
    switch (d_h) {
        case 16: go(std::integral_constant<int, 16>{}); break;
        case 32: go(std::integral_constant<int, 32>{}); break;
        case 64: go(std::integral_constant<int, 64>{}); break;
        default: go(std::integral_constant<int, 128>{}); break;
    }
    return hipGetLastError();
}

}  // namespace hgf
