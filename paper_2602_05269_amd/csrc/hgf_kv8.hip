// The paged 8-bit cache: writing new tokens, reading positions back, copying pages.
//
// 16 positions of one head share a scale 2^e, the smallest with 127 2^e >= the largest magnitude written.  A
// wavefront works on whole blocks of 16 positions, one 16-byte piece of codes to a lane: for K a piece is 16 columns of
// one position, for V 16 positions of one column (the order in which the attention's matrix instructions take
// them), so a block is d_h pieces and a head of 16, 32, 64, 128 columns takes a quarter, half, one or two wavefronts' worth.
// A block that gets new tokens is read (where older positions stay), rescaled where a new token is larger than what
// the scale reaches, and written whole by the lanes that hold it: no two wavefronts touch one block, so nothing is atomic and the codes
// do not depend on timing.
#include "hgf_kv8.h"

#include <type_traits>

namespace hgf {

namespace {

// Largest over aligned groups of G lanes, in every lane of the group.
template <int G>
__device__ inline float group_max(float v)
{
#pragma unroll
    for (int o = 1; o < G; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// Eight fp16 with what is not a number as 0 and infinities as the largest number.
__device__ inline v4u storable(v4u x)
{
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t r = 0;
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            const uint32_t v = (x[d] >> h) & 0xffffu, m = v & 0x7fffu;
            r |= (m < kOddBits ? v : m == kOddBits ? (v & 0x8000u) | 0x7bffu : 0u) << h;
        }
        x[d] = r;
    }
    return x;
}

// The smallest power of two 2^e, e >= -30, with 127 * 2^e >= amax (127 = 1.984375 * 2^6: the mantissa decides).
__device__ inline float block_scale(float amax)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x7e0000u ? 6 : 5);
    return __builtin_bit_cast(float, (uint32_t)(max(e, -30) + 127) << 23);
}

__device__ inline int code_of(float x) { return (int)fminf(fmaxf(rintf(x), -127.0f), 127.0f); }

// Byte i of a piece, sign extended.
__device__ inline int byte_of(v4u p, int i) { return (int)(int8_t)(p[i >> 2] >> (8 * (i & 3))); }

struct AppendParams {
    KvView kv;
    const _Float16 *k, *v;
    const int32_t *cu;                  // null: one token per row
    int B, T, k_groups;                 // workgroups that share the K heads of a block; the rest share the V heads
};

// Which 16 positions of which sequence a slot of the grid stands for.  With offsets, row b owns the slots from
// cu[b] / 16 + 2 b on: n tokens touch at most n / 16 + 2 blocks, and that many lie before the next row's.
struct Slot {
    int seq, blk, start, len, first_row;            // tokens: positions start .. len-1, rows first_row ..
};
__device__ inline bool find_slot(const KvView &kv, const int32_t *cu, int B, int T, int at, Slot &s)
{
    int b, n, i = 0;
    if (cu) {
        b = slot_entry<4, 2>(cu, B, T, at, s.first_row, n);
        i = at - (s.first_row >> 4) - 2 * b;
    } else {
        b = at;
        s.first_row = b;
        n = 1;
    }
    s.seq = kv.seq(b);
    if (s.seq < 0 || n == 0 || i < 0) return false;
    s.len = kv.len(s.seq);
    s.start = s.len - n;
    s.blk = (max(s.start, 0) >> 4) + i;             // (tokens in front of position 0 are dropped)
    return s.blk * kKvBlock < s.len;
}

template <int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(AppendParams p)
{
    constexpr int LPU = D < 64 ? D : 64, PPL = D / LPU, UNITS = 256 / LPU;      // lanes and pieces of a head, heads of a workgroup
    const KvView &kv = p.kv;
    Slot s;
    if (!find_slot(kv, p.cu, p.B, p.T, blockIdx.x, s)) return;
    const int page = kv.page_of(s.seq, s.blk);
    if (page < 0) return;
    const bool is_v = (int)blockIdx.y >= p.k_groups;
    const int heads = is_v ? kv.n_heads : 2 * kv.n_heads;
    const int head = (is_v ? blockIdx.y - p.k_groups : blockIdx.y) * UNITS + threadIdx.x / LPU;
    if (head >= heads) return;                      // (whole groups of LPU lanes)
    const int lane = threadIdx.x % LPU;
    const int pos0 = s.blk * kKvBlock, from = max(s.start, 0);
    const int lo = max(from - pos0, 0), hi = min(s.len - pos0, kKvBlock);       // the block's new positions: lo .. hi-1
    const int row0 = s.first_row + pos0 - s.start;  // row of the block's position 0 (it may lie in front of the tokens)
    const size_t at = kv.block(page, heads, head, s.blk);
    float *scale = (is_v ? kv.vs : kv.ks) + at;
    v4u *pieces = reinterpret_cast<v4u *>((is_v ? kv.v : kv.k) + at * 16 * D);
    const float old = lo > 0 ? *scale : 0.0f;
    // (V's new rows are read as rows and taken by columns from LDS)
    __shared__ __align__(16) _Float16 rows_s[UNITS][16][D + 8];
    auto &rows = rows_s[threadIdx.x / LPU];         // (the lanes of a head are lanes of one wavefront)
    if (is_v) {
#pragma unroll
        for (int j = 0; j < 2 * PPL; ++j) {
            const int chunk = j * LPU + lane, r = chunk / (D / 8), c = chunk % (D / 8), use = min(max(r, lo), hi - 1);
            *reinterpret_cast<v8h *>(&rows[r][c * 8]) =
                *reinterpret_cast<const v8h *>(p.v + ((size_t)(row0 + use) * heads + head) * D + c * 8);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    v4u x[PPL][2];                                  // 16 values of each of the lane's pieces
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < PPL; ++i) {
        const int piece = i * LPU + lane;
        if (!is_v) {
            const int pos = piece & 15, c = piece >> 4;
            const int use = min(max(pos, lo), hi - 1);              // (always a row of this sequence)
            const v4u *src = reinterpret_cast<const v4u *>(p.k + ((size_t)(row0 + use) * heads + head) * D + c * 16);
            x[i][0] = src[0];
            x[i][1] = src[1];
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                v8h t;
#pragma unroll
                for (int e = 0; e < 8; ++e) t[e] = rows[j * 8 + e][piece];
                x[i][j] = __builtin_bit_cast(v4u, t);
            }
        }
        largest = max_magnitudes(x[i][1], max_magnitudes(x[i][0], largest));
    }
    if (odd_magnitudes(largest)) {
        largest = 0;
#pragma unroll
        for (int i = 0; i < PPL; ++i) {
            x[i][0] = storable(x[i][0]);
            x[i][1] = storable(x[i][1]);
            largest = max_magnitudes(x[i][1], max_magnitudes(x[i][0], largest));
        }
    }
    const float scale_new = fmaxf(old, block_scale(group_max<LPU>(larger_magnitude(largest))));
    const float inv = 1.0f / scale_new, ratio = old / scale_new;    // (powers of two: exact)
    if (lane == 0) *scale = scale_new;
#pragma unroll
    for (int i = 0; i < PPL; ++i) {
        const int piece = i * LPU + lane;
        const int pos = piece & 15;
        int unused = 0;
        const uint2 q0 = eight_codes(x[i][0], inv, false, unused), q1 = eight_codes(x[i][1], inv, false, unused);
        v4u q = {q0.x, q0.y, q1.x, q1.y};
        if (!is_v) {
            if (pos >= lo && pos < hi) {
                pieces[piece] = q;
            } else if (pos < lo && ratio != 1.0f) {
                const v4u was = pieces[piece];
                v4u r = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 16; ++e) r[e >> 2] |= (uint32_t)(code_of((float)byte_of(was, e) * ratio) & 0xff) << (8 * (e & 3));
                pieces[piece] = r;
            }
        } else {
            if (lo > 0 || hi < kKvBlock) {
                const v4u was = pieces[piece];
                v4u r = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int b = byte_of(was, e);
                    const int kept = e < lo ? code_of((float)b * ratio) : b;
                    r[e >> 2] |= (e >= lo && e < hi ? (q[e >> 2] >> (8 * (e & 3))) & 0xffu : (uint32_t)(kept & 0xff)) << (8 * (e & 3));
                }
                q = r;
            }
            pieces[piece] = q;
        }
    }
}

struct GatherParams {
    KvView kv;
    const int32_t *cu;
    _Float16 *k, *v;
    int B, T, k_groups;
};

__device__ inline _Float16 value_of(int code, float scale)
{
    return (_Float16)fminf(fmaxf((float)code * scale, -65504.0f), 65504.0f);
}

// Positions in front of 0 (rows that ask for more than there is) become zero: the slots of a row count blocks from its
// first row's position, which may be negative.  A block's values go through LDS, so that they are stored as whole rows of a head:
// stored from the pieces as they lie (32 bytes of a position, two bytes of a column) 10600 positions of 32 heads of 64 columns
// took 46 us, 37 so.
template <int D>
__global__ __launch_bounds__(256) void kv8_gather_kernel(GatherParams p)
{
    constexpr int LPU = D < 64 ? D : 64, PPL = D / LPU, UNITS = 256 / LPU;
    const KvView &kv = p.kv;
    int row, n;
    const int b = slot_entry<4, 2>(p.cu, p.B, p.T, blockIdx.x, row, n);
    const int i = (int)blockIdx.x - (row >> 4) - 2 * b;
    const int seq = kv.seq(b);
    if (n == 0 || i < 0 || seq < 0) return;
    const int len = kv.len(seq), start = len - n;
    const int blk = (start >> 4) + i, pos0 = blk * kKvBlock;         // (start may be negative: the shift rounds down)
    if (pos0 >= len) return;
    const int page = blk >= 0 ? kv.page_of(seq, blk) : -1;
    const bool is_v = (int)blockIdx.y >= p.k_groups;
    const int heads = is_v ? kv.n_heads : 2 * kv.n_heads;
    const int head = (is_v ? blockIdx.y - p.k_groups : blockIdx.y) * UNITS + threadIdx.x / LPU;
    if (head >= heads) return;
    const int lane = threadIdx.x % LPU;
    const size_t at = kv.block(max(page, 0), heads, head, max(blk, 0));
    const float scale = page >= 0 ? (is_v ? kv.vs : kv.ks)[at] : 0.0f;
    const v4u *pieces = reinterpret_cast<const v4u *>((is_v ? kv.v : kv.k) + at * 16 * D);
    __shared__ __align__(16) _Float16 rows_s[UNITS][16][D + 8];
    auto &rows = rows_s[threadIdx.x / LPU];         // (the lanes of a head are lanes of one wavefront)
#pragma unroll
    for (int j = 0; j < PPL; ++j) {
        const int piece = j * LPU + lane;
        v4u q = {0, 0, 0, 0};
        if (page >= 0) q = pieces[piece];
        if (!is_v) {
            v8h a, z;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = value_of(byte_of(q, e), scale);
                z[e] = value_of(byte_of(q, 8 + e), scale);
            }
            v8h *dst = reinterpret_cast<v8h *>(&rows[piece & 15][(piece >> 4) * 16]);
            dst[0] = a;
            dst[1] = z;
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) rows[e][piece] = value_of(byte_of(q, e), scale);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    _Float16 *out = is_v ? p.v : p.k;
#pragma unroll
    for (int j = 0; j < 2 * PPL; ++j) {
        const int chunk = j * LPU + lane, r = chunk / (D / 8), c = chunk % (D / 8), pos = pos0 + r;
        const v8h x = *reinterpret_cast<const v8h *>(&rows[r][c * 8]);
        if (pos >= start && pos < len) *reinterpret_cast<v8h *>(out + ((size_t)(row + pos - start) * heads + head) * D + c * 8) = x;
    }
}

struct CopyParams {
    unsigned char *part[4];             // codes and scales of K and V
    size_t bytes[4];                    // of a page
    const int32_t *pairs, *count;
    int n, n_pages, splits;
};

constexpr int kCopyPiece = 16384;       // bytes of codes that a workgroup moves at a time

__global__ __launch_bounds__(256) void kv8_copy_kernel(CopyParams p)
{
    const int n = p.count ? min(max(*p.count, 0), p.n) : p.n;
    for (int i = blockIdx.y; i < n; i += gridDim.y) {
        const int src = p.pairs[2 * i], dst = p.pairs[2 * i + 1];
        if ((unsigned)src >= (unsigned)p.n_pages || (unsigned)dst >= (unsigned)p.n_pages || src == dst) continue;
#pragma unroll
        for (int part = 0; part < 4; part += 2) {
            const v4u *from = reinterpret_cast<const v4u *>(p.part[part] + src * p.bytes[part]);
            v4u *to = reinterpret_cast<v4u *>(p.part[part] + dst * p.bytes[part]);
            const size_t pieces = p.bytes[part] / 16;
            for (size_t at = (size_t)blockIdx.x * (kCopyPiece / 16); at < pieces; at += (size_t)p.splits * (kCopyPiece / 16)) {
                v4u x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = from[min(at + j * 256 + threadIdx.x, pieces - 1)];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (at + j * 256 + threadIdx.x < pieces) to[at + j * 256 + threadIdx.x] = x[j];
            }
        }
        if (blockIdx.x == 0) {
#pragma unroll
            for (int part = 1; part < 4; part += 2) {
                const uint32_t *from = reinterpret_cast<const uint32_t *>(p.part[part] + src * p.bytes[part]);
                uint32_t *to = reinterpret_cast<uint32_t *>(p.part[part] + dst * p.bytes[part]);
                for (int j = threadIdx.x; j < (int)(p.bytes[part] / 4); j += 256) to[j] = from[j];
            }
        }
    }
}

template <class F>
void for_head_size(int d_h, F f)
{
    switch (d_h) {
        case 16: f(std::integral_constant<int, 16>{}); break;
        case 32: f(std::integral_constant<int, 32>{}); break;
        case 64: f(std::integral_constant<int, 64>{}); break;
        default: f(std::integral_constant<int, 128>{}); break;
    }
}
int groups_of(int heads, int d_h)
{
    const int units = 256 / (d_h < 64 ? d_h : 64);
    return (heads + units - 1) / units;
}

}  // namespace

hipError_t launch_kv8_append(const void *k, const void *v, const KvView &kv, int d_h, const int32_t *cu, int B, int T,
                             hipStream_t st)
{
    AppendParams p = {kv, reinterpret_cast<const _Float16 *>(k), reinterpret_cast<const _Float16 *>(v), cu, B, T,
                      groups_of(2 * kv.n_heads, d_h)};
    const dim3 grid(cu ? T / kKvBlock + 2 * B : B, p.k_groups + groups_of(kv.n_heads, d_h));
    for_head_size(d_h, [&](auto d) { hipLaunchKernelGGL(kv8_append_kernel<decltype(d)::value>, grid, dim3(256), 0, st, p); });
    return hipGetLastError();
}

hipError_t launch_kv8_gather(const KvView &kv, int d_h, const int32_t *cu, int B, int T, void *k, void *v, hipStream_t st)
{
    GatherParams p = {kv, cu, reinterpret_cast<_Float16 *>(k), reinterpret_cast<_Float16 *>(v), B, T, groups_of(2 * kv.n_heads, d_h)};
    const dim3 grid(T / kKvBlock + 2 * B, p.k_groups + groups_of(kv.n_heads, d_h));
    for_head_size(d_h, [&](auto d) { hipLaunchKernelGGL(kv8_gather_kernel<decltype(d)::value>, grid, dim3(256), 0, st, p); });
    return hipGetLastError();
}

hipError_t launch_kv8_copy_pages(const hgf_kv8_cache &c, const int32_t *pairs, const int32_t *count, int n, hipStream_t st)
{
    CopyParams p;
    p.part[0] = reinterpret_cast<unsigned char *>(c.k_codes);
    p.part[1] = reinterpret_cast<unsigned char *>(c.k_scale);
    p.part[2] = reinterpret_cast<unsigned char *>(c.v_codes);
    p.part[3] = reinterpret_cast<unsigned char *>(c.v_scale);
    p.bytes[0] = (size_t)2 * c.n_heads * c.page * c.d_h;
    p.bytes[2] = p.bytes[0] / 2;
    p.bytes[1] = (size_t)2 * c.n_heads * (c.page / kKvBlock) * sizeof(float);
    p.bytes[3] = p.bytes[1] / 2;
    p.pairs = pairs;
    p.count = count;
    p.n = n;
    p.n_pages = c.n_pages;
    const int pieces = (int)((p.bytes[0] + kCopyPiece - 1) / kCopyPiece);
    p.splits = pieces < 64 ? pieces : 64;
    // (lists whose count lies on the device may be far longer than what is in them: not a workgroup for every pair there
    // could be)
    const int most = 8192 / p.splits, rows = n < most ? n : most;
    hipLaunchKernelGGL(kv8_copy_kernel, dim3(p.splits, rows), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace hgf
