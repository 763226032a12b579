// Differential attention over prompts: many query rows, ragged batches, capped or biased scores, masks.
//
//   out = (softmax(s1) V - lambda softmax(s2) V) / 2, both branches in one pass over the keys with running maxima and sums.
//
// A workgroup holds 128 query rows of one head and sequence, a wavefront 32 of them for both branches, and takes the
// keys 64 at a time: K1, K2 and V of the tile in LDS, double buffered, requested a tile ahead.  All products are
// computed transposed, S^T = K Q^T and O^T = V^T P^T on the 32x32x16 fp16 matrix instruction, so that a lane
// owns one query: its maximum, sum and rescaling are registers of the lane (one exchange between the halves of the wavefront),
// and the 8 weights of a step that a lane holds after S^T are the ones it has to supply for O^T if V's keys are taken in
// the order in which the accumulator's rows lie (4 h .. 4 h + 3 and 8 + 4 h .. for half h): P never moves.  V is
// transposed on its way into LDS.
// Weights are relative to the running maximum in base 2 and carried 2^7 larger, so that fp16 holds them down to
// 2^-31; the maximum is only raised when a tile exceeds it by 2^8 (which the factor leaves room for), which spares
// most rescalings.  fp32: scores, weights before rounding, sums, outputs.  The sum adds up the rounded weights.
// Masks are one comparison per element, key < limit of the row, and a comparison of document numbers where documents are
// given, both only in tiles that need them.  What a row does not see has weight 0; values of V that
// are no finite numbers are taken out of the tile and added to the rows that see them (0 * inf would reach
// the others).
// Bound by the exponentials and the vector instructions around them: 64 scores per lane and tile against
// 32 matrix instructions (64 columns).
#include "hgf_kv8.h"

#include <type_traits>

namespace hgf {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kRows = 128, kKeys = 64;
constexpr float kLift = 7.0f, kSlack = 8.0f;

struct PrefillParams {
    PrefillArgs a;
    float scale;
    int slots;
};

__device__ inline float soft_cap(float x, float cap, float inv)
{
    const float y = x * inv, y2 = y * y;
    const float series = y * __builtin_fmaf(y2, __builtin_fmaf(y2, __builtin_fmaf(y2, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.0f * kLog2e)) + 1.0f);
    return cap * (fabsf(y) < 0.3f ? series : t);
}

// Position of a 16-byte chunk of row `row` in LDS, so that the eight rows that are read together lie in different banks.
template <int D>
__device__ inline int k_chunk(int row, int c)
{
    constexpr int C = D / 8;                        // chunks of a row
    return row * C + (C >= 8 ? c ^ (row & 7) : C == 4 ? c ^ ((row >> 1) & 3) : c ^ ((row >> 2) & 1));
}
__device__ inline int v_chunk(int d, int c) { return d * (kKeys / 8) + (c ^ ((d ^ (d >> 3)) & 7)); }

template <int D>
struct Tile {
    static constexpr int kK = kKeys * D, kV = (D < 32 ? 32 : D) * kKeys;        // halves
    static constexpr int kHalves = 2 * kK + kV;
};

template <int D, bool MOD>
__global__ __launch_bounds__(256) void prefill_attn_kernel(PrefillParams p)
{
    constexpr int KS = D / 16, DT = (D + 31) / 32;  // steps of S^T; row tiles of O^T
    constexpr int KP = kKeys * D / 8 / 256 > 0 ? kKeys * D / 8 / 256 : 1;       // 16-byte pieces of a K per thread (D = 16: half the threads)
    constexpr int VT = kKeys * D / 16;              // 4 x 4 pieces of V of a tile
    constexpr int VP = VT / 256 > 0 ? VT / 256 : 1;
    extern __shared__ __align__(16) _Float16 lds[];
    __shared__ int odd_s[2][4];
    __shared__ int doc_s[2][kKeys];
    const PrefillArgs &a = p.a;
    const int H = a.n_heads, h = blockIdx.x % H;
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = l >> 5, col = l & 31;

    // ---- which rows: the slots of sequence b begin at cu_q[b] / 128 + b; the last ones first (they see the most keys)
    const int slot = p.slots - 1 - (int)(blockIdx.x / H);
    const int b = wave_search(a.B, slot, [&](int x) { return min(max(a.cu_q[x], 0), a.Tq) / kRows + x; });
    int q0, nq, k0, nk;
    clipped_rows(a.cu_q, b, a.Tq, q0, nq);
    clipped_rows(a.cu_k, b, a.Tk, k0, nk);
    const int first = (slot - q0 / kRows - b) * kRows;
    if (first < 0 || first >= nq) return;
    const int row = first + w * 32 + col;           // the lane's query
    const bool real = row < nq;
    const int pos = nk - nq + row;                  // its position among the keys
    int limit = a.causal ? max(pos + 1, a.prefix ? a.prefix[b] : 0) : nk;       // it sees keys below
    limit = min(max(limit, 0), nk);
    int doc = 0;
    if (a.doc_q) {
        doc = real ? a.doc_q[q0 + row] : -1;
        if (doc < 0) limit = 0;
    }
    if (!real) limit = 0;
    // rows of the wavefront that see the fewest and the most (missing rows do not count as seeing few)
    const int least = -(int)wave_max((float)-(real && doc >= 0 ? limit : nk)), most = (int)wave_max((float)limit);
    __shared__ int most_s[4];
    if (l == 0) most_s[w] = most;
    __syncthreads();
    const int end = max(max(most_s[0], most_s[1]), max(most_s[2], most_s[3]));
    const int tiles = (end + kKeys - 1) / kKeys;

    // ---- the queries, operand B of S^T
    v8h q[2][KS];
    {
        const size_t at = ((size_t)(q0 + min(row, nq - 1)) * 2 * H + h) * D + half * 8;
#pragma unroll
        for (int br = 0; br < 2; ++br)
#pragma unroll
            for (int s = 0; s < KS; ++s) q[br][s] = *reinterpret_cast<const v8h *>(a.q + at + (size_t)br * H * D + s * 16);
    }
    const float cap = a.softcap, cap_inv = cap > 0.0f ? 1.0f / cap : 0.0f;
    float slope[2] = {0.0f, 0.0f};
    if (MOD && a.slopes) {
        slope[0] = a.slopes[h] * kLog2e;
        slope[1] = a.slopes[H + h] * kLog2e;
    }
    const float unit = MOD ? p.scale : p.scale * kLog2e;

    v4u kr[2][KP];
    uint2 vr[VP][4];
    int doc_r = 0;
    auto request = [&](int tile) {
        const int key0 = tile * kKeys;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int at = i * 256 + tid, key = min(key0 + at / (D / 8), nk - 1), c = at % (D / 8);
            if (D >= 32 || tid < kKeys * D / 8) {
#pragma unroll
                for (int br = 0; br < 2; ++br)
                    kr[br][i] = *reinterpret_cast<const v4u *>(a.k + ((size_t)(k0 + key) * 2 * H + br * H + h) * D + c * 8);
            }
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const int at = i * 256 + tid, key = key0 + at / (D / 4) * 4, c = at % (D / 4);
            if (VT >= 256 || tid < VT) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    vr[i][j] = *reinterpret_cast<const uint2 *>(a.v + ((size_t)(k0 + min(key + j, nk - 1)) * H + h) * D + c * 4);
            }
        }
        if (a.doc_k && tid < kKeys) doc_r = key0 + tid < nk ? a.doc_k[k0 + key0 + tid] : -1;
    };
    // Into LDS; V as columns of 64 keys, the keys of a step of 16 in the order 0-3, 8-11, 4-7, 12-15.
    auto deposit = [&](int buf) {
        _Float16 *kb = lds + buf * Tile<D>::kHalves, *vb = kb + 2 * Tile<D>::kK;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int at = i * 256 + tid;
            if (D >= 32 || tid < kKeys * D / 8) {
#pragma unroll
                for (int br = 0; br < 2; ++br)
                    reinterpret_cast<v4u *>(kb + br * Tile<D>::kK)[k_chunk<D>(at / (D / 8), at % (D / 8))] = kr[br][i];
            }
        }
        bool odd = false;
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const int at = i * 256 + tid, quad = at / (D / 4), c = at % (D / 4);
            if (VT >= 256 || tid < VT) {
                const int slot8 = (quad & ~3) + ((quad & 1) << 1 | (quad & 2) >> 1);    // 8-byte place in a column
                uint32_t o = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    asm("v_pk_max_u16 %0, %1, %2" : "=v"(o) : "v"(o), "v"(vr[i][j].x & 0x7fff7fffu));
                    asm("v_pk_max_u16 %0, %1, %2" : "=v"(o) : "v"(o), "v"(vr[i][j].y & 0x7fff7fffu));
                }
                if (odd_magnitudes(o)) {
                    odd = true;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        auto clean = [](uint32_t x) {
                            if ((x & 0x7c00u) == 0x7c00u) x &= 0xffff0000u;
                            if ((x & 0x7c000000u) == 0x7c000000u) x &= 0x0000ffffu;
                            return x;
                        };
                        vr[i][j].x = clean(vr[i][j].x);
                        vr[i][j].y = clean(vr[i][j].y);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
                    auto word = [&](int j) { return e < 2 ? vr[i][j].x : vr[i][j].y; };
                    const uint2 x = make_uint2(__builtin_amdgcn_perm(word(1), word(0), sel), __builtin_amdgcn_perm(word(3), word(2), sel));
                    const int chunk = v_chunk(c * 4 + e, slot8 >> 1);
                    *reinterpret_cast<uint2 *>(vb + chunk * 8 + (slot8 & 1) * 4) = x;
                }
            }
        }
        if (a.doc_k && tid < kKeys) doc_s[buf][tid] = doc_r;
        const bool any = __any(odd);
        if (l == 0) odd_s[buf][w] = any ? 1 : 0;
    };

    float m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
    v16f o[2][DT];
#pragma unroll
    for (int br = 0; br < 2; ++br)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[br][t][e] = 0.0f;

    if (tiles > 0) {
        request(0);
        deposit(0);
    }
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        const int buf = tile & 1, key0 = tile * kKeys;
        if (tile + 1 < tiles) request(tile + 1);
        if (key0 < most) {
            const _Float16 *kb = lds + buf * Tile<D>::kHalves, *vb = kb + 2 * Tile<D>::kK;
            const bool partial = key0 + kKeys > least || a.doc_k;
            v8h pr[2][4];                           // weights of both branches, operand B of O^T
#pragma unroll
            for (int br = 0; br < 2; ++br) {
                v16f s[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[kt][e] = 0.0f;
#pragma unroll
                    for (int st = 0; st < KS; ++st) {
                        const v8h x = *reinterpret_cast<const v8h *>(kb + br * Tile<D>::kK + k_chunk<D>(kt * 32 + col, st * 2 + half) * 8);
                        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[br][st], s[kt], 0, 0, 0);
                    }
                }
                // scores in base 2
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x = s[kt][e] * unit;
                        if (MOD) {
                            const int key = key0 + kt * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                            if (cap > 0.0f) x = soft_cap(x, cap, cap_inv);
                            x = x * kLog2e - slope[br] * fabsf((float)(pos - key));
                        }
                        s[kt][e] = x;
                    }
                if (partial) {
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int in = kt * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                            bool seen = key0 + in < limit;
                            if (a.doc_k) seen = seen && doc_s[buf][in] == doc;
                            s[kt][e] = seen ? s[kt][e] : -INFINITY;
                        }
                }
                float top = s[0][0];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kt][e]);
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const bool raise = top > m[br] + kSlack;            // (for each row by itself: no row depends on its neighbours)
                if (__any(raise)) {
                    const float next = raise ? top : m[br];
                    const float corr = __builtin_amdgcn_exp2f(m[br] - (next == -INFINITY ? 0.0f : next));
                    m[br] = next;
                    sum[br] *= corr;
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[br][t][e] *= corr;
                }
                const float base = (m[br] == -INFINITY ? 0.0f : m[br]) - kLift;
                float add = 0.0f;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const _Float16 x = (_Float16)__builtin_amdgcn_exp2f(s[kt][e] - base);
                        pr[br][kt * 2 + (e >> 3)][e & 7] = x;
                        add += (float)x;
                    }
                sum[br] += add;
            }
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    const v8h x = *reinterpret_cast<const v8h *>(vb + v_chunk(t * 32 + col, st * 2 + half) * 8);
#pragma unroll
                    for (int br = 0; br < 2; ++br) o[br][t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, pr[br][st], o[br][t], 0, 0, 0);
                }
            if (odd_s[buf][0] | odd_s[buf][1] | odd_s[buf][2] | odd_s[buf][3]) {
                // values that are no finite numbers, to the rows that see them
                const int n = min(kKeys, nk - key0);
                for (int j = 0; j < n; ++j) {
                    bool seen = key0 + j < limit;
                    if (a.doc_k) seen = seen && doc_s[buf][j] == doc;
                    if (!__any(seen)) continue;
                    const _Float16 *v = a.v + ((size_t)(k0 + key0 + j) * H + h) * D;
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int d = t * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                            const float x = (float)v[d < D ? d : 0];
                            if (seen && !(fabsf(x) <= 65504.0f)) {
                                o[0][t][e] += x;
                                o[1][t][e] += x;
                            }
                        }
                }
            }
        }
        if (tile + 1 < tiles) deposit(buf ^ 1);
        __syncthreads();
    }
    if (!real) return;
    float f[2];
#pragma unroll
    for (int br = 0; br < 2; ++br) {
        const float total = sum[br] + __shfl_xor(sum[br], 32, 64);
        f[br] = total == 0.0f ? 0.0f : 0.5f / total;
    }
    f[1] *= a.lambda;
    _Float16 *out = a.out + ((size_t)(q0 + row) * H + h) * D;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int d = t * 32 + 8 * e4 + 4 * half;
            v4h x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (_Float16)(o[0][t][e4 * 4 + e] * f[0] - o[1][t][e4 * 4 + e] * f[1]);
            if (d < D) *reinterpret_cast<v4h *>(out + d) = x;
        }
}

}  // namespace

hipError_t launch_diff_attn_prefill(const PrefillArgs &a, int d_h, hipStream_t st)
{
    PrefillParams p;
    p.a = a;
    p.scale = 1.0f / sqrtf((float)d_h);
    p.slots = a.Tq / kRows + a.B;
    const bool mod = a.softcap > 0.0f || a.slopes;
    hipError_t e = hipSuccess;
    auto go = [&](auto d, auto m) {
        constexpr int D = decltype(d)::value;
        constexpr bool MOD = decltype(m)::value;
        constexpr size_t bytes = 2 * Tile<D>::kHalves * sizeof(_Float16);
        static OncePerDevice once;
        e = allow_lds(once, (const void *)(prefill_attn_kernel<D, MOD>), bytes);
        if (e == hipSuccess)
            hipLaunchKernelGGL((prefill_attn_kernel<D, MOD>), dim3((unsigned)p.slots * a.n_heads), dim3(256), bytes, st, p);
    };
    auto both = [&](auto d) {
        if (mod) go(d, std::true_type{});
        else go(d, std::false_type{});
    };
    switch (d_h) {
        case 16: both(std::integral_constant<int, 16>{}); break;
        case 32: both(std::integral_constant<int, 32>{}); break;
        case 64: both(std::integral_constant<int, 64>{}); break;
        default: both(std::integral_constant<int, 128>{}); break;
    }
    if (e != hipSuccess) return e;
    return hipGetLastError();
}

}  // namespace hgf
