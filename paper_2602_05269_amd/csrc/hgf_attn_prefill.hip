// Differential attention over prompts: many query rows, ragged batches, capped or biased scores, masks.
//
//   out = (softmax(s1) V - lambda softmax(s2) V) / 2, both branches in one pass over the keys with running maxima and sums.
//
// A workgroup of eight wavefronts holds 128 query rows of one head and sequence, a wavefront 32 of them for one of the branches, and
// takes the keys 64 at a time: K1, K2 and V of the tile in LDS, double buffered, requested a tile ahead.  All
// products are computed transposed, S^T = K Q^T and O^T = V^T P^T on the 32x32x16 fp16 matrix instruction, so that
// a lane owns one query: its maximum, sum and rescaling are registers of the lane (one exchange between the halves of the
// wavefront), and the 8 weights of a step that a lane holds after S^T are the ones it has to supply for O^T if V's
// keys are taken in the order in which the accumulator's rows lie (4 h .. 4 h + 3 and 8 + 4 h .. for half h): P never
// moves.  V is transposed on its way into LDS.
// Few rows would leave most of the chip idle: then (SPLIT) a workgroup holds 32 rows, takes 128 keys at a time, and its
// wavefronts share the keys of a tile; they are merged at the end.
// Weights are relative to the running maximum in base 2 and carried 2^7 larger, so that fp16 holds them down to
// 2^-31; a row's maximum is only raised when a tile exceeds it by 2^8 (which the factor leaves room for), which spares
// most rescalings.  fp32: scores, weights before rounding, sums, outputs.  The sum adds up the rounded weights.
// Masks are one comparison per element, key < limit of the row, and a comparison of document numbers where documents are
// given, both only in tiles that need them; tiles whose document numbers lie outside those of the rows are not
// read.  What a row does not see has weight 0; values of V that are no finite numbers are taken out of the tile and
// added to the rows that see them (0 * inf would reach the others).
// Bound by the exponentials and the vector instructions around them up to 64 columns: 32 scores per lane and
// tile against 16 matrix instructions.
#include "hgf_kv8.h"

#include <limits.h>
#include <type_traits>

namespace hgf {

namespace {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr float kLift = 7.0f, kSlack = 8.0f;
// From here on 1 - 2 / (e^2y + 1) is too coarse a tanh near 0: its error, 2^-23 of the cap, passes 6e-5.
constexpr float kCoarseCap = 512.0f;

struct PrefillParams {
    PrefillArgs a;
    float scale;
    int slots;
};

// Sizes of one variant.
template <int D, int SPLIT>
struct Shape {
    static constexpr int kRows = 128 / SPLIT, kKeys = SPLIT == 1 ? 64 : 128;
    static constexpr int kSub = kKeys / 32 / SPLIT;             // groups of 32 keys per wavefront and tile
    static constexpr int kChunksK = D / 8, kChunksV = kKeys / 8;
    static constexpr int kK = kKeys * D, kV = (D < 32 ? 32 : D) * kKeys, kHalves = 2 * kK + kV;
    static constexpr int kBufs = 2 * kHalves * 2 <= 147456 ? 2 : 1;
    static constexpr int kTileT = (D + 31) / 32;                // row tiles of O^T
    // outputs on their way between wavefronts, in the tiles' place
    static constexpr size_t kLds = (size_t)kBufs * kHalves * 2;
    static_assert((size_t)(SPLIT == 1 ? 4 : 6) * kTileT * 4096 <= kLds, "the merge fits where the tiles were");
};

// Place of a 16-byte chunk of row `row` of K, and of column d of V, so that the eight rows that are read together lie in
// different banks.
template <int C>
__device__ inline int k_chunk(int row, int c)
{
    return row * C + (C >= 8 ? c ^ (row & 7) : C == 4 ? c ^ ((row >> 1) & 3) : c ^ ((row >> 2) & 1));
}
template <int C>
__device__ inline int v_chunk(int d, int c) { return d * C + (c ^ ((d ^ (d >> 3)) & 7)); }

// A value that the compiler does not see through: what rare paths compute from it is computed there, instead of being kept
// in registers across the loop.
__device__ inline int opaque(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
// The larger of a lane's value and of the lane 32 further on or back.
__device__ inline float halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}

template <int D, bool MOD, int SPLIT>
__global__ __launch_bounds__(kThreads, 2) void prefill_attn_kernel(PrefillParams p)
{
    using S = Shape<D, SPLIT>;
    constexpr int KS = D / 16, DT = S::kTileT, SUB = S::kSub, CK = S::kChunksK, CV = S::kChunksV;
    constexpr int KP = 2 * S::kKeys * CK / kThreads > 0 ? 2 * S::kKeys * CK / kThreads : 1;     // 16-byte pieces of K per thread
    constexpr int KALL = 2 * S::kKeys * CK;
    constexpr int VALL = S::kKeys * D / 16, VP = VALL > kThreads ? VALL / kThreads : 1;         // 4 x 4 pieces of V per thread
    extern __shared__ __align__(16) _Float16 lds[];
    __shared__ int odd_s[2][kWaves], doc_s[2][S::kKeys];
    __shared__ int most_s[kWaves], least_s[kWaves], lo_s[kWaves], hi_s[kWaves], win_lo[kWaves][64], win_hi[kWaves][64];
    __shared__ float m_s[SPLIT][2][32], sum_s[SPLIT][2][32];
    const PrefillArgs &a = p.a;
    const int H = a.n_heads, h = blockIdx.x % H;
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = l >> 5, col = l & 31;
    const int br = w >> 2, group = SPLIT == 1 ? w & 3 : 0, split = SPLIT == 1 ? 0 : w & 3;

    // ---- which rows: the slots of sequence b begin at cu_q[b] / kRows + b; the last ones first (they see the most keys)
    const int slot = p.slots - 1 - (int)(blockIdx.x / H);
    const int b = wave_search(a.B, slot, [&](int x) { return min(max(a.cu_q[x], 0), a.Tq) / S::kRows + x; });
    int q0, nq, k0, nk;
    clipped_rows(a.cu_q, b, a.Tq, q0, nq);
    clipped_rows(a.cu_k, b, a.Tk, k0, nk);
    const int first = (slot - q0 / S::kRows - b) * S::kRows;
    if (first < 0 || first >= nq) return;
    const int row = first + group * 32 + col;       // the lane's query
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
    const bool counts = real && doc >= 0;
    // the fewest keys that a row of the wavefront sees (0 for padding: its rows see none), and the most
    const int least = -(int)wave_max((float)-(real ? limit : nk)), most = (int)wave_max((float)limit);
    int tiles, whole, doc_lo = 0, doc_hi = 0;       // tiles that some row sees, that all rows see whole
    {
        int lo = counts ? doc : INT_MAX, hi = counts ? doc : -1;
        if (a.doc_q) {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                lo = min(lo, __shfl_xor(lo, o, 64));
                hi = max(hi, __shfl_xor(hi, o, 64));
            }
        }
        if (l == 0) {
            most_s[w] = most;
            least_s[w] = least;
            lo_s[w] = lo;
            hi_s[w] = hi;
        }
        __syncthreads();
        int end = 0, all = INT_MAX;
        doc_lo = INT_MAX;
        doc_hi = -1;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            end = max(end, most_s[i]);
            all = min(all, least_s[i]);
            doc_lo = min(doc_lo, lo_s[i]);
            doc_hi = max(doc_hi, hi_s[i]);
        }
        tiles = __builtin_amdgcn_readfirstlane((end + S::kKeys - 1) / S::kKeys);
        whole = min(tiles, __builtin_amdgcn_readfirstlane(all / S::kKeys));
    }

    // ---- the queries, operand B of S^T
    v8h q[KS];
    {
        const _Float16 *src = a.q + ((size_t)(q0 + min(row, nq - 1)) * 2 * H + br * H + h) * D + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8h *>(src + s * 16);
    }
    const float cap = a.softcap;
    float slope = 0.0f;
    if (MOD && a.slopes) slope = a.slopes[br * H + h] * kLog2e;
    const float unit = MOD ? 1.0f : p.scale * kLog2e;
    const v2h ones = {(_Float16)1.0f, (_Float16)1.0f};

    // ---- tiles on their way: global memory -> registers -> LDS.
    // A tile's rows are read through a descriptor that ends where the sequence does: rows behind it are zeros, and what a
    // thread adds to the tile's address does not change from tile to tile.
    const unsigned k_row = (unsigned)H * D * 4, v_row = (unsigned)H * D * 2;
    auto rows_of = [&](const _Float16 *base, unsigned row_bytes, int key0) {
        return make_rsrc(reinterpret_cast<const char *>(base) + (size_t)(k0 + key0) * row_bytes, (unsigned)min(nk - key0, S::kKeys) * row_bytes);
    };
    v4u kr[KP];
    uint2 vr[VP][4];
    int doc_r = 0;
    const unsigned k_off = (unsigned)(tid % (KALL / 2) / CK) * k_row + (unsigned)((tid / (KALL / 2) * H + h) * D + tid % CK * 8) * 2;
    const unsigned v_off = (unsigned)(tid / (D / 4) * 4) * v_row + (unsigned)(h * D + tid % (D / 4) * 4) * 2;
    auto request_k = [&](int tile) {
        const rsrc_t r = rows_of(a.k, k_row, tile * S::kKeys);
        if (KALL >= kThreads || tid < KALL) {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                // (piece i * kThreads + tid: so many rows, or the other K, further on)
                constexpr int HALF = KALL / 2;
                const unsigned more = (unsigned)(i * kThreads % HALF / CK) * k_row + (unsigned)(i * kThreads / HALF * H * D) * 2;
                kr[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(r, (int)k_off, (int)more, 0));
            }
        }
    };
    auto request_v = [&](int tile) {
        const rsrc_t r = rows_of(a.v, v_row, tile * S::kKeys);
        if (VALL >= kThreads || tid < VALL) {
#pragma unroll
            for (int i = 0; i < VP; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    vr[i][j] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(
                                                             r, (int)v_off, (int)((unsigned)(i * (kThreads / (D / 4)) * 4 + j) * v_row), 0));
        }
        if (a.doc_k && tid < S::kKeys) {
            const int key = tile * S::kKeys + tid;
            doc_r = key < nk ? a.doc_k[k0 + key] : -1;
        }
    };
    auto deposit_k = [&](int buf) {
        _Float16 *kb = lds + buf * 2 * S::kK;
        if (KALL >= kThreads || tid < KALL) {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int at = i * kThreads + tid;
                reinterpret_cast<v4u *>(kb + at / (KALL / 2) * S::kK)[k_chunk<CK>(at % (KALL / 2) / CK, at % CK)] = kr[i];
            }
        }
    };
    // V as columns of keys, the keys of a step of 16 in the order 0-3, 8-11, 4-7, 12-15.
    auto deposit_v = [&](int buf) {
        _Float16 *vb = lds + S::kBufs * 2 * S::kK + buf * S::kV;
        bool odd = false;
        if (VALL >= kThreads || tid < VALL) {
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                const int at = i * kThreads + tid, quad = at / (D / 4), c = at % (D / 4);
                const int place = (quad & ~3) + ((quad & 1) << 1 | (quad & 2) >> 1);    // 8-byte place in a column
                v2h o = {(_Float16)0.0f, (_Float16)0.0f};           // 0 * x: what is no finite number leaves a NaN
                const v2h zero = o;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o = __builtin_elementwise_fma(__builtin_bit_cast(v2h, vr[i][j].x), zero, o);
                    o = __builtin_elementwise_fma(__builtin_bit_cast(v2h, vr[i][j].y), zero, o);
                }
                if ((__builtin_bit_cast(uint32_t, o) & 0x7fff7fffu) != 0) {
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
                    *reinterpret_cast<uint2 *>(vb + v_chunk<CV>(c * 4 + e, place >> 1) * 8 + (place & 1) * 4) = x;
                }
            }
        }
        if (a.doc_k && tid < S::kKeys) doc_s[buf][tid] = doc_r;
        const bool any = __any(odd);
        if (l == 0) odd_s[buf][w] = any ? 1 : 0;
    };

    auto request = [&](int tile) {
        request_k(tile);
        request_v(tile);
    };
    auto deposit = [&](int buf) {
        deposit_k(buf);
        deposit_v(buf);
    };

    float m = -INFINITY, sum = 0.0f;
    v16f o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    const int sub0 = split * SUB;                   // the wavefront's groups of 32 keys in a tile
    // its operands' places in LDS: of K for chunk 2 st + half (another chunk of 8 is 128 bytes further on, 32 rows are
    // a constant too), of V for the even and the odd row tiles of O^T
    constexpr int KA = KS < 4 ? KS : 4;
    int k_at[KA], v_at[2][SUB * 2];
#pragma unroll
    for (int st = 0; st < KA; ++st) k_at[st] = br * S::kK + k_chunk<CK>(sub0 * 32 + col, st * 2 + half) * 8;
#pragma unroll
    for (int par = 0; par < 2; ++par)
#pragma unroll
        for (int st = 0; st < SUB * 2; ++st)
            v_at[par][st] = SPLIT == 1 && par ? v_at[0][st ^ 2] : (v_chunk<CV>(par * 32 + col, (sub0 * 2 + st) * 2 + half) - par * 32 * CV) * 8;

    auto scores = [&](int buf, v16f (&x)[SUB]) {
        const _Float16 *kb = lds + buf * 2 * S::kK;
        constexpr int KB = D == 128 ? 1 : SUB;          // groups of 32 keys whose operands are requested together
#pragma unroll
        for (int k1 = 0; k1 < SUB; k1 += KB) {
            v8h f[KB][KS];
#pragma unroll
            for (int kt = 0; kt < KB; ++kt)
#pragma unroll
                for (int st = 0; st < KS; ++st)
                    f[kt][st] = *reinterpret_cast<const v8h *>(kb + k_at[st % KA] + ((k1 + kt) * 32 * CK + st / KA * 8) * 8);
#pragma unroll
            for (int kt = 0; kt < KB; ++kt) {
#pragma unroll
                for (int e = 0; e < 16; ++e) x[k1 + kt][e] = 0.0f;
#pragma unroll
                for (int st = 0; st < KS; ++st) x[k1 + kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[kt][st], q[st], x[k1 + kt], 0, 0, 0);
            }
        }
    };
    // One tile.  MASKED: some row may not see some key.
    auto compute = [&](auto masked, int tile, int buf, bool same) {
        constexpr bool MASKED = decltype(masked)::value;
        const int key0 = tile * S::kKeys + sub0 * 32;
        const _Float16 *vb = lds + S::kBufs * 2 * S::kK + buf * S::kV;
        v16f s[SUB];
        scores(buf, s);
        // in base 2 from here on: s * unit
        if (MOD) {
            if (cap > 0.0f) {
                const float in = p.scale / cap, out = cap * kLog2e;
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float y = s[kt][e] * in;
                        const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.0f * kLog2e)) + 1.0f);
                        if (cap > kCoarseCap) {
                            const float y2 = y * y;
                            const float series = y * __builtin_fmaf(y2, __builtin_fmaf(y2, __builtin_fmaf(y2, -17.0f / 315.0f, 2.0f / 15.0f),
                                                                                     -1.0f / 3.0f), 1.0f);
                            s[kt][e] = (fabsf(y) < 0.3f ? series : t) * out;
                        } else {
                            s[kt][e] = t * out;
                        }
                    }
            } else {
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[kt][e] *= p.scale * kLog2e;
            }
            if (a.slopes) {
                const float away = (float)(pos - key0 - 4 * half);
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        s[kt][e] = __builtin_fmaf(-slope, fabsf(away - (float)(kt * 32 + 8 * (e >> 2) + (e & 3))), s[kt][e]);
            }
        }
        if (MASKED) {
            const int left = opaque(limit - key0 - 4 * half);
            if (a.doc_k && !same) {
                const v4i *ids = reinterpret_cast<const v4i *>(doc_s[buf] + sub0 * 32 + opaque(4 * half));
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const v4i id = ids[kt * 8 + e4 * 2];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[kt][e4 * 4 + e] = kt * 32 + 8 * e4 + e < left && id[e] == doc ? s[kt][e4 * 4 + e] : -INFINITY;
                    }
            } else {
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[kt][e] = kt * 32 + 8 * (e >> 2) + (e & 3) < left ? s[kt][e] : -INFINITY;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
            for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, s[kt][e]), s[kt][e + 1]);
        top = halves_max(top) * unit;
        const bool raise = top > m + kSlack;            // (for each row by itself: no row depends on its neighbours)
        if (__any(raise)) {
            const float next = raise ? top : m;
            const float corr = __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.0f : next));
            m = next;
            sum *= corr;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= corr;
        }
        const float base = kLift - (m == -INFINITY ? 0.0f : m);
        constexpr int VB = DT > 2 ? 2 : DT;             // row tiles of O^T whose operands are requested together
        v8h vx[VB][SUB * 2], pr[SUB * 2];
        auto load_v = [&](int t1) {
#pragma unroll
            for (int t = 0; t < VB; ++t)
#pragma unroll
                for (int st = 0; st < SUB * 2; ++st)
                    vx[t][st] = *reinterpret_cast<const v8h *>(vb + v_at[(t1 + t) & 1][st] + (t1 + t) * 32 * CV * 8);
        };
        load_v(0);
#pragma unroll
        for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {           // the weights, operand B of O^T
                v2f x;
                x[0] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][e], unit, base));
                x[1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][e + 1], unit, base));
                const v2h y = __builtin_convertvector(x, v2h);
                sum = __builtin_amdgcn_fdot2(y, ones, sum, false);
                pr[kt * 2 + (e >> 3)][e & 7] = y[0];
                pr[kt * 2 + (e >> 3)][(e & 7) + 1] = y[1];
            }
#pragma unroll
        for (int t1 = 0; t1 < DT; t1 += VB) {
            if (t1 > 0) load_v(t1);
#pragma unroll
            for (int st = 0; st < SUB * 2; ++st)
#pragma unroll
                for (int t = 0; t < VB; ++t) o[t1 + t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vx[t][st], pr[st], o[t1 + t], 0, 0, 0);
        }
        int odd = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) odd |= odd_s[buf][i];
        if (__builtin_amdgcn_readfirstlane(odd)) {
            // values that are no finite numbers, to the rows that see them
            const int n = min(SUB * 32, nk - key0);
            for (int j = 0; j < n; ++j) {
                bool seen = key0 + j < limit;
                if (a.doc_k) seen = seen && doc_s[buf][sub0 * 32 + j] == doc;
                if (!__any(seen)) continue;
                const _Float16 *v = a.v + ((size_t)(k0 + key0 + j) * H + h) * D + opaque(4 * half);
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int d = t * 32 + 8 * (e >> 2) + (e & 3);
                        if (d >= D) continue;                       // (16 columns: rows of O^T that nobody stores)
                        const float x = (float)v[d];
                        if (seen && !(fabsf(x) <= 65504.0f)) o[t][e] += x;
                    }
            }
        }
    };

    // ---- the keys, in windows: all of them, or 64 tiles at a time of which those are taken whose documents can matter
    for (int from = 0; from < tiles; from += 64) {
        unsigned long long visit = 0, uniform = 0;
        if (a.doc_k) {
            constexpr int EACH = S::kKeys / kWaves;     // a lane looks at so many keys of tile from + l
            int lo = INT_MAX, hi = INT_MIN;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int id = a.doc_k[k0 + min((from + l) * S::kKeys + w * EACH + j, nk - 1)];
                lo = min(lo, id);
                hi = max(hi, id);
            }
            win_lo[w][l] = lo;
            win_hi[w][l] = hi;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                lo = min(lo, win_lo[i][l]);
                hi = max(hi, win_hi[i][l]);
            }
            visit = __ballot(from + l < tiles && hi >= doc_lo && lo <= doc_hi);
            uniform = __ballot(lo == hi && lo == doc_lo && lo == doc_hi);
            __syncthreads();                            // (the window's arrays are read before the next window's are written)
            if (!visit) continue;
        }
        const int stop = a.doc_k ? min(from + 64, tiles) : tiles;
        int tile = a.doc_k ? from + (int)__builtin_ctzll(visit) : 0, buf = 0;
        request(tile);
        deposit(0);
        __syncthreads();
        auto step = [&](auto masked) {
            int next = tile + 1;
            bool same = false;
            if (a.doc_k) {
                same = (uniform >> (tile - from)) & 1;
                visit &= visit - 1;
                next = visit ? from + (int)__builtin_ctzll(visit) : stop;
            }
            if (next < stop) request(next);
            if (!decltype(masked)::value || tile * S::kKeys + sub0 * 32 < most) compute(masked, tile, buf, same);
            if (S::kBufs == 1) __syncthreads();
            else buf ^= 1;
            if (next < stop) deposit(buf);
            __syncthreads();
            tile = next;
        };
        // (a loop for the tiles that every row sees whole, and one for the others: what differs between them inside one loop costs
        // copies of the accumulators)
        if (!a.doc_k) {
            while (tile < whole) step(std::false_type{});
        }
        while (tile < stop) step(std::true_type{});
        if (!a.doc_k) break;
    }

    // ---- merge: the wavefronts that shared keys, then the branches
    sum += __shfl_xor(sum, 32, 64);
    float *xchg = reinterpret_cast<float *>(lds);
    auto place = [&](int i, int t, int e) { return ((i * DT + t) * 16 + e) * 64 + l; };
    if (SPLIT > 1) {
        if (l < 32) {
            m_s[split][br][col] = m;
            sum_s[split][br][col] = sum;
        }
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < SPLIT; ++i) top = fmaxf(top, m_s[i][br][col]);
        top = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < SPLIT; ++i) sum += sum_s[i][br][col] * __builtin_amdgcn_exp2f(m_s[i][br][col] - top);
        const float f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                o[t][e] *= f;
                if (split > 0) xchg[place((split - 1) * 2 + br, t, e)] = o[t][e];
            }
        __syncthreads();
        if (split == 0) {
#pragma unroll
            for (int i = 0; i < SPLIT - 1; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[t][e] += xchg[place(i * 2 + br, t, e)];
        }
        __syncthreads();
    }
    const float f = (sum == 0.0f ? 0.0f : 0.5f / sum) * (br ? a.lambda : 1.0f);
    if (br == 1 && split == 0) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) xchg[place(group, t, e)] = o[t][e] * f;
    }
    __syncthreads();
    if (br == 1 || split > 0 || !real) return;
    _Float16 *out = a.out + ((size_t)(q0 + row) * H + h) * D;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int d = t * 32 + 8 * e4 + 4 * half;
            v4h x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (_Float16)(o[t][e4 * 4 + e] * f - xchg[place(group, t, e4 * 4 + e)]);
            if (d < D) *reinterpret_cast<v4h *>(out + d) = x;
        }
}

}  // namespace

hipError_t launch_diff_attn_prefill(const PrefillArgs &a, int d_h, hipStream_t st)
{
    PrefillParams p;
    p.a = a;
    p.scale = 1.0f / sqrtf((float)d_h);
    const bool mod = a.softcap > 0.0f || a.slopes;
    // fewer workgroups of 128 rows than the chip holds at a time: 32 rows each
    const bool few = (long long)(a.Tq / 128 + a.B) * a.n_heads < 512;
    hipError_t e = hipSuccess;
    auto go = [&](auto d, auto m, auto split) {
        constexpr int D = decltype(d)::value, SPLIT = decltype(split)::value;
        constexpr bool MOD = decltype(m)::value;
        using S = Shape<D, SPLIT>;
        static OncePerDevice once;
        e = allow_lds(once, (const void *)(prefill_attn_kernel<D, MOD, SPLIT>), S::kLds);
        p.slots = a.Tq / S::kRows + a.B;
        if (e == hipSuccess)
            hipLaunchKernelGGL((prefill_attn_kernel<D, MOD, SPLIT>), dim3((unsigned)p.slots * a.n_heads), dim3(kThreads), S::kLds, st, p);
    };
    auto variant = [&](auto d, auto m) {
        if (few) go(d, m, std::integral_constant<int, 4>{});
        else go(d, m, std::integral_constant<int, 1>{});
    };
    auto both = [&](auto d) {
        if (mod) variant(d, std::true_type{});
        else variant(d, std::false_type{});
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
