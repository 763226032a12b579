// Differential attention over prompts: many query rows, ragged batches, capped or biased scores, masks.
//
//   out = (softmax(s1) V - lambda softmax(s2) V) / 2, both branches in one pass over the keys with running maxima and sums.
//
// A workgroup of eight wavefronts holds 128 query rows of one head and sequence, a wavefront 32 of them for one of the branches, and
// takes the keys 64 at a time: K1, K2 and V of a tile go straight into LDS, three tiles at a time, requested two ahead.  All
// products are computed transposed, S^T = K Q^T and O^T = V^T P^T on the 32x32x16 fp16 matrix instruction, so that
// a lane owns one query: its maximum, sum and rescaling are registers of the lane (one exchange between the halves of the
// wavefront), and the 8 weights of a step that a lane holds after S^T are the ones it has to supply for O^T if V's
// keys are taken in the order in which the accumulator's rows lie (4 h .. 4 h + 3 and 8 + 4 h .. for half h): P never
// moves.  V is transposed by the LDS reads that fetch it.
// Few rows would leave most of the chip idle: then (SPLIT) a workgroup holds 64 rows, or 32 and takes 128 keys at a time, and its
// wavefronts share the keys of a tile; they are merged at the end.
// Weights are relative to the running maximum in base 2 and carried 2^7 larger, so that fp16 holds them down to
// 2^-31; a row's maximum is only raised when a tile exceeds it by 2^8 (which the factor leaves room for), which spares
// most rescalings.  fp32: scores, weights before rounding, sums, outputs.  The sum adds up the rounded weights.
// A lane adds its keys up one step after the other: over four million random keys outputs stay within their rounding to fp16, over a
// million equal ones behind a first key that outweighs them all together they are off by up to 1.4e-3.
// The weights' rounding to fp16 leaves outputs 2.2e-4 to 2.6e-4 of their size (root mean square) off the result in 64 bits, of
// which rounding the outputs themselves is 2.1e-4.  With what the rounding leaves as a second product that is all there is, but 4096
// rows of 32 heads of 64 columns take 267 us in place of 182, three turns of 128 columns 206 in place of 177.
// Masks are one comparison per element, key < limit of the row, and a comparison of document numbers where documents are
// given, both only in tiles that need them; tiles whose document numbers lie outside those of the rows are not
// read.  What a row does not see has weight 0; values of V that are no finite numbers are taken out of the tile and
// added to the rows that see them (0 * inf would reach the others).
// Bound by vector instructions, at the clock that the chip's power limit leaves: of the 340 000 clocks of a pass of 4096 rows, 32 heads
// of 64 columns, the vector units issue in 237 000 (12 instructions to a matrix instruction) and the matrix cores are busy in 132 000,
// at 1.74 GHz; with two wavefronts to a SIMD in place of four it was 404 000 clocks at 1.97 GHz, and taking out any part (staging,
// matrix instructions, exponentials) saves about that part's time alone.  181 to 195 us by the card, 758 TFLOP/s (770 without
// causality, 865 with 128 columns), against 1350 of a plain matrix product of 8192.
#include "hgf_kv8.h"

#include <limits.h>
#include <type_traits>

namespace hgf {

namespace {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void *lds_ptr_t;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr float kLift = 7.0f, kSlack = 8.0f;
// From here on 1 - 2 / (e^2y + 1) is too coarse a tanh near 0: its error, up to 2^-22 of the cap however small the score, passes
// 1.2e-4, a quarter of what rounding a weight to fp16 costs.
constexpr float kCoarseCap = 512.0f;

struct PrefillParams {
    PrefillArgs a;
    float scale;
    int slots, layer;
};

// Sizes of one variant.
template <int D, int SPLIT>
struct Shape {
    static constexpr int kRows = 128 / SPLIT, kGroups = 4 / SPLIT;         // rows, and groups of 32 of them
    static constexpr int kKeys = SPLIT == 1 ? 64 : 32 * SPLIT;
    static constexpr int kSub = kKeys / 32 / SPLIT;             // groups of 32 keys per wavefront and tile, and of them worked on
    static constexpr int kStep = D == 64 ? 1 : kSub;            // together (64 columns: two at a time leave room for half the wavefronts)
    static constexpr int kChunks = D / 8;                       // 16-byte chunks of a row of K or V
    static constexpr int kK = kKeys * D, kHalves = 3 * kK;      // a tile: K1, K2, V
    static constexpr int kTileT = (D + 31) / 32;                // row tiles of O^T
    // outputs on their way between wavefronts, in the tiles' place
    static constexpr size_t kMerge = (size_t)(SPLIT == 1 ? 4 : 2 * (SPLIT - 1) * kGroups) * kTileT * 4096;
    static constexpr size_t kTiles = (size_t)3 * kHalves * 2;
    static constexpr size_t kLds = kTiles > kMerge ? kTiles : kMerge;
};

// Where a 16-byte chunk of a row of K and of V lies in the row, so that the rows that are read together lie in different
// banks (its own inverse).
template <int C>
__device__ inline int k_swap(int row, int c) { return C >= 8 ? c ^ (row & 7) : C == 4 ? c ^ ((row >> 1) & 3) : c ^ ((row >> 2) & 1); }
template <int C>
__device__ inline int v_swap(int row, int c) { return C >= 8 ? c ^ ((row & 3) << 1) : C == 4 ? c ^ (row & 2) : c; }

// A value that the compiler does not see through: what rare paths compute from it is computed there, instead of being kept
// in registers across the loop.
__device__ inline int opaque(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
// 64 x 16 bytes from memory straight into LDS, in flight until a wait on vmcnt.  (In assembly because with the builtin the compiler
// waits for everything in flight before the transposing LDS reads, whichever buffer they read.  Nothing comes back in
// registers, and the kernel's own waits are the only ones that are needed.  Five wait states lie between whatever stands in front and
// the load: that many the hardware wants after a vector instruction that wrote the descriptor's registers, as one does that
// fetches them from where they were spilled; the compiler keeps them for its own loads only.)
__device__ inline void load_to_lds(v4u rsrc, unsigned lds_byte, unsigned lane_off)
{
    unsigned kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds_byte), "v"(lane_off), "s"(rsrc) : "memory");
}
__device__ inline void load4_to_lds(v4u rsrc, unsigned lds_byte, unsigned lane_off)      // 64 x 4 bytes
{
    unsigned kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dword %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds_byte), "v"(lane_off), "s"(rsrc) : "memory");
}
__device__ inline v4u rsrc_words(const void *base, unsigned bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    return v4u{(unsigned)a, (unsigned)(a >> 32) & 0xffffu, bytes, 0x00020000u};
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
    constexpr int KS = D / 16, DT = S::kTileT, SUB = S::kStep, C = S::kChunks;
    constexpr int KI = 2 * S::kKeys * C / 64, VI = S::kKeys * C / 64;           // KiB of K1 and K2, and of V, in a tile
    constexpr int KP = KI > kWaves ? KI / kWaves : 1, VP = VI > kWaves ? VI / kWaves : 1;       // of them per wavefront
    extern __shared__ __align__(16) _Float16 lds[];
    __shared__ int odd_s[3], doc_s[3][S::kKeys];
    __shared__ int most_s[kWaves], least_s[kWaves], lo_s[kWaves], hi_s[kWaves], win_lo[kWaves][64], win_hi[kWaves][64];
    __shared__ float m_s[SPLIT][2][S::kGroups][32], sum_s[SPLIT][2][S::kGroups][32];
    const PrefillArgs &a = p.a;
    const int H = a.n_heads, h = blockIdx.x % H;
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = l >> 5, col = l & 31;
    const int br = w >> 2, group = (w & 3) % S::kGroups, split = (w & 3) / S::kGroups;

    // ---- which rows.  Workgroups that see the most keys come first: of up to 64 sequences those with the most keys,
    // of a sequence the last rows.
    const int slot = blockIdx.y * p.layer + blockIdx.x / H;
    int b, q0, nq, k0, nk, first;
    if (a.B <= 64) {
        int fq, n, fk, m;
        clipped_rows(a.cu_q, min(l, a.B - 1), a.Tq, fq, n);
        clipped_rows(a.cu_k, min(l, a.B - 1), a.Tk, fk, m);
        const int mine = l < a.B ? (n + S::kRows - 1) / S::kRows : 0;
        int before = 0;                             // tiles of the sequences that come before the lane's
        for (int j = 0; j < a.B; ++j) {
            const int mj = __builtin_amdgcn_readlane(m, j);
            before += mj > m || (mj == m && j < l) ? __builtin_amdgcn_readlane(mine, j) : 0;
        }
        const unsigned long long at = __ballot(slot >= before && slot < before + mine);
        if (!at) return;
        b = __builtin_ctzll(at);
        q0 = __builtin_amdgcn_readlane(fq, b);
        nq = __builtin_amdgcn_readlane(n, b);
        k0 = __builtin_amdgcn_readlane(fk, b);
        nk = __builtin_amdgcn_readlane(m, b);
        first = (__builtin_amdgcn_readlane(before + mine, b) - 1 - slot) * S::kRows;
    } else {
        // (the slots of sequence b begin at cu_q[b] / kRows + b)
        if (slot >= p.slots) return;
        constexpr int SHIFT = S::kRows == 128 ? 7 : S::kRows == 64 ? 6 : 5;
        b = slot_entry<SHIFT, 1>(a.cu_q, a.B, a.Tq, p.slots - 1 - slot, q0, nq);
        clipped_rows(a.cu_k, b, a.Tk, k0, nk);
        first = (p.slots - 1 - slot - (q0 >> SHIFT) - b) * S::kRows;
    }
    if (first < 0 || first >= nq) return;
    const int row = first + group * 32 + col;       // the lane's query
    const bool real = row < nq;
    // the queries, operand B of S^T (requested before anything else is looked up)
    v8h q[KS];
    {
        const _Float16 *src = a.q + ((size_t)(q0 + min(row, nq - 1)) * 2 * H + br * H + h) * D + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8h *>(src + s * 16);
    }
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
    int tiles, whole;                               // tiles that some row sees, that all rows see whole
    int doc_lo, doc_hi, wave_lo, wave_hi;           // document numbers of all rows, and of the wavefront's
    {
        int lo = counts ? doc : INT_MAX, hi = counts ? doc : -1;
        if (a.doc_q) {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                lo = min(lo, __shfl_xor(lo, o, 64));
                hi = max(hi, __shfl_xor(hi, o, 64));
            }
        }
        wave_lo = lo;
        wave_hi = hi;
        if (tid < 3) odd_s[tid] = -1;
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

    const float cap = a.softcap, cap_in = cap > 0.0f ? p.scale / cap * (2.0f * kLog2e) : 0.0f, cap_out = cap * kLog2e;
    float slope = 0.0f;
    if (MOD && a.slopes) slope = a.slopes[br * H + h] * kLog2e;
    const float unit = MOD ? 1.0f : p.scale * kLog2e;
    const v2h ones = {(_Float16)1.0f, (_Float16)1.0f};

    // ---- tiles on their way, straight from memory into LDS, two tiles ahead.  A tile's rows are read through a descriptor
    // that ends where the sequence does: rows behind it are zeros, and what a lane adds to the tile's address does not change
    // from tile to tile.  (All of it is in the lane's offset: that is what the descriptor's end is held against.)
    const unsigned k_row = (unsigned)H * D * 4, v_row = (unsigned)H * D * 2;
    auto rows_of = [&](const _Float16 *base, unsigned row_bytes, int key0) {
        return rsrc_words(reinterpret_cast<const char *>(base) + (size_t)(k0 + key0) * row_bytes, (unsigned)min(nk - key0, S::kKeys) * row_bytes);
    };
    // KiB i * kWaves + w of a tile, 64 chunks, is the wavefront's; further ones are a constant number of rows (or the other K) on
    const unsigned lds_at = (unsigned)reinterpret_cast<uintptr_t>((lds_ptr_t)lds);
    const int chunk = w * 64 + l;
    const int k_in = chunk % (S::kKeys * C);
    const unsigned k_off = (unsigned)(k_in / C) * k_row + (unsigned)((chunk / (S::kKeys * C) * H + h) * D + k_swap<C>(k_in / C, k_in % C) * 8) * 2;
    const unsigned v_off = (unsigned)(chunk / C) * v_row + (unsigned)(h * D + v_swap<C>(chunk / C, chunk % C) * 8) * 2;
    const unsigned doc_at = (unsigned)reinterpret_cast<uintptr_t>((lds_ptr_t)doc_s);
    const bool has_k = KI >= kWaves || w < KI, has_v = VI >= kWaves || w < VI, has_doc = a.doc_k && w < S::kKeys / 64;
    static_assert(S::kKeys / 64 <= VI && VI <= KI, "who has documents has V, and who has V has K");
    auto request = [&](int tile, int buf) {
        const unsigned kb = lds_at + buf * S::kHalves * 2 + w * 1024, vb = kb + 4 * S::kK;
        if (has_k) {
            const v4u r = rows_of(a.k, k_row, tile * S::kKeys);
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                constexpr int HALF = KI / 2;
                const unsigned more = (unsigned)(i * kWaves % HALF * 64 / C) * k_row + (unsigned)(i * kWaves / HALF * H * D) * 2;
                load_to_lds(r, kb + i * kWaves * 1024, k_off + more);
            }
        }
        if (has_v) {
            const v4u r = rows_of(a.v, v_row, tile * S::kKeys);
#pragma unroll
            for (int i = 0; i < VP; ++i)
                load_to_lds(r, vb + i * kWaves * 1024, v_off + (unsigned)(i * kWaves * 64 / C) * v_row);
        }
        if (has_doc) {                              // (behind the sequence zeros: no row sees those keys)
            const int key0 = tile * S::kKeys;
            load4_to_lds(rsrc_words(a.doc_k + k0 + key0, (unsigned)min(nk - key0, S::kKeys) * 4), doc_at + (buf * S::kKeys + w * 64) * 4,
                         (unsigned)tid * 4);
        }
    };
    // The wavefront's part of a tile has landed (`behind`: one more tile has been requested since).  It looks its V through:
    // values that are no finite numbers become zeros there, and the tile is marked.
    auto settle = [&](int tile, int buf, bool behind) {
        if (behind && has_doc) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KP + VP + 1) : "memory");
        else if (behind && has_v) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KP + VP) : "memory");
        else if (behind && has_k) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KP) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (has_v) {
            v4u *mine = reinterpret_cast<v4u *>(lds + buf * S::kHalves + 2 * S::kK) + w * 64 + l;
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                v4u v = mine[i * kWaves * 64];
                v2h x = {(_Float16)0.0f, (_Float16)0.0f};           // 0 * v: what is no finite number leaves a NaN
                const v2h zero = x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x = __builtin_elementwise_fma(__builtin_bit_cast(v2h, (uint32_t)v[j]), zero, x);
                if ((__builtin_bit_cast(uint32_t, x) & 0x7fff7fffu) != 0) {
                    odd_s[buf] = tile;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t y = v[j];
                        if ((y & 0x7c00u) == 0x7c00u) y &= 0xffff0000u;
                        if ((y & 0x7c000000u) == 0x7c000000u) y &= 0x0000ffffu;
                        v[j] = y;
                    }
                    mine[i * kWaves * 64] = v;
                }
            }
        }
    };

    if (!a.doc_k) {                                 // (with documents it is not known yet which tiles)
        if (tiles > 0) request(0, 0);
        if (tiles > 1) request(1, 1);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));     // (they are waited for here, not in the loop)

    float m = -INFINITY, sum = 0.0f;
    v16f o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    // its operands' places in LDS: of K for chunk 2 st + half (another eight chunks are 128 bytes further on, 32 rows
    // are a constant too); of V for the even and odd row tiles of O^T, where lane j of 16 asks for 4 columns of key j / 4, and gets
    // 4 keys of column j
    constexpr int KA = KS < 4 ? KS : 4;
    int k_at[KA], v_at[2];
#pragma unroll
    for (int st = 0; st < KA; ++st) k_at[st] = br * S::kK + col * D + k_swap<C>(col, st * 2 + half) * 8;
    {
        const int key = 4 * half + (l >> 2 & 3), c4 = D < 32 ? l & 3 : (l >> 4 & 1) * 4 + (l & 3);  // quad of columns
#pragma unroll
        for (int par = 0; par < 2; ++par) v_at[par] = key * D + v_swap<C>(key, (D < 64 ? 0 : par * 4) + c4 / 2) * 8 + (c4 & 1) * 4;
    }
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s *lds_v4s_t;

    auto scores = [&](const _Float16 *kb, v16f (&x)[SUB]) {
        constexpr int KB = D == 128 ? 1 : SUB;          // groups of 32 keys whose operands are requested together
#pragma unroll
        for (int k1 = 0; k1 < SUB; k1 += KB) {
            v8h f[KB][KS];
#pragma unroll
            for (int kt = 0; kt < KB; ++kt)
#pragma unroll
                for (int st = 0; st < KS; ++st)
                    f[kt][st] = *reinterpret_cast<const v8h *>(kb + k_at[st % KA] + (k1 + kt) * 32 * D + st / KA * 64);
#pragma unroll
            for (int kt = 0; kt < KB; ++kt) {
#pragma unroll
                for (int e = 0; e < 16; ++e) x[k1 + kt][e] = 0.0f;
#pragma unroll
                for (int st = 0; st < KS; ++st) x[k1 + kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[kt][st], q[st], x[k1 + kt], 0, 0, 0);
            }
        }
    };
    // The keys of a tile from group sub0 on.  MASKED: some row may not see some key.
    auto compute = [&](auto masked, int tile, int sub0, int buf, bool same, int odd_tile) {
        constexpr bool MASKED = decltype(masked)::value;
        const int key0 = tile * S::kKeys + sub0 * 32;
        _Float16 *kb = lds + buf * S::kHalves + sub0 * 32 * D, *vb = kb + 2 * S::kK;
        v16f s[SUB];
        scores(kb, s);
        // in base 2 from here on: s * unit
        if (MOD) {
            if (cap > 0.0f) {
                // cap tanh(x / cap) = cap - 2 cap / (e^(2 x / cap) + 1)
#pragma unroll
                for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float y = s[kt][e] * cap_in;          // 2 x / cap, in base 2
                        const float t = __builtin_fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y) + 1.0f), -2.0f * cap_out, cap_out);
                        if (cap > kCoarseCap) {
                            const float z = y * (0.5f / kLog2e);
                            s[kt][e] = fabsf(z) < kTanhSeries ? tanh_series(z) * cap_out : t;
                        } else {
                            s[kt][e] = t;
                        }
                    }
            }
            const float by = cap > 0.0f ? 1.0f : p.scale * kLog2e;
            const float away = (float)(pos - key0 - 4 * half);
#pragma unroll
            for (int kt = 0; kt < SUB; ++kt)
#pragma unroll
                for (int e = 0; e < 16; ++e)                        // (without slopes: slope is 0)
                    s[kt][e] = __builtin_fmaf(s[kt][e], by, -slope * fabsf(away - (float)(kt * 32 + 8 * (e >> 2) + (e & 3))));
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
                for (int st = 0; st < SUB * 2; ++st) {
                    _Float16 *at = vb + v_at[(t1 + t) & 1] + (t1 + t) / 2 * 64 + st * 16 * D;
                    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)at);
                    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)(at + 8 * D));
                    vx[t][st] = __builtin_bit_cast(v8h, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
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
        if (odd_tile == tile) {
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
        unsigned long long visit = 0, mine = 0, uniform = 0;        // tiles of the window: to be read, for this wavefront, of one document
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
            mine = __ballot(hi >= wave_lo && lo <= wave_hi);
            uniform = __ballot(lo == hi && lo == wave_lo && lo == wave_hi);
            __syncthreads();                            // (the window's arrays are read before the next window's are written)
            if (!visit) continue;
        }
        const int stop = a.doc_k ? min(from + 64, tiles) : tiles;
        auto after = [&](int t) {                       // the tile that follows, or `stop`
            if (!a.doc_k) return min(t + 1, stop);
            const unsigned long long rest = t - from >= 63 ? 0 : visit >> (t - from + 1) << (t - from + 1);
            return rest ? from + (int)__builtin_ctzll(rest) : stop;
        };
        int tile = a.doc_k ? from + (int)__builtin_ctzll(visit) : 0, next = after(tile), buf = 0;
        if (a.doc_k) {
            request(tile, 0);
            if (next < stop) request(next, 1);
        }
        settle(tile, 0, next < stop);
        __syncthreads();
        auto step = [&](auto masked) {
            const int third = next < stop ? after(next) : stop, ahead = buf == 2 ? 0 : buf + 1;
            if (third < stop) request(third, buf == 0 ? 2 : buf - 1);           // (where the tile before this one was)
            const bool same = a.doc_k && ((uniform >> (tile - from)) & 1), skip = a.doc_k && !((mine >> (tile - from)) & 1);
            const int odd_tile = __builtin_amdgcn_readfirstlane(odd_s[buf]);
#pragma unroll
            for (int i = 0; i < S::kSub; i += SUB) {
                const int sub0 = split * S::kSub + i;
                if (!decltype(masked)::value || (!skip && tile * S::kKeys + sub0 * 32 < most)) compute(masked, tile, sub0, buf, same, odd_tile);
            }
            if (next < stop) settle(next, ahead, third < stop);
            __syncthreads();
            buf = ahead;
            tile = next;
            next = third;
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
            m_s[split][br][group][col] = m;
            sum_s[split][br][group][col] = sum;
        }
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < SPLIT; ++i) top = fmaxf(top, m_s[i][br][group][col]);
        top = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < SPLIT; ++i) sum += sum_s[i][br][group][col] * __builtin_amdgcn_exp2f(m_s[i][br][group][col] - top);
        const float f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                o[t][e] *= f;
                if (split > 0) xchg[place(((split - 1) * 2 + br) * S::kGroups + group, t, e)] = o[t][e];
            }
        __syncthreads();
        if (split == 0) {
#pragma unroll
            for (int i = 0; i < SPLIT - 1; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[t][e] += xchg[place((i * 2 + br) * S::kGroups + group, t, e)];
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
    // Rows per workgroup.  128 need the fewest reads, but few of them leave compute units idle, and of causal ones, one or two to a
    // unit, the last rows' decide: then 64 rows each, and 32 where even those are few.  Where all rows see about as many
    // keys (not causal, or behind many earlier keys) there is nothing to level out, and 128 are the faster ones from 200 workgroups
    // on.  (us, 128 / 64 / 32 rows: 32 columns, 1000 rows of 16 heads - / 16.0 / 12.4, of 32 21.8 / 18.4 / 20.4, 8000 of 5 134 / 104 / 106,
    // of 8 151 / 143 / 158, 2000 of 40 53 / 60 / -; 64 columns, 1000 of 16 27.3 / 20.8 / 20.3, of 20 - / 21.7 / 28.1, 2000 of 16 49.5 / 39.0 /
    // 55.9, of 20 52.5 / 40.8 / 71, of 32 58.9 / 59.7 / 110, 8 times 300 of 16 17.7 / 19.6 / -, 2000 of 16 not causal 50.4 / 54.0 / -, behind
    // 8000 226 / 223 / -; 128 columns, for whose tiles of 128 keys LDS has no room three times, 2000 of 16 77 / 69, of 32 98 / 132, 1900
    // rows and 7600 keys, 16 heads, 177 / 197.)
    const long long wide = (long long)(a.Tq / 128 + a.B) * a.n_heads;       // workgroups of 128 rows
    const bool alike = !a.causal || a.Tk / 2 > a.Tq;
    int split;
    if (d_h == 128) split = wide < (a.Tk / 2 > a.Tq ? 200 : 300) ? 2 : 1;
    else split = wide < (d_h == 64 ? 130 : alike ? 200 : 256) ? 4 : wide < (alike ? 200 : 400) ? 2 : 1;
    hipError_t e = hipSuccess;
    auto go = [&](auto d, auto m, auto s) {
        constexpr int D = decltype(d)::value, SPLIT = decltype(s)::value;
        constexpr bool MOD = decltype(m)::value;
        using S = Shape<D, SPLIT>;
        static OncePerDevice once;
        e = allow_lds(once, (const void *)(prefill_attn_kernel<D, MOD, SPLIT>), S::kLds);
        p.slots = a.Tq / S::kRows + a.B;
        // (one dimension of a grid, unless many heads of many sequences are more threads than it may have: heads, slots and layers
        // as three dimensions took 187 us where one takes 181)
        const int most = (int)(((1u << 31) / kThreads) / a.n_heads);
        p.layer = p.slots < most ? p.slots : most;
        const dim3 grid((unsigned)(p.layer * a.n_heads), (p.slots + p.layer - 1) / p.layer);
        if (e == hipSuccess)
            hipLaunchKernelGGL((prefill_attn_kernel<D, MOD, SPLIT>), grid, dim3(kThreads), S::kLds, st, p);
    };
    auto variant = [&](auto d, auto m) {
        if (split == 1) go(d, m, std::integral_constant<int, 1>{});
        else if (split == 2) go(d, m, std::integral_constant<int, 2>{});
        else if constexpr (decltype(d)::value < 128) go(d, m, std::integral_constant<int, 4>{});
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
