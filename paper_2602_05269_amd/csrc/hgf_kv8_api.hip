// C ABI of the paged 8-bit cache and of the attention over prompts: host-side argument validation and dispatch.
// Every check happens before the first HIP call, so the error paths run without a GPU.
#include "hgf_kv8.h"

#include <math.h>

using namespace hgf;

namespace hgf {

KvView kv_view(const hgf_kv8_cache &c, const hgf_kv8_pages &p, const int32_t *seqs)
{
    KvView v;
    v.k = c.k_codes;
    v.v = c.v_codes;
    v.ks = c.k_scale;
    v.vs = c.v_scale;
    v.table = p.table;
    v.lens = p.lens;
    v.seqs = seqs;
    v.n_pages = p.n_pages;
    v.n_seqs = p.n_seqs;
    v.max_pages = p.max_pages;
    v.n_heads = c.n_heads;
    v.page_log2 = __builtin_ctz((unsigned)p.page);
    return v;
}

}  // namespace hgf

namespace {

constexpr int kMaxTokens = 1 << 24, kMaxHeads = 1024, kMaxPages = 1 << 24;

bool aligned(const void *p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool head_ok(int n_heads, int d_h)
{
    return n_heads >= 1 && n_heads <= kMaxHeads && (d_h == 16 || d_h == 32 || d_h == 64 || d_h == 128);
}
bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128 || page == 256; }
bool cap_ok(float cap) { return cap == 0.0f || (cap >= 1e-20f && cap <= 1e20f); }      // (what is not a number is not)
bool number_ok(float v) { return !isnan(v) && !isinf(v); }

hgf_status check_pages(const hgf_kv8_pages *p)
{
    if (!p || !p->table || !p->lens || !p->refs) return HGF_ERR_NULL;
    if (p->n_pages < 1 || p->n_pages > kMaxPages || !page_ok(p->page) || p->n_seqs < 1 || p->n_seqs > kMaxSeqs ||
        p->max_pages < 1 || (long long)p->max_pages * p->page > kMaxTokens)
        return HGF_ERR_SHAPE;
    if (!aligned(p->table, 4) || !aligned(p->lens, 4) || !aligned(p->refs, 16)) return HGF_ERR_ALIGN;
    return HGF_OK;
}
hgf_status check_cache(const hgf_kv8_cache *c)
{
    if (!c || !c->k_codes || !c->k_scale || !c->v_codes || !c->v_scale) return HGF_ERR_NULL;
    if (c->n_pages < 1 || c->n_pages > kMaxPages || !page_ok(c->page) || !head_ok(c->n_heads, c->d_h)) return HGF_ERR_SHAPE;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
        return HGF_ERR_ALIGN;
    return HGF_OK;
}
hgf_status check_both(const hgf_kv8_cache *c, const hgf_kv8_pages *p, const int32_t *seqs, int B)
{
    hgf_status e = check_cache(c);
    if (e == HGF_OK) e = check_pages(p);
    if (e != HGF_OK) return e;
    if (c->n_pages != p->n_pages || c->page != p->page) return HGF_ERR_SHAPE;
    if (B < 1 || B > kMaxSeqs || (!seqs && B > p->n_seqs)) return HGF_ERR_SHAPE;
    if (!aligned(seqs, 4)) return HGF_ERR_ALIGN;
    return HGF_OK;
}
hgf_status from(hipError_t e) { return e == hipSuccess ? HGF_OK : HGF_ERR_DEVICE; }
hipStream_t st(void *stream) { return reinterpret_cast<hipStream_t>(stream); }

}  // namespace

extern "C" {

hgf_status hgf_diff_attention_prefill(const void *q_f16, const void *k_f16, const void *v_f16, const int32_t *cu_q,
                                      const int32_t *cu_k, int B, int Tq, int Tk, int n_heads, int d_h, float lambda,
                                      int causal, const int32_t *prefix, const int32_t *doc_q, const int32_t *doc_k,
                                      float softcap, const float *slopes, void *out_f16, void *stream)
{
    if (!q_f16 || !k_f16 || !v_f16 || !cu_q || !out_f16 || !doc_q != !doc_k) return HGF_ERR_NULL;
    if (B < 1 || B > kMaxSeqs || Tq < 1 || Tq >= kMaxTokens || Tk < 1 || Tk >= kMaxTokens || (!cu_k && Tk != Tq) ||
        !head_ok(n_heads, d_h) || !cap_ok(softcap) || !number_ok(lambda))
        return HGF_ERR_SHAPE;
    if (!aligned(q_f16, 16) || !aligned(k_f16, 16) || !aligned(v_f16, 16) || !aligned(out_f16, 16) || !aligned(cu_q, 4) ||
        !aligned(cu_k, 4) || !aligned(prefix, 4) || !aligned(doc_q, 4) || !aligned(doc_k, 4) || !aligned(slopes, 4))
        return HGF_ERR_ALIGN;
    PrefillArgs a;
    a.q = reinterpret_cast<const _Float16 *>(q_f16);
    a.k = reinterpret_cast<const _Float16 *>(k_f16);
    a.v = reinterpret_cast<const _Float16 *>(v_f16);
    a.cu_q = cu_q;
    a.cu_k = cu_k ? cu_k : cu_q;
    a.prefix = prefix;
    a.doc_q = doc_q;
    a.doc_k = doc_k;
    a.slopes = slopes;
    a.out = reinterpret_cast<_Float16 *>(out_f16);
    a.B = B;
    a.Tq = Tq;
    a.Tk = Tk;
    a.n_heads = n_heads;
    a.causal = causal != 0;
    a.lambda = lambda;
    a.softcap = softcap;
    return from(launch_diff_attn_prefill(a, d_h, st(stream)));
}

hgf_status hgf_kv8_pages_grow(const hgf_kv8_pages *pages, const int32_t *seqs, const int32_t *new_tokens, int n,
                              int32_t *ok_out, void *stream)
{
    if (!seqs || !new_tokens || !ok_out) return HGF_ERR_NULL;
    const hgf_status e = check_pages(pages);
    if (e != HGF_OK) return e;
    if (n < 1 || n > kMaxSeqs) return HGF_ERR_SHAPE;
    if (!aligned(seqs, 4) || !aligned(new_tokens, 4) || !aligned(ok_out, 4)) return HGF_ERR_ALIGN;
    return from(launch_pages_grow(*pages, seqs, new_tokens, n, ok_out, st(stream)));
}

hgf_status hgf_kv8_pages_fork(const hgf_kv8_pages *pages, const int32_t *src, const int32_t *dst, int n,
                              int32_t *pairs_out, int32_t *ok_out, void *stream)
{
    if (!src || !dst || !pairs_out || !ok_out) return HGF_ERR_NULL;
    const hgf_status e = check_pages(pages);
    if (e != HGF_OK) return e;
    if (n < 1 || n > kMaxSeqs) return HGF_ERR_SHAPE;
    if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(pairs_out, 4) || !aligned(ok_out, 4)) return HGF_ERR_ALIGN;
    return from(launch_pages_fork(*pages, src, dst, n, pairs_out, ok_out, st(stream)));
}

hgf_status hgf_kv8_pages_free(const hgf_kv8_pages *pages, const int32_t *seqs, int n, void *stream)
{
    if (!seqs) return HGF_ERR_NULL;
    const hgf_status e = check_pages(pages);
    if (e != HGF_OK) return e;
    if (n < 1 || n > kMaxSeqs) return HGF_ERR_SHAPE;
    if (!aligned(seqs, 4)) return HGF_ERR_ALIGN;
    return from(launch_pages_free(*pages, seqs, n, st(stream)));
}

hgf_status hgf_kv8_pages_compact(const hgf_kv8_pages *pages, int32_t *pairs_out, int32_t *count_out, int32_t *moved_out,
                                 void *stream)
{
    if (!pairs_out || !count_out || !moved_out) return HGF_ERR_NULL;
    const hgf_status e = check_pages(pages);
    if (e != HGF_OK) return e;
    if (!aligned(pairs_out, 4) || !aligned(count_out, 4) || !aligned(moved_out, 4)) return HGF_ERR_ALIGN;
    return from(launch_pages_compact(*pages, pairs_out, count_out, moved_out, st(stream)));
}

hgf_status hgf_kv8_copy_pages(const hgf_kv8_cache *cache, const int32_t *pairs, const int32_t *count, int n, void *stream)
{
    if (!pairs) return HGF_ERR_NULL;
    const hgf_status e = check_cache(cache);
    if (e != HGF_OK) return e;
    if (n < 1 || n > kMaxPages) return HGF_ERR_SHAPE;
    if (!aligned(pairs, 4) || !aligned(count, 4)) return HGF_ERR_ALIGN;
    return from(launch_kv8_copy_pages(*cache, pairs, count, n, st(stream)));
}

hgf_status hgf_kv8_append(const void *k_f16, const void *v_f16, const hgf_kv8_cache *cache, const hgf_kv8_pages *pages,
                          const int32_t *seqs, const int32_t *cu_new, int B, int T, void *stream)
{
    if (!k_f16 || !v_f16) return HGF_ERR_NULL;
    const hgf_status e = check_both(cache, pages, seqs, B);
    if (e != HGF_OK) return e;
    if (T < 1 || T >= kMaxTokens || (!cu_new && T != B)) return HGF_ERR_SHAPE;
    if (!aligned(k_f16, 16) || !aligned(v_f16, 16) || !aligned(cu_new, 4)) return HGF_ERR_ALIGN;
    return from(launch_kv8_append(k_f16, v_f16, kv_view(*cache, *pages, seqs), cache->d_h, cu_new, B, T, st(stream)));
}

hgf_status hgf_kv8_gather(const hgf_kv8_cache *cache, const hgf_kv8_pages *pages, const int32_t *seqs, const int32_t *cu,
                          int B, int T, void *k_f16, void *v_f16, void *stream)
{
    if (!k_f16 || !v_f16 || !cu) return HGF_ERR_NULL;
    const hgf_status e = check_both(cache, pages, seqs, B);
    if (e != HGF_OK) return e;
    if (T < 1 || T >= kMaxTokens) return HGF_ERR_SHAPE;
    if (!aligned(k_f16, 16) || !aligned(v_f16, 16) || !aligned(cu, 4)) return HGF_ERR_ALIGN;
    return from(launch_kv8_gather(kv_view(*cache, *pages, seqs), cache->d_h, cu, B, T, k_f16, v_f16, st(stream)));
}

size_t hgf_diff_attention_kv8_workspace_bytes(int B, const hgf_kv8_pages *pages, int n_heads, int d_h)
{
    if (!pages || B < 1 || B > kMaxSeqs || !head_ok(n_heads, d_h) || !page_ok(pages->page) || pages->max_pages < 1 ||
        (long long)pages->max_pages * pages->page > kMaxTokens)
        return 0;
    return diff_attn_kv8_workspace_bytes(B, (long long)pages->max_pages * pages->page, n_heads, d_h);
}

hgf_status hgf_diff_attention_decode_kv8(const void *q_f16, const hgf_kv8_cache *cache, const hgf_kv8_pages *pages,
                                         const int32_t *seqs, int B, float lambda, float softcap, const float *slopes,
                                         void *out_f16, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q_f16 || !out_f16) return HGF_ERR_NULL;
    const hgf_status e = check_both(cache, pages, seqs, B);
    if (e != HGF_OK) return e;
    if (!cap_ok(softcap) || !number_ok(lambda)) return HGF_ERR_SHAPE;
    if (!aligned(q_f16, 16) || !aligned(out_f16, 2) || !aligned(slopes, 4)) return HGF_ERR_ALIGN;
    const size_t need = diff_attn_kv8_workspace_bytes(B, (long long)pages->max_pages * pages->page, cache->n_heads, cache->d_h);
    if (need > 0 && (!workspace || workspace_bytes < need)) return HGF_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return HGF_ERR_ALIGN;
    return from(launch_diff_attn_kv8(q_f16, kv_view(*cache, *pages, seqs), B, cache->d_h, lambda, softcap, slopes, out_f16,
                                     workspace, st(stream)));
}

}  // extern "C"
