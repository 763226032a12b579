"""CPU-only checks of the entry points of the 8-bit cache and the attention over prompts: every argument error is caught
on the host, before anything is launched (fake addresses, never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2602_05269_amd import binding as hb

BIG = 1 << 40


def _pages(**kw):
    d = dict(n_pages=8, page=64, n_seqs=4, max_pages=4, table=0x1000, lens=0x2000, refs=0x3000)
    d.update(kw)
    return hb.hgf_kv8_pages(**d)


def _cache(**kw):
    d = dict(n_pages=8, page=64, n_heads=2, d_h=64, k_codes=0x1000, k_scale=0x2000, v_codes=0x3000, v_scale=0x4000)
    d.update(kw)
    return hb.hgf_kv8_cache(**d)


def _prefill(**kw):
    d = dict(q=0x100, k=0x200, v=0x300, cu_q=0x400, cu_k=None, B=1, Tq=8, Tk=8, H=2, d=64, lam=0.5, causal=1, prefix=None, doc_q=None,
             doc_k=None, cap=0.0, slopes=None, out=0x500, stream=None)
    d.update(kw)
    return hb.lib().hgf_diff_attention_prefill(*d.values())


def test_prefill_refusals():
    for name in ("q", "k", "v", "cu_q", "out"):
        assert _prefill(**{name: None}) == 1
    assert _prefill(doc_q=0x600) == 1 and _prefill(doc_k=0x600) == 1
    for bad in (dict(B=0), dict(B=16385), dict(Tq=0), dict(Tk=0), dict(Tq=1 << 24, cu_k=0x700), dict(Tk=9), dict(H=0), dict(H=1025), dict(d=8),
                dict(d=48), dict(d=256), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-21), dict(cap=2e20), dict(lam=float("nan"))):
        assert _prefill(**bad) == 2, bad
    for name in ("q", "k", "v", "out"):
        assert _prefill(**{name: 0x108}) == 3
    assert _prefill(cu_q=0x402) == 3 and _prefill(slopes=0x602) == 3 and _prefill(prefix=0x601) == 3


@pytest.mark.parametrize("bad,status", [
    (dict(table=None), 1), (dict(lens=None), 1), (dict(refs=None), 1), (dict(n_pages=0), 2), (dict(n_pages=(1 << 24) + 1), 2), (dict(page=24), 2),
    (dict(page=512), 2), (dict(n_seqs=0), 2), (dict(n_seqs=16385), 2), (dict(max_pages=0), 2), (dict(max_pages=1 << 19), 2), (dict(refs=0x3004), 3),
    (dict(table=0x1002), 3)])
def test_page_operations_refuse_bad_tables(bad, status):
    L, p = hb.lib(), ctypes.byref(_pages(**bad))
    assert L.hgf_kv8_pages_grow(p, 0x100, 0x200, 1, 0x300, None) == status
    assert L.hgf_kv8_pages_fork(p, 0x100, 0x200, 1, 0x300, 0x400, None) == status
    assert L.hgf_kv8_pages_free(p, 0x100, 1, None) == status
    assert L.hgf_kv8_pages_compact(p, 0x100, 0x200, 0x300, None) == status
    c = ctypes.byref(_cache())
    assert L.hgf_kv8_append(0x100, 0x100, c, p, None, None, 1, 1, None) == status
    assert L.hgf_kv8_gather(c, p, None, 0x100, 1, 1, 0x100, 0x100, None) == status
    assert L.hgf_diff_attention_decode_kv8(0x100, c, p, None, 1, 0.5, 0.0, None, 0x100, 0x100, BIG, None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(k_codes=None), 1), (dict(v_scale=None), 1), (dict(n_pages=0), 2), (dict(page=17), 2), (dict(n_heads=0), 2), (dict(d_h=8), 2),
    (dict(d_h=24), 2), (dict(k_codes=0x1008), 3), (dict(v_codes=0x1004), 3), (dict(k_scale=0x2001), 3)])
def test_cache_operations_refuse_bad_caches(bad, status):
    L, c, p = hb.lib(), ctypes.byref(_cache(**bad)), ctypes.byref(_pages())
    assert L.hgf_kv8_copy_pages(c, 0x100, None, 1, None) == status
    assert L.hgf_kv8_append(0x100, 0x100, c, p, None, None, 1, 1, None) == status
    assert L.hgf_kv8_gather(c, p, None, 0x100, 1, 1, 0x100, 0x100, None) == status
    assert L.hgf_diff_attention_decode_kv8(0x100, c, p, None, 1, 0.5, 0.0, None, 0x100, 0x100, BIG, None) == status


def test_cache_and_pages_have_to_fit_each_other_and_the_batch():
    L = hb.lib()
    c, p = _cache(), _pages()
    dec = lambda c=c, p=p, q=0x100, seqs=None, B=1, lam=0.5, cap=0.0, out=0x100, ws=0x100, n=BIG: L.hgf_diff_attention_decode_kv8(
        q, ctypes.byref(c), ctypes.byref(p), seqs, B, lam, cap, None, out, ws, n, None)
    assert dec(p=_pages(n_pages=9)) == 2 and dec(p=_pages(page=32)) == 2
    assert dec(q=None) == 1 and dec(out=None) == 1 and dec(B=0) == 2 and dec(B=5) == 2 and dec(B=16385, seqs=0x100) == 2
    assert dec(cap=-1.0) == 2 and dec(lam=float("inf")) == 2 and dec(q=0x102) == 3 and dec(out=0x101) == 3 and dec(seqs=0x101) == 3
    need = L.hgf_diff_attention_kv8_workspace_bytes(1, ctypes.byref(_pages(max_pages=64)), 2, 64)
    assert need > 0
    big = _pages(max_pages=64)
    assert dec(p=big, ws=None) == 5 and dec(p=big, n=need - 1) == 5 and dec(p=big, ws=0x108) == 3
    # one part per sequence needs no workspace
    assert L.hgf_diff_attention_kv8_workspace_bytes(1, ctypes.byref(_pages(page=16)), 2, 64) == 0
    for args in ((0, p, 2, 64), (1, p, 0, 64), (1, p, 2, 65), (1, _pages(page=8), 2, 64), (1, _pages(max_pages=0), 2, 64)):
        assert L.hgf_diff_attention_kv8_workspace_bytes(args[0], ctypes.byref(args[1]), args[2], args[3]) == 0
    app = lambda k=0x100, v=0x100, cu=None, B=1, T=1: L.hgf_kv8_append(k, v, ctypes.byref(c), ctypes.byref(p), None, cu, B, T, None)
    assert app(k=None) == 1 and app(v=None) == 1 and app(T=2) == 2 and app(T=0, cu=0x100) == 2 and app(T=1 << 24, cu=0x100) == 2
    assert app(k=0x108) == 3 and app(cu=0x102) == 3
    gat = lambda k=0x100, cu=0x100, T=1: L.hgf_kv8_gather(ctypes.byref(c), ctypes.byref(p), None, cu, 1, T, k, 0x100, None)
    assert gat(k=None) == 1 and gat(cu=None) == 1 and gat(T=0) == 2 and gat(k=0x108) == 3
    assert L.hgf_kv8_pages_grow(ctypes.byref(p), 0x100, 0x100, 16385, 0x100, None) == 2
    assert L.hgf_kv8_pages_grow(ctypes.byref(p), 0x100, 0x100, 0, 0x100, None) == 2
    assert L.hgf_kv8_pages_grow(ctypes.byref(p), None, 0x100, 1, 0x100, None) == 1
    assert L.hgf_kv8_pages_fork(ctypes.byref(p), 0x100, 0x100, 1, None, 0x100, None) == 1
    assert L.hgf_kv8_pages_free(ctypes.byref(p), 0x102, 1, None) == 3
    assert L.hgf_kv8_pages_compact(ctypes.byref(p), 0x100, None, 0x100, None) == 1
    assert L.hgf_kv8_copy_pages(ctypes.byref(c), None, None, 1, None) == 1
    assert L.hgf_kv8_copy_pages(ctypes.byref(c), 0x100, None, 0, None) == 2


def test_refused_launches_are_reported():
    if torch.cuda.is_available():
        pytest.skip("needs a host where launches are refused (no GPU)")
    L, c, p = hb.lib(), ctypes.byref(_cache()), ctypes.byref(_pages())
    assert _prefill() == 6
    assert L.hgf_kv8_pages_grow(p, 0x100, 0x200, 1, 0x300, None) == 6
    assert L.hgf_kv8_pages_compact(p, 0x100, 0x200, 0x300, None) == 6
    assert L.hgf_kv8_append(0x100, 0x100, c, p, None, None, 1, 1, None) == 6
    assert L.hgf_diff_attention_decode_kv8(0x100, c, p, None, 1, 0.5, 0.0, None, 0x100, 0x100, BIG, None) == 6


def test_binding_refuses_wrong_tensors():
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        hb.hgf_diff_attention_prefill(h(4, 2, 32), h(4, 2, 32), h(4, 1, 32), cu, 0.5)          # not in device memory
    with pytest.raises(ValueError):
        hb.Kv8Cache(4, 16, 1, 24, device="cpu")
    pages, cache = hb.Kv8Pages(4, 16, 2, 2, device="cpu"), hb.Kv8Cache(4, 16, 1, 16, device="cpu")
    with pytest.raises(ValueError):
        hb.hgf_kv8_append(h(1, 2, 16), h(1, 1, 16), cache, pages)
    with pytest.raises(ValueError):
        hb.hgf_kv8_pages_free(pages, torch.zeros(1, dtype=torch.int32))
