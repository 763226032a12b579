"""GPU parity of the differential attention over prompts against the oracle in fp64."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb
from kv8 import close, dev, half, ints

pytestmark = pytest.mark.gpu


def _inputs(seed, H, d, lq, lk=None, scale=1.0):
    rng = np.random.default_rng(seed)
    lk = lq if lk is None else lk
    return (half(rng, sum(lq), 2 * H, d, scale=scale), half(rng, sum(lk), 2 * H, d), half(rng, sum(lk), H, d),
            [int(x) for x in np.cumsum([0] + lq)], [int(x) for x in np.cumsum([0] + lk)], rng)


def _check(q, k, v, cu_q, lam=0.8, cu_k=None, **kw):
    opt = {n: (ints(x) if n in ("prefix", "doc_q", "doc_k") else dev(x) if n == "slopes" else x) for n, x in kw.items() if x is not None}
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu_q), lam, cu_k=None if cu_k is None else ints(cu_k), **opt)
    ref = ko.prefill(q, k, v, cu_q, lam, cu_k=cu_k, **kw)
    finite = np.isfinite(v.astype(np.float64))
    close(out.cpu().numpy(), ref, float(np.abs(v.astype(np.float64)[finite]).max()), lam, True, str((cu_q, cu_k, list(kw))))
    return out


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("lens", [[1], [2, 31, 32, 33], [64, 0, 65], [127, 128, 129], [300, 1]])
def test_lengths(d, lens):
    H = {16: 3, 32: 2, 64: 2, 128: 1}[d]
    q, k, v, cu, _, _ = _inputs(d + sum(lens), H, d, lens)
    _check(q, k, v, cu)
    _check(q, k, v, cu, causal=False, lam=-0.4)


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("lq,lk", [([1], [200]), ([40, 7, 0], [41, 300, 5]), ([130, 3], [400, 3]), ([70, 5], [64, 0]), ([200], [20])])
def test_rows_behind_earlier_keys_and_before_them(d, lq, lk):
    """More keys than queries, as many, fewer (rows with nothing before them), none at all."""
    q, k, v, cu_q, cu_k, _ = _inputs(d + sum(lq) + sum(lk), 2, d, lq, lk)
    _check(q, k, v, cu_q, cu_k=cu_k)
    _check(q, k, v, cu_q, cu_k=cu_k, prefix=[3, 100, 1][:len(lq)])


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("softcap,bias", [(8.0, False), (30.0, True), (0.0, True), (1e-3, True), (1e5, False)])
def test_caps_and_biases(d, softcap, bias):
    H = 2
    q, k, v, cu, _, rng = _inputs(d + int(softcap), H, d, [150, 70])
    slopes = (2.0 ** -rng.uniform(0, 8, 2 * H)).astype(np.float32) if bias else None
    _check(q, k, v, cu, softcap=softcap, slopes=slopes)
    _check(q, k, v, cu, softcap=softcap, slopes=slopes, prefix=[90, 200])


def test_documents():
    """In rising order, in any order, one number to every row, padding in the middle and at the end, rows that see nothing."""
    H, d, n = 2, 64, 333
    q, k, v, cu, _, rng = _inputs(5, H, d, [n, 40])
    rising = np.sort(rng.integers(0, 6, n)).tolist() + [3] * 40
    mixed = rng.integers(0, 4, n + 40).tolist()
    padded = [(-1 if 60 < i < 200 or i > 320 else i // 100) for i in range(n)] + [-7] * 40
    for docs in (rising, mixed, padded, list(range(n + 40))):
        _check(q, k, v, cu, doc_q=docs, doc_k=docs)
        _check(q, k, v, cu, doc_q=docs, doc_k=docs, prefix=[250, 10], softcap=20.0)
        _check(q, k, v, cu, doc_q=docs, doc_k=docs, causal=False)
    out = _check(q, k, v, cu, doc_q=padded, doc_k=padded)
    assert not out[61:200].any() and not out[n:].any()
    # one document and padding among the same 32 rows
    ends = [0] * 180 + [-1] * 20
    out = _check(q[:200], k[:200], v[:200], [0, 200], doc_q=ends, doc_k=ends)
    assert not out[180:].any()
    # documents of the queries that no key has
    _check(q, k, v, cu, doc_q=[9] * (n + 40), doc_k=rising)


@pytest.mark.parametrize("H", [2, 150])                   # workgroups of few rows, and of 128
@pytest.mark.parametrize("d", [16, 64, 128])
def test_infinities_and_what_is_not_a_number(d, H):
    """They reach the rows that see them, and no other."""
    n = 200
    q, k, v, cu, _, _ = _inputs(6 + d, H, d, [n])
    docs = [0] * 180 + [-1] * 20
    clean = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, doc_q=ints(docs), doc_k=ints(docs))
    k[180:], v[180:] = np.nan, np.inf                         # padding
    k[120, 1, 3], v[100, 0, 5], v[90, 1, 2] = np.nan, np.inf, np.nan
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, doc_q=ints(docs), doc_k=ints(docs)).float()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[120:180, 1], want[100:180, 0, 5], want[90:180, 1, 2] = True, True, True
    assert torch.equal(bad, want)
    assert torch.equal(out[~bad], clean.float()[~bad])
    # a query row of them concerns itself only
    q[50] = np.inf
    again = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, doc_q=ints(docs), doc_k=ints(docs)).float()
    keep = torch.arange(n) != 50
    assert torch.equal(torch.nan_to_num(again[keep], 7.0), torch.nan_to_num(out[keep], 7.0)) and not torch.isfinite(again[50]).any()


def test_peaked_scores_that_rise_along_the_keys():
    """Maxima that grow by much and by little from tile to tile, and a row whose largest score comes first."""
    H, d, n = 1, 32, 400
    q, k, v, cu, _, rng = _inputs(7, H, d, [n])
    ramp = np.linspace(0.0, 1.5, n)[:, None, None]
    q = np.abs(q).astype(np.float16)
    _check(q, (np.abs(k) * ramp).astype(np.float16), v, cu)
    _check(q, (np.abs(k) * ramp[::-1]).astype(np.float16), v, cu)
    _check((q * 0).astype(np.float16), k, v, cu)


def test_rows_outside_the_sequences_stay():
    H, d = 2, 32
    q, k, v, _, _, _ = _inputs(8, H, d, [100])
    out = torch.full((100, H, d), 3.0, dtype=torch.float16, device="cuda")
    hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints([10, 40, 30, 90]), 0.8, out=out)
    assert (out[:10] == 3.0).all() and (out[90:] == 3.0).all()
    ref = ko.prefill(q, k, v, [10, 40], 0.8)[10:40]
    close(out[10:30].cpu().numpy(), ref[:20], float(np.abs(v).max()), 0.8, True)           # (rows 30 .. 39 belong to two sequences)
    # offsets beyond the tensor are clipped to it
    clipped = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints([-5, 60, 1000]), 0.8)
    want = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints([0, 60, 100]), 0.8)
    assert torch.equal(clipped, want)


def test_many_sequences():
    rng = np.random.default_rng(9)
    lens = [int(x) for x in rng.integers(0, 6, 500)]
    q, k, v, cu, _, _ = _inputs(10, 1, 16, lens)
    _check(q, k, v, cu)


@pytest.mark.parametrize("H,d", [(1, 16), (6, 64), (5, 128)])
def test_more_sequences_than_lanes(H, d):
    """70 ragged sequences, in workgroups of 32 (64) and of 128 rows, with and without documents and earlier keys."""
    rng = np.random.default_rng(H)
    lq = [int(x) for x in rng.integers(0, 60, 70)]
    lq[3] = 150
    lk = [n + int(x) for n, x in zip(lq, rng.integers(0, 30, 70))]
    q, k, v, cu_q, cu_k, _ = _inputs(13 + d, H, d, lq, lk)
    docs = [list(rng.integers(-1, 3, n)) for n in lk]
    doc_k = np.concatenate(docs)
    doc_q = np.concatenate([x[len(x) - n:] for x, n in zip(docs, lq)])
    if H == 1:
        _check(q, k, v, cu_q, cu_k=cu_k)
    _check(q, k, v, cu_q, cu_k=cu_k, doc_q=doc_q, doc_k=doc_k, prefix=[9] * 70)


@pytest.mark.parametrize("H,d,n", [(1, 16, 8500), (8, 64, 4500)])
def test_documents_over_more_tiles_than_one_window(H, d, n):
    """Documents far apart: windows of 64 tiles of which all, some or no tile matters; rows against the oracle one by one."""
    q, k, v, cu, _, rng = _inputs(14 + d, H, d, [n])
    far = np.full(n, 7)
    far[:50], far[n - 300:n - 20] = 3, 3                                  # one document at both ends
    rising = np.sort(rng.integers(0, 12, n))
    for docs in (far, rising):
        out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, doc_q=ints(docs), doc_k=ints(docs)).cpu().numpy()
        for i in [0, 49, 50, n - 301, n - 300, n - 21, n - 20, n - 1] + [int(x) for x in rng.integers(0, n, 6)]:
            seen = ((np.arange(n) <= i) & (docs == docs[i]))[None, :]
            ref = ko.attend(q[i:i + 1], k, v, 0.8, seen, np.abs(i - np.arange(n))[None, :])
            close(out[i:i + 1], ref, float(np.abs(v).max()), 0.8, True, f"row {i}")


def test_a_prefix_means_nothing_without_causality_and_is_clipped_with_it():
    q, k, v, cu, _, _ = _inputs(15, 2, 32, [90, 40])
    run = lambda **kw: hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, **kw)
    assert torch.equal(run(causal=False), run(causal=False, prefix=ints([5, 1000])))
    assert torch.equal(run(), run(prefix=ints([-3, -2147483648])))
    assert torch.equal(run(prefix=ints([2147483647, 40])), run(prefix=ints([90, 40])))


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", ["plain", "cap", "bias", "documents", "earlier keys"])
def test_workgroups_of_128_rows(d, kind):
    """So many heads that short sequences fill the chip: every kind of score and mask there, some heads against the oracle."""
    H, lq = 110, [150, 33, 1, 200]
    lk = [n + 70 for n in lq] if kind == "earlier keys" else lq
    q, k, v, cu_q, cu_k, rng = _inputs(18 + d, H, d, lq, lk)
    slopes = (2.0 ** -rng.uniform(0, 8, 2 * H)).astype(np.float32)
    docs = np.sort(rng.integers(-1, 4, sum(lk)))
    kw = {"plain": {}, "cap": dict(softcap=20.0, prefix=[100, 5, 1, 0]), "bias": dict(slopes=slopes, causal=False),
          "documents": dict(doc_q=docs, doc_k=docs, softcap=600.0, slopes=slopes), "earlier keys": dict(cu_k=cu_k, prefix=[90, 90, 9, 260])}[kind]
    opt = {n: (ints(x) if n in ("prefix", "doc_q", "doc_k", "cu_k") else dev(x) if n == "slopes" else x) for n, x in kw.items()}
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu_q), 0.8, **opt).cpu().numpy()
    for h in (0, 57, 109):
        two = [h, H + h]
        ref_kw = dict(kw, slopes=slopes[two]) if "slopes" in kw else kw
        ref = ko.prefill(q[:, two], k[:, two], v[:, [h]], cu_q, 0.8, **ref_kw)
        close(out[:, [h]], ref, float(np.abs(v).max()), 0.8, True, f"{kind}, head {h}")


@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("kind", ["plain", "cap", "documents", "infinities"])
def test_workgroups_of_64_rows(d, kind):
    """As many heads as fill the chip by half with 128 rows each; some heads against the oracle, 4 sequences and 70."""
    H, rng = 50, np.random.default_rng(d)
    for n, lq in ((H, [150, 33, 1, 200]), (4, [150] + [int(x) for x in rng.integers(0, 60, 69)])):
        q, k, v, cu, _, rng = _inputs(20 + d, n, d, lq)
        docs = np.sort(rng.integers(-1, 4, sum(lq)))
        if kind == "infinities":
            v[100, :, d - 3], v[170, :, 2] = np.inf, np.nan
        kw = {"cap": dict(softcap=20.0, prefix=[70] * len(lq)), "documents": dict(doc_q=docs, doc_k=docs)}.get(kind, {})
        opt = {m: ints(x) if m != "softcap" else x for m, x in kw.items()}
        out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8, **opt).cpu().numpy()
        for h in {0, n // 2, n - 1}:
            two = [h, n + h]
            ref = ko.prefill(q[:, two], k[:, two], v[:, [h]], cu, 0.8, **kw)
            known, vmax = np.isfinite(ref), float(np.abs(v[np.isfinite(v)]).max())
            assert np.array_equal(np.isfinite(out[:, [h]]), known), f"{kind}, {len(lq)} sequences, head {h}"
            close(out[:, [h]][known], ref[known], vmax, 0.8, True, f"{kind}, {len(lq)} sequences, head {h}")


def test_many_heads():
    """Rows of a key that are a quarter of a MiB long."""
    q, k, v, cu, _, _ = _inputs(16, 512, 128, [70])
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8).cpu().numpy()
    for h in (0, 311, 511):
        ref = ko.prefill(q[:, [h, 512 + h]], k[:, [h, 512 + h]], v[:, [h]], cu, 0.8)
        close(out[:, [h]], ref, float(np.abs(v).max()), 0.8, True, f"head {h}")


def test_many_heads_of_many_sequences():
    """More threads than a grid may have in one dimension: 2^13 + 300 sequences of one token, 1024 heads.  A row sees one key, so it
    is (1 - lambda) / 2 of its value: the weight cancels in a quotient, four roundings in fp32 and one to fp16."""
    B, H, d = 8492, 1024, 16
    gen = torch.Generator(device="cuda").manual_seed(19)
    q, k = (torch.randn((B, 2 * H, d), generator=gen, device="cuda", dtype=torch.float16) for _ in range(2))
    v = torch.randn((B, H, d), generator=gen, device="cuda", dtype=torch.float16)
    out = hb.hgf_diff_attention_prefill(q, k, v, torch.arange(B + 1, dtype=torch.int32, device="cuda"), 0.25)
    ref = v.double() * 0.375
    # each branch is within 3 * 2^-24 of 0.5 and 0.125 times the value; fp16: half a step, or half of 2^-24 below its normal numbers
    bound = ref.abs() * 2.0 ** -11 + v.double().abs() * (0.625 * 4 * 2.0 ** -24) + 2.0 ** -25
    assert bool(((out.double() - ref).abs() <= bound * 1.001).all())


def test_two_calls_at_once():
    q, k, v, cu, _, _ = _inputs(17, 4, 64, [700, 300])
    a, b = (tuple(dev(t) for t in (q, k, v)) for _ in range(2))
    a[0].mul_(0.5)
    want = [hb.hgf_diff_attention_prefill(*x, ints(cu), 0.8) for x in (a, b)]
    cu_d, streams = ints(cu), [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[hb.hgf_diff_attention_prefill(*x, cu_d, 0.8, stream=s) for s, x in zip(streams, (a, b))] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        assert torch.equal(pair[0], want[0]) and torch.equal(pair[1], want[1])


@pytest.mark.parametrize("H,d,n", [(8, 32, 500), (4, 64, 1500), (2, 128, 1100)])
def test_longer_prompts(H, d, n):
    """Against the decode step's own plain form, row by row, for some of the rows."""
    q, k, v, cu, _, rng = _inputs(H + d, H, d, [n])
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints(cu), 0.8).cpu().numpy()
    for i in [0, n - 1] + [int(x) for x in rng.integers(0, n, 12)]:
        seen = (np.arange(n) <= i)[None, :]
        ref = ko.attend(q[i:i + 1], k, v, 0.8, seen, np.abs(i - np.arange(n))[None, :])
        close(out[i:i + 1], ref, float(np.abs(v).max()), 0.8, True, f"row {i}")


def test_another_stream_and_a_captured_call():
    H, d = 2, 64
    q, k, v, cu, _, _ = _inputs(12, H, d, [200, 70])
    dq, dk, dv, dcu = dev(q), dev(k), dev(v), ints(cu)
    want = hb.hgf_diff_attention_prefill(dq, dk, dv, dcu, 0.8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hb.hgf_diff_attention_prefill(dq, dk, dv, dcu, 0.8, stream=side)
    side.synchronize()
    assert torch.equal(want, got)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hgf_diff_attention_prefill(dq, dk, dv, dcu, 0.8, out=out)
    for i in range(3):
        dq.mul_(0.5), dcu.copy_(ints([0, 150 + i, 270]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, hb.hgf_diff_attention_prefill(dq, dk, dv, dcu, 0.8))
