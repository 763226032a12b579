"""Attention over prompts by the rows that a workgroup holds (32, 64 or 128), which follow from rows and heads: every test
says which, and looks at the captured launch, so that another rule cannot leave a variant untested.  Against the oracle in fp64
for some rows and heads."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb
from kv8 import close, dev, half, ints
from launches import launches

pytestmark = pytest.mark.gpu

LAM = 0.8
VARIANTS = [(16, 128), (16, 64), (16, 32), (32, 128), (32, 64), (32, 32), (64, 128), (64, 64), (64, 32), (128, 128), (128, 64)]


def _heads(d, rows, tokens, sequences=1):
    """Heads for which workgroups hold `rows` rows, of causal rows without many earlier keys."""
    wide = {(128, 128): 310, (128, 64): 150, (64, 64): 240, (64, 32): 60}.get((d, rows), {128: 420, 64: 320, 32: 100}[rows])
    return max(1, -(-wide // (tokens // 128 + sequences)))


def _run(q, k, v, cu, rows, cu_k=None, **kw):
    """The call on the GPU, and that its workgroups hold so many rows; twice the same bits."""
    H, B = v.shape[1], len(cu) - 1
    args = [dev(q), dev(k), dev(v), ints(cu), LAM]
    opt = {n: (ints(x) if n in ("prefix", "doc_q", "doc_k") else dev(x) if n == "slopes" else x) for n, x in kw.items()}
    if cu_k is not None:
        opt["cu_k"] = ints(cu_k)
    out = hb.hgf_diff_attention_prefill(*args, **opt)
    again = torch.full_like(out, 7.0)
    call = lambda: hb.hgf_diff_attention_prefill(*args, out=again, **opt)
    call()
    assert torch.equal(torch.nan_to_num(out, 9.0), torch.nan_to_num(again, 9.0))
    (threads, grid), = launches(call)
    assert threads == 512 and grid == ((q.shape[0] // rows + B) * H, 1, 1), (grid, H)
    return out.cpu().numpy()


def _some(rng, n, *more):
    """Rows about the borders of tiles and workgroups, and others."""
    return sorted({i for i in (0, 1, 31, 32, 63, 64, 127, 128, 129, n - 130, n - 65, n - 33, n - 2, n - 1, *more) if 0 <= i < n}
                  | {int(x) for x in rng.integers(0, n, 6)})


def _compare(out, q, k, v, picks, seen_of, heads, what, earlier=0, softcap=0.0, slopes=None):
    H, nk = v.shape[1], len(k)
    vmax = float(np.abs(v.astype(np.float64)[np.isfinite(v)]).max())
    j = np.arange(nk)
    for h in heads:
        two = [h, H + h]
        seen = np.stack([seen_of(i) for i in picks])
        away = np.stack([np.abs(earlier + i - j) for i in picks])
        ref = ko.attend(q[picks][:, two], k[:, two], v[:, [h]], LAM, seen, away, softcap, None if slopes is None else slopes[two])
        close(out[picks][:, [h]], ref, vmax, LAM, True, f"{what}, head {h} of {H}, rows {picks}")


@pytest.mark.parametrize("d,rows", VARIANTS)
@pytest.mark.parametrize("kind", ["plain", "cap", "coarse cap and bias", "prefix"])
def test_a_long_prompt(d, rows, kind):
    """1500 keys: every buffer of tiles used several times, tiles that all rows see whole and tiles that they do not."""
    n = 1500
    H = _heads(d, rows, n)
    rng = np.random.default_rng(d + rows)
    q, k, v = half(rng, n, 2 * H, d), half(rng, n, 2 * H, d), half(rng, n, H, d)
    slopes = (2.0 ** -rng.uniform(1, 9, 2 * H)).astype(np.float32)
    kw = {"plain": {}, "cap": dict(softcap=25.0), "coarse cap and bias": dict(softcap=2000.0, slopes=slopes), "prefix": dict(prefix=[700])}[kind]
    out = _run(q, k, v, [0, n], rows, **kw)
    j = np.arange(n)
    kw.pop("prefix", None)
    _compare(out, q, k, v, _some(rng, n, 699, 700, 701), lambda i: (j <= i) | ((j < 700) if kind == "prefix" else False), {0, H // 2, H - 1},
             kind, **kw)


@pytest.mark.parametrize("d,rows", VARIANTS)
def test_documents_over_more_than_one_window_of_tiles(d, rows):
    """64 tiles are looked through at a time: documents at both ends, in windows of which nothing matters, and rising ones."""
    n = 8500 if rows == 32 else 4500                          # (tiles of 128 keys where workgroups hold 32 rows)
    H = _heads(d, rows, n)
    rng = np.random.default_rng(2 * d + rows)
    q, k, v = half(rng, n, 2 * H, d), half(rng, n, 2 * H, d), half(rng, n, H, d)
    far = np.full(n, 7)
    far[:50], far[n - 300:n - 20], far[n - 20:] = 3, 3, -1
    j = np.arange(n)
    for name, docs in (("far", far), ("rising", np.sort(rng.integers(0, 12, n)))):
        out = _run(q, k, v, [0, n], rows, doc_q=docs, doc_k=docs)
        picks = _some(rng, n, 49, 50, n - 301, n - 300, n - 299, n - 21, n - 20, n // 2)
        _compare(out, q, k, v, picks, lambda i: (j <= i) & (docs == docs[i]) & (docs >= 0), {0, H - 1}, name)


@pytest.mark.parametrize("d,rows", VARIANTS)
@pytest.mark.parametrize("documents", [False, True])
def test_infinities_and_what_is_not_a_number(d, rows, documents):
    """They reach the rows that see them and no other, from tiles in every buffer, the masked ones of the diagonal among them."""
    n = 600
    H = _heads(d, rows, n)
    rng = np.random.default_rng(3 * d + rows)
    q, k, v = half(rng, n, 2 * H, d), half(rng, n, 2 * H, d), half(rng, n, H, d)
    docs = np.where(np.arange(n) < 580, 0, -1) if documents else None
    kw = dict(doc_q=docs, doc_k=docs) if documents else {}
    clean = _run(q, k, v, [0, n], rows, **kw)
    v[3, 0, d - 1], v[70, H - 1, 1], v[255, 0, 5], v[256, 0, 7], v[400, H // 2, 0], k[501, H - 1, 2] = np.inf, np.nan, -np.inf, np.nan, np.inf, np.nan
    want = np.zeros(v.shape, dtype=bool)
    last = 580 if documents else n
    for key, h, c in ((3, 0, d - 1), (70, H - 1, 1), (255, 0, 5), (256, 0, 7), (400, H // 2, 0)):
        want[key:last, h, c] = True
    want[501:last, H - 1] = True
    if documents:
        k[580:], v[580:] = np.nan, np.inf
    out = _run(q, k, v, [0, n], rows, **kw)
    assert np.array_equal(~np.isfinite(out), want)
    assert np.array_equal(out[~want], clean[~want])


@pytest.mark.parametrize("d,rows", VARIANTS)
def test_ragged_sequences(d, rows):
    """Lengths about the rows of a workgroup, one token and none, in a packed batch."""
    lens = [200, 0, 1, 127, 128, 129, 33, 64]
    H = _heads(d, rows, sum(lens), len(lens))
    rng = np.random.default_rng(4 * d + rows)
    cu = [int(x) for x in np.cumsum([0] + lens)]
    q, k, v = (half(rng, cu[-1], h, d) for h in (2 * H, 2 * H, H))
    out = _run(q, k, v, cu, rows)
    for h in {0, H - 1}:
        two = [h, H + h]
        close(out[:, [h]], ko.prefill(q[:, two], k[:, two], v[:, [h]], cu, LAM), float(np.abs(v).max()), LAM, True, f"head {h} of {H}")


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_128_rows_that_see_about_as_many_keys(d, causal):
    """Without causality, or behind many earlier keys, 128 rows are taken from fewer workgroups on."""
    n, earlier = 300, 1100 if causal else 0
    H = 104 if d == 128 and not causal else 70                # (three workgroups a head)
    rng = np.random.default_rng(5 * d + causal)
    q, k, v = half(rng, n, 2 * H, d), half(rng, n + earlier, 2 * H, d), half(rng, n + earlier, H, d)
    out = _run(q, k, v, [0, n], 128, cu_k=[0, n + earlier], causal=causal)
    j = np.arange(n + earlier)
    _compare(out, q, k, v, _some(rng, n), lambda i: (j <= i + earlier) | (not causal), {0, H - 1}, "alike", earlier=earlier)
