"""The decode step over the 8-bit cache where a sequence is taken in several parts and merged by a second launch: tables with room
for more positions than one part takes, few rows.  Against the oracle in fp64, on the values that the cache holds."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb
from kv8 import Both, close, dev, half, ints
from launches import launches

pytestmark = pytest.mark.gpu

PAGE, MAX_PAGES = 64, 80                                     # (tables of 5120 positions)
DIMS = [16, 32, 64, 128]


def _made(seed, d, H, lens, spare=2):
    rng = np.random.default_rng(seed)
    t = Both(sum((n + PAGE - 1) // PAGE for n in lens) + spare, PAGE, len(lens), MAX_PAGES, H, d)
    t.place(lens, rng)
    t.fill(rng)
    return t, rng


def _run(t, q, rows, **kw):
    return hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, 0.8, seqs=ints(rows), **kw)


def _check(t, q, rows, softcap=0.0, slopes=None):
    assert hb.hgf_diff_attention_kv8_workspace_bytes(len(rows), t.pages, t.H, q.shape[2]) > 0
    out = _run(t, q, rows, softcap=softcap, slopes=None if slopes is None else dev(slopes))
    ref = ko.decode(q, *t.pools[0], t.ref.table, t.ref.lens, rows, 0.8, softcap, slopes)
    vmax = max(1e-30, float(np.abs(t.pools[0][1].codes * np.repeat(t.pools[0][1].scale, 16, axis=2)[..., None]).max()))
    close(out.cpu().numpy(), ref, vmax, 0.8, False, f"lens {t.ref.lens}, rows {rows}")
    return out


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("kind", ["plain", "cap", "bias", "both"])
def test_lengths_about_the_parts(d, kind):
    """No position, one, one part more or less a position, many parts, all of the table."""
    H, lens = 2, [0, 1, 255, 256, 257, 1300, 2047, 5120]
    t, rng = _made(d, d, H, lens)
    slopes = (2.0 ** -rng.uniform(2, 10, 2 * H)).astype(np.float32) if kind in ("bias", "both") else None
    softcap = 20.0 if kind in ("cap", "both") else 0.0
    _check(t, half(rng, 8, 2 * H, d), list(range(8)), softcap, slopes)
    _check(t, half(rng, 5, 2 * H, d), [7, -1, 0, 8, 7], softcap, slopes)      # one twice, two that do not exist


@pytest.mark.parametrize("d", DIMS)
def test_two_launches(d):
    t, rng = _made(3, d, 3, [700, 30])
    q, rows, slopes = dev(half(rng, 2, 6, d)), ints([1, 0]), dev(np.full(6, 0.01, dtype=np.float32))
    scratch = torch.empty(hb.hgf_diff_attention_kv8_workspace_bytes(2, t.pages, 3, d), dtype=torch.uint8, device="cuda")
    out = torch.empty((2, 3, d), dtype=torch.float16, device="cuda")
    for kw in ({}, dict(softcap=30.0), dict(slopes=slopes)):
        call = lambda: hb.hgf_diff_attention_decode_kv8(q, t.caches[0], t.pages, 0.8, seqs=rows, out=out, workspace=scratch, **kw)
        call()
        (threads, grid), (merge, _) = launches(call)
        assert (threads, merge) == (256, 512) and grid[0] == 3 and grid[1] > 1 and grid[2] == 2


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("softcap", [0.0, 30.0])
def test_missing_pages(d, softcap):
    """A page inside a part, all pages of a part, of the first, of the last, of every part; a length beyond the table."""
    lens = [1500, 1500, 1500, 700, 300, 5120]
    t, rng = _made(50 + d, d, 2, lens)
    n_pages = len(t.ref.refs)
    t.ref.table[0, 5] = -1
    t.ref.table[1, 4:8], t.ref.table[2, :4], t.ref.table[3, 8:11], t.ref.table[4, :5] = n_pages, -7, 1 << 20, -1
    t.ref.lens[5] = 1 << 29
    t.push()
    out = _check(t, half(rng, 6, 4, d), list(range(6)), softcap)
    assert not out[4].any()


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_queries_that_are_no_numbers(d, bad):
    """Their head of their row becomes NaN, in every part that has positions or none, and nothing else changes."""
    lens = [1500, 300, 5000]
    t, rng = _made(70 + d, d, 2, lens)
    t.ref.table[0, 4:8] = -1                                  # (a part without positions among others)
    t.push()
    q = half(rng, 3, 4, d)
    clean = _check(t, q, [0, 1, 2])
    q[0, 0, d - 1], q[2, 3, 0] = bad, bad                     # (branch 1 of head 0, branch 2 of head 1)
    out = _run(t, q, [0, 1, 2])
    assert torch.isnan(out[0, 0]).all() and torch.isnan(out[2, 1]).all()
    for b, h in ((0, 1), (1, 0), (1, 1), (2, 0)):
        assert torch.equal(out[b, h], clean[b, h])


@pytest.mark.parametrize("d", DIMS)
def test_parts_of_very_different_scores_and_scales(d):
    """Maxima and V's scales that differ by many powers of two from part to part, rising and falling."""
    rng = np.random.default_rng(90 + d)
    n = 1600
    for order in (1, -1):
        t = Both(30, PAGE, 1, MAX_PAGES, 1, d)
        t.place([n], rng)
        ramp = np.linspace(0.02, 2.0, n)[::order, None, None]
        size = np.exp2(np.arange(n) // 16 % 16 - 8.0)[:, None, None]
        t.append((np.abs(half(rng, n, 2, d)) * ramp / np.sqrt(d / 16)).astype(np.float16), (half(rng, n, 1, d) * size).astype(np.float16), [0], [n])
        _check(t, (np.abs(half(rng, 1, 2, d)) * 0.7).astype(np.float16), [0])
        _check(t, np.zeros((1, 2, d), dtype=np.float16), [0])


@pytest.mark.parametrize("d", DIMS)
def test_agrees_with_the_fp16_decode_step(d):
    """The bound: both are within the other tests' bound of the same values' attention."""
    lens = [1900, 513]
    t, rng = _made(110 + d, d, 2, lens)
    q = half(rng, 2, 4, d)
    k = torch.zeros((2, 1900, 4, d), dtype=torch.float16, device="cuda")
    v = torch.zeros((2, 1900, 2, d), dtype=torch.float16, device="cuda")
    for s, n in enumerate(lens):
        hb.hgf_kv8_gather(t.caches[0], t.pages, ints([0, n]), k[s], v[s], seqs=ints([s]))
    a = _check(t, q, [0, 1]).double()
    b = hb.hgf_diff_attention_decode(dev(q), k, v, ints(lens), 0.8).double()
    assert ((a - b).abs() <= 2.0 ** -10 * a.abs() + 2.0 ** -24 + 2 * 2.3e-5 * 1.8 * float(v.abs().max())).all()


@pytest.mark.parametrize("d", DIMS)
def test_two_captured_steps_share_a_workspace(d):
    """Grow, append and attend as graphs over two caches of one table, replayed in turn across the borders of parts."""
    H, lens = 2, [254, 1022, 0]
    rng = np.random.default_rng(130 + d)
    t = Both(40, PAGE, 3, MAX_PAGES, H, d, layers=2)
    t.place(lens, rng)
    t.fill(rng, layer=0), t.fill(rng, layer=1)
    q = [dev(half(rng, 3, 2 * H, d)) for _ in range(2)]
    k, v = torch.zeros((3, 2 * H, d), dtype=torch.float16, device="cuda"), torch.zeros((3, H, d), dtype=torch.float16, device="cuda")
    seqs, ones, ok = ints([0, 1, 2]), ints([1, 1, 1]), ints([0, 0, 0])
    out = [torch.empty((3, H, d), dtype=torch.float16, device="cuda") for _ in range(2)]
    scratch = torch.empty(hb.hgf_diff_attention_kv8_workspace_bytes(3, t.pages, H, d), dtype=torch.uint8, device="cuda")
    assert scratch.numel() > 0
    for layer in range(2):
        hb.hgf_diff_attention_decode_kv8(q[layer], t.caches[layer], t.pages, 0.8, seqs=seqs, out=out[layer], workspace=scratch)

    def step(layer):
        if layer == 0:
            hb.hgf_kv8_pages_grow(t.pages, seqs, ones, ok=ok)
        hb.hgf_kv8_append(k, v, t.caches[layer], t.pages, seqs=seqs)
        hb.hgf_diff_attention_decode_kv8(q[layer], t.caches[layer], t.pages, 0.8, seqs=seqs, out=out[layer], workspace=scratch)

    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for layer, g in enumerate(graphs):
        with torch.cuda.graph(g):
            step(layer)
    for i in range(4):
        assert t.ref.grow([0, 1, 2], [1, 1, 1]).all()
        for layer in range(2):
            k_new, v_new = half(rng, 3, 2 * H, d, scale=float(i + 1)), half(rng, 3, H, d)
            k.copy_(dev(k_new)), v.copy_(dev(v_new))
            graphs[layer].replay()
            torch.cuda.synchronize()
            for s in range(3):
                for pool, x in zip(t.pools[layer], (k_new, v_new)):
                    pool.write(t.ref.table[s], int(t.ref.lens[s]) - 1, x[s:s + 1])
            t.check_tables(), t.check_pools(layer)
            ref = ko.decode(q[layer].cpu().numpy(), *t.pools[layer], t.ref.table, t.ref.lens, [0, 1, 2], 0.8)
            vmax = float(np.abs(t.pools[layer][1].codes * np.repeat(t.pools[layer][1].scale, 16, axis=2)[..., None]).max())
            close(out[layer].cpu().numpy(), ref, vmax, 0.8, False, f"step {i}, layer {layer}")
            again = hb.hgf_diff_attention_decode_kv8(q[layer], t.caches[layer], t.pages, 0.8, seqs=seqs)
            assert torch.equal(again, out[layer])
