"""GPU parity of the decode step over the 8-bit cache against the oracle in fp64, on the values that the cache holds."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb
from kv8 import Both, close, dev, half, ints

pytestmark = pytest.mark.gpu


def _check(t, q, rows, lam=0.8, softcap=0.0, slopes=None, seqs=True):
    out = hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, lam, seqs=ints(rows) if seqs else None, softcap=softcap,
                                           slopes=None if slopes is None else dev(slopes))
    ref = ko.decode(q, *t.pools[0], t.ref.table, t.ref.lens, rows, lam, softcap, slopes)
    vmax = max(1e-30, float(np.abs(t.pools[0][1].codes * np.repeat(t.pools[0][1].scale, 16, axis=2)[..., None]).max()))
    close(out.cpu().numpy(), ref, vmax, lam, False, f"lens {t.ref.lens}")
    return out


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("lens", [[1], [0, 2, 15, 16, 17], [63, 64, 65, 0, 255], [256, 257, 1, 700]])
def test_lengths(d, page, lens):
    rng = np.random.default_rng(d + page + sum(lens))
    H = {16: 3, 32: 8, 64: 2, 128: 1}[d]
    t = Both(sum(n // page + 1 for n in lens) + 2, page, len(lens) + 1, max(lens) // page + 2, H, d)
    t.place(lens, rng)
    t.fill(rng)
    _check(t, half(rng, len(lens), 2 * H, d), list(range(len(lens))), seqs=False)
    rows = [int(r) for r in rng.permutation(len(lens))] + [len(lens), len(lens) + 1, -1, 0]       # one empty, two that do not exist, one twice
    _check(t, half(rng, len(rows), 2 * H, d, scale=2.0), rows, lam=0.35)


@pytest.mark.parametrize("softcap,bias", [(5.0, False), (50.0, True), (0.0, True), (1e-3, False), (1e5, True)])
@pytest.mark.parametrize("d", [32, 128])
def test_caps_and_biases(softcap, bias, d):
    rng = np.random.default_rng(int(softcap) + d)
    H, lens = 3, [400, 77]
    t = Both(20, 64, 2, 8, H, d)
    t.place(lens, rng)
    t.fill(rng)
    slopes = (2.0 ** -rng.uniform(0, 8, 2 * H)).astype(np.float32) if bias else None
    _check(t, half(rng, 2, 2 * H, d), [0, 1], softcap=softcap, slopes=slopes)


def test_one_long_sequence_in_many_parts():
    rng = np.random.default_rng(11)
    t = Both(1100, 16, 1, 1100, 1, 16)
    t.place([16401], rng)
    t.fill(rng)
    _check(t, half(rng, 1, 2, 16), [0])
    # the same sequence as a short one of the same table: parts that have nothing to do
    for n in (1, 64, 65, 1000):
        t.ref.lens[0] = n
        t.push()
        _check(t, half(rng, 1, 2, 16), [0])


@pytest.mark.parametrize("d,lens", [(16, [1030, 33]), (32, [0, 700]), (64, [200, 1]), (128, [90, 0])])
def test_many_heads_over_a_long_table(d, lens):
    """So many heads that a sequence is one part although its table has room for more than 1024 positions."""
    rng = np.random.default_rng(18 + d)
    H = 512
    t = Both(sum(n // 16 + 1 for n in lens), 16, 2, 65, H, d)
    assert hb.hgf_diff_attention_kv8_workspace_bytes(2, t.pages, H, d) == 0
    t.place(lens, rng)
    t.fill(rng)
    _check(t, half(rng, 2, 2 * H, d), [0, 1])
    _check(t, half(rng, 2, 2 * H, d), [1, 0], softcap=30.0, slopes=(2.0 ** -rng.uniform(0, 8, 2 * H)).astype(np.float32))


def test_one_long_sequence_among_many_short_ones():
    """Parts that follow from the table's capacity: short sequences have fewer of them, some exactly one tile or part."""
    rng = np.random.default_rng(19)
    H, d, page = 24, 16, 64
    lens = [11000, 0, 1, 64, 255, 256, 257, 511, 512, 513, 768, 769] + [int(x) for x in rng.integers(0, 200, 48)]
    t = Both(sum(n // page + 1 for n in lens), page, len(lens), 180, H, d)
    assert hb.hgf_diff_attention_kv8_workspace_bytes(len(lens), t.pages, H, d) > 0
    t.place(lens, rng)
    t.fill(rng)
    _check(t, half(rng, len(lens), 2 * H, d), list(range(len(lens))))


def test_blocks_of_very_different_scales_and_peaked_scores():
    """V's scales and the softmax spread over many powers of two inside one tile of positions."""
    rng = np.random.default_rng(12)
    H, d, n = 2, 64, 200
    t = Both(8, 32, 1, 8, H, d)
    t.place([n], rng)
    size = np.exp2(rng.integers(-12, 8, (n // 16 + 1, 1, 1))).repeat(16, axis=0)[:n]
    t.append((half(rng, n, 2 * H, d) * 2).astype(np.float16), (half(rng, n, H, d) * size).astype(np.float16), [0], [n])
    t.check_pools()
    _check(t, (half(rng, 1, 2 * H, d) * 2).astype(np.float16), [0])
    _check(t, np.zeros((1, 2 * H, d), dtype=np.float16), [0])
    tiny = np.full((1, 2 * H, d), 2.0 ** -24, dtype=np.float16)
    tiny[0, 1, 3] = 60000.0
    _check(t, (tiny * np.float16(0.001)).astype(np.float16), [0])


def test_what_lies_behind_the_length_or_in_no_page_does_not_matter():
    rng = np.random.default_rng(13)
    H, d, page = 2, 32, 32
    t = Both(10, page, 3, 4, H, d)
    t.place([70, 100, 33], rng)
    t.fill(rng)
    q = half(rng, 3, 2 * H, d)
    first = _check(t, q, [0, 1, 2])
    c = t.caches[0]
    spare = [p for p in range(10) if t.ref.refs[p] == 0]
    for x in (c.k_scale, c.v_scale):
        x[spare] = float("nan")
    for s, n in enumerate([70, 100, 33]):                   # the blocks behind the newest one
        pg, blk = int(t.ref.table[s, n // page]), n % page // 16 + 1
        for x in (c.k_scale, c.v_scale):
            x[pg, :, blk:] = float("nan")
    t.pages.table[0, 3] = 1 << 30
    again = hb.hgf_diff_attention_decode_kv8(dev(q), c, t.pages, 0.8)
    assert torch.equal(first, again)
    # a page that is missing in the middle; a sequence of nothing else; lens beyond the table
    t = Both(10, page, 3, 4, H, d)
    t.place([128, 100, 33], rng)
    t.fill(rng)
    t.ref.table[1, 1], t.ref.table[2] = -5, 10
    t.ref.lens[0] = 1000
    t.push()
    _check(t, q, [0, 1, 2])


def test_queries_that_are_no_numbers():
    rng = np.random.default_rng(14)
    t = Both(4, 64, 2, 2, 2, 64)
    t.place([100, 50], rng)
    t.fill(rng)
    q = half(rng, 2, 4, 64)
    clean = hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, 0.8)
    q[0, 1, 3], q[1, 2, 0] = np.nan, np.inf
    out = hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, 0.8)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(out[1, 0]).all()
    assert torch.equal(out[0, 0], clean[0, 0]) and torch.equal(out[1, 1], clean[1, 1])


def test_agrees_with_the_fp16_decode_step_on_the_same_values():
    rng = np.random.default_rng(15)
    H, d, lens = 4, 64, [300, 513]
    t = Both(20, 64, 2, 9, H, d)
    t.place(lens, rng)
    t.fill(rng)
    q = dev(half(rng, 2, 2 * H, d))
    k = torch.zeros((2, 520, 2 * H, d), dtype=torch.float16, device="cuda")
    v = torch.zeros((2, 520, H, d), dtype=torch.float16, device="cuda")
    for s, n in enumerate(lens):
        hb.hgf_kv8_gather(t.caches[0], t.pages, ints([0, n]), k[s], v[s], seqs=ints([s]))
    a = hb.hgf_diff_attention_decode_kv8(q, t.caches[0], t.pages, 0.8)
    b = hb.hgf_diff_attention_decode(q, k, v, ints(lens), 0.8)
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -10 * a.float().abs().max() + 3e-4


def test_another_stream_and_a_captured_step():
    rng = np.random.default_rng(16)
    H, d = 2, 32
    t = Both(8, 64, 2, 4, H, d)
    t.place([130, 64], rng)
    t.fill(rng)
    q = dev(half(rng, 2, 2 * H, d))
    want = hb.hgf_diff_attention_decode_kv8(q, t.caches[0], t.pages, 0.8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hb.hgf_diff_attention_decode_kv8(q, t.caches[0], t.pages, 0.8, stream=side)
    side.synchronize()
    assert torch.equal(want, got)
    # grow, append and attend as one graph, replayed as the sequences become longer
    k, v = torch.zeros((2, 2 * H, d), dtype=torch.float16, device="cuda"), torch.zeros((2, H, d), dtype=torch.float16, device="cuda")
    seqs, ones, ok = ints([0, 1]), ints([1, 1]), ints([0, 0])
    out = torch.empty_like(want)
    scratch = torch.empty(hb.hgf_diff_attention_kv8_workspace_bytes(2, t.pages, H, d), dtype=torch.uint8, device="cuda")

    def step():
        hb.hgf_kv8_pages_grow(t.pages, seqs, ones, ok=ok)
        hb.hgf_kv8_append(k, v, t.caches[0], t.pages, seqs=seqs)
        hb.hgf_diff_attention_decode_kv8(q, t.caches[0], t.pages, 0.8, seqs=seqs, out=out, workspace=scratch)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        k_new, v_new = half(rng, 2, 2 * H, d, scale=float(i + 1)), half(rng, 2, H, d)
        k.copy_(dev(k_new)), v.copy_(dev(v_new))
        graph.replay()
        torch.cuda.synchronize()
        assert t.ref.grow([0, 1], [1, 1]).all() and bool(ok.all())
        for s in (0, 1):
            for pool, x in zip(t.pools[0], (k_new, v_new)):
                pool.write(t.ref.table[s], int(t.ref.lens[s]) - 1, x[s:s + 1])
        t.check_tables(), t.check_pools()
        vmax = float(np.abs(v_new).max()) * 4
        close(out.cpu().numpy(), ko.decode(q.cpu().numpy(), *t.pools[0], t.ref.table, t.ref.lens, [0, 1], 0.8), vmax, 0.8, False)
