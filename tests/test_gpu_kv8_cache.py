"""GPU tests of the 8-bit cache: appending (every code and scale of the pool against the oracle, bit for bit), gathering,
copying pages."""
import numpy as np
import pytest
import torch

from paper_2602_05269_amd import binding as hb
from kv8 import Both, dev, half, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,H,page", [(16, 3, 16), (32, 2, 64), (64, 5, 32), (128, 1, 256), (64, 1, 16), (128, 3, 64), (16, 9, 128), (32, 9, 32)])
def test_append_in_pieces(d, H, page):
    """Ragged pieces, one token at a time among them, that begin and end anywhere in blocks and pages; larger ones later."""
    rng = np.random.default_rng(d + H + page)
    t = Both(40, page, 5, 12, H, d)
    seqs = [3, 0, 4]
    for step, n in enumerate([[17, 1, 33], [1, 1, 1], [1, 20, 15], [48, 1, 1], [1, 1, 1], [5, 16, 64]]):
        t.grow(seqs, n)
        scale = [1.0, 4.0, 0.5, 2.0, 60.0, 1.0][step]
        t.append(half(rng, sum(n), 2 * H, d, scale=scale), half(rng, sum(n), H, d, scale=scale), seqs, n, cu=n != [1, 1, 1])
        t.check_pools()
    t.check_tables()
    # everything back, in another order, more rows asked for than there are, and rows that nobody asked for
    lens = [int(t.ref.lens[s]) for s in seqs]
    asked = [lens[0], 7, lens[2] + 20]
    cu = np.cumsum([2] + asked)
    T = int(cu[-1]) + 3
    k = torch.full((T, 2 * H, d), 5.0, dtype=torch.float16, device="cuda")
    v = torch.full((T, H, d), 5.0, dtype=torch.float16, device="cuda")
    hb.hgf_kv8_gather(t.caches[0], t.pages, ints(cu), k, v, seqs=ints(seqs))
    for got, pool in ((k, t.pools[0][0]), (v, t.pools[0][1])):
        got = got.cpu().numpy()
        for b, s in enumerate(seqs):
            ref = pool.read(t.ref.table[s], range(lens[b] - asked[b], lens[b]))
            assert np.array_equal(got[cu[b]:cu[b + 1]].astype(np.float64), np.clip(ref, -65504, 65504).astype(np.float16).astype(np.float64))
        assert (got[:2] == 5.0).all() and (got[cu[-1]:] == 5.0).all()


def test_append_of_what_int8_cannot_hold_and_of_nothing():
    rng = np.random.default_rng(1)
    t = Both(4, 16, 2, 2, 2, 32)
    t.grow([0, 1], [20, 3])
    k, v = half(rng, 23, 4, 32), half(rng, 23, 2, 32)
    k[3, 1, 5], k[4, 1, 5], v[7, 0, 2], v[19, 1, 1] = np.nan, np.inf, -np.inf, np.nan
    k[16:20, 2], v[:16, 1], v[20:, 0] = 0, 0, 2.0 ** -24
    t.append(k, v, [0, 1], [20, 3])
    t.check_pools()
    before = [x.clone() for x in (t.caches[0].k_codes, t.caches[0].v_codes, t.caches[0].k_scale, t.caches[0].v_scale)]
    # sequences without new rows, sequences that do not exist, offsets beyond the tensor or falling
    one = dev(half(rng, 1, 4, 32)), dev(half(rng, 1, 2, 32))
    hb.hgf_kv8_append(*one, t.caches[0], t.pages, cu_new=ints([0, 0, 0]), seqs=ints([0, 1]))
    hb.hgf_kv8_append(*one, t.caches[0], t.pages, cu_new=ints([0, 1]), seqs=ints([2]))
    hb.hgf_kv8_append(*one, t.caches[0], t.pages, cu_new=ints([0, 1]), seqs=ints([-1]))
    hb.hgf_kv8_append(*one, t.caches[0], t.pages, cu_new=ints([1, 0]), seqs=ints([0]))
    hb.hgf_kv8_append(*one, t.caches[0], t.pages, cu_new=ints([1, 9]), seqs=ints([0]))
    for x, y in zip(before, (t.caches[0].k_codes, t.caches[0].v_codes, t.caches[0].k_scale, t.caches[0].v_scale)):
        assert torch.equal(x, y)


def test_append_of_more_tokens_than_positions_and_to_missing_pages():
    """The first tokens of a list that is longer than its sequence are dropped; positions without a page are not written."""
    rng = np.random.default_rng(2)
    t = Both(6, 16, 3, 4, 1, 64)
    t.place([40, 25, 9])
    t.ref.table[0, 1], t.ref.table[1, 0] = -1, 6
    t.push()
    n = [50, 25, 9]
    k, v = half(rng, 84, 2, 64), half(rng, 84, 1, 64)
    t.append(k, v, [0, 1, 2], n)
    t.check_pools()
    kk = torch.empty((40, 2, 64), dtype=torch.float16, device="cuda")
    vv = torch.empty((40, 1, 64), dtype=torch.float16, device="cuda")
    hb.hgf_kv8_gather(t.caches[0], t.pages, ints([0, 40]), kk, vv, seqs=ints([0]))
    assert not kk[16:32].any() and not vv[16:32].any()
    assert np.array_equal(vv.cpu().numpy().astype(np.float64), t.pools[0][1].read(t.ref.table[0], range(40)))


@pytest.mark.parametrize("B", [64, 65, 300, 4200])
def test_append_of_many_rows(B):
    """More batch rows than one, two steps of the search over offsets take, most of them empty."""
    rng = np.random.default_rng(3)
    t = Both(3 * B, 16, B, 3, 1, 16)
    n = [int(x) for x in rng.integers(0, 4, B) * rng.integers(0, 12, B)]
    seqs = [int(s) for s in rng.permutation(B)]
    t.grow(seqs, n)
    t.append(half(rng, sum(n), 2, 16), half(rng, sum(n), 1, 16), seqs, n)
    t.check_pools()
    k = torch.empty((sum(n), 2, 16), dtype=torch.float16, device="cuda")
    v = torch.empty((sum(n), 1, 16), dtype=torch.float16, device="cuda")
    hb.hgf_kv8_gather(t.caches[0], t.pages, ints(np.cumsum([0] + n)), k, v, seqs=ints(seqs))
    ref = np.concatenate([t.pools[0][0].read(t.ref.table[s], range(m)) for s, m in zip(seqs, n)])
    assert np.array_equal(k.cpu().numpy().astype(np.float64), ref)


@pytest.mark.parametrize("d,H,page", [(16, 1, 16), (64, 3, 64), (128, 5, 256)])
def test_copy_pages(d, H, page):
    rng = np.random.default_rng(page)
    t = Both(9, page, 2, 4, H, d)
    t.place([4 * page, 3 * page - 5], rng)
    t.fill(rng)
    free = [p for p in range(9) if t.ref.refs[p] == 0]
    used = [int(p) for p in t.ref.table[0]]
    pairs = [[used[0], free[0]], [-1, -1], [used[1], free[1]], [used[2], 9], [9, used[2]], [used[3], used[3]]]
    hb.hgf_kv8_copy_pages(t.caches[0], ints(pairs))
    for pool in t.pools[0]:
        pool.copy(pairs)
    t.check_pools()
    # a count on the device: beyond the list, in it, below zero
    for count, m in ((5, 1), (1, 1), (0, 0), (-3, 0)):
        more = [[used[count % 4], free[0]]]
        hb.hgf_kv8_copy_pages(t.caches[0], ints(more), count=ints([count]))
        for pool in t.pools[0]:
            pool.copy(more[:m])
        t.check_pools()


def test_pools_beyond_32_bit_offsets():
    """Pages that lie more than 4 GiB into the pool."""
    H, d, page = 16, 128, 256
    n_pages = (1 << 32) // (2 * H * page * d) + 3
    pages = hb.Kv8Pages(n_pages, page, 1, 2)
    cache = hb.Kv8Cache(n_pages, page, H, d)
    pages.table[0, 0], pages.table[0, 1] = n_pages - 1, 0
    pages.lens[0] = page + 40
    rng = np.random.default_rng(4)
    k, v = dev(half(rng, page + 40, 2 * H, d)), dev(half(rng, page + 40, H, d))
    hb.hgf_kv8_append(k, v, cache, pages, cu_new=ints([0, page + 40]))
    kk, vv = torch.empty_like(k), torch.empty_like(v)
    hb.hgf_kv8_gather(cache, pages, ints([0, page + 40]), kk, vv)
    for x, y in ((k, kk), (v, vv)):
        assert (x.float() - y.float()).abs().max() <= 0.51 * x.float().abs().max() / 63.5
    hb.hgf_kv8_copy_pages(cache, ints([[n_pages - 1, n_pages - 2]]))
    assert torch.equal(cache.k_codes[n_pages - 2], cache.k_codes[n_pages - 1]) and torch.equal(cache.v_scale[n_pages - 2], cache.v_scale[n_pages - 1])
    q = dev(half(rng, 1, 2 * H, d))
    out = hb.hgf_diff_attention_decode_kv8(q, cache, pages, 0.8)
    pages.table[0, 0] = n_pages - 2
    assert torch.equal(out, hb.hgf_diff_attention_decode_kv8(q, cache, pages, 0.8)) and out.abs().max() > 0
