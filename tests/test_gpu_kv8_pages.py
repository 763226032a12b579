"""GPU tests of the page tables: tables, lengths, counts and lists against the oracle, number for number."""
import numpy as np
import pytest
import torch

from paper_2602_05269_amd import binding as hb
from kv8 import Both, half, ints

pytestmark = pytest.mark.gpu


def _fork(t, src, dst):
    pairs, ok = hb.hgf_kv8_pages_fork(t.pages, ints(src), ints(dst))
    ref_pairs, ref_ok = t.ref.fork(src, dst)
    assert np.array_equal(pairs.cpu().numpy(), ref_pairs) and np.array_equal(ok.cpu().numpy(), ref_ok)
    for c, pools in zip(t.caches, t.pools):
        hb.hgf_kv8_copy_pages(c, pairs)
        for pool in pools:
            pool.copy(ref_pairs)


def _free(t, seqs):
    hb.hgf_kv8_pages_free(t.pages, ints(seqs))
    t.ref.free(seqs)


def _compact(t):
    pairs, count, moved = hb.hgf_kv8_pages_compact(t.pages)
    ref_pairs, n, ref_moved = t.ref.compact()
    assert np.array_equal(pairs.cpu().numpy(), ref_pairs) and count.item() == n and np.array_equal(moved.cpu().numpy(), ref_moved)
    for c, pools in zip(t.caches, t.pools):
        hb.hgf_kv8_copy_pages(c, pairs, count=count)
        for pool in pools:
            pool.copy(ref_pairs[:n])


def test_requests_that_are_refused():
    t = Both(6, 16, 4, 4, 1, 16)
    t.grow([0, 1], [20, 16])
    _fork(t, [0, 1], [2, 3])
    t.check_tables()
    t.grow([0, 1, 2, 3, 3], [17, 33, 1, 1, 1])            # too few pages; one that needs none; a sequence named twice
    t.grow([1], [64])                                     # beyond the table
    t.grow([1, 0], [2147483647, -1])
    t.grow([4, -1, 2147483647, -2147483648], [1, 1, 1, 1])
    t.check_tables()
    _free(t, [3, 3, 9, -1])
    _fork(t, [0, 9, 1, 1], [0, 3, 2, 17])                 # itself, no such source, a place that is taken, no such place
    t.check_tables()
    _free(t, [2])
    _fork(t, [2, 0, 1], [3, 3, 2])                        # an empty one; its place again; one of whole pages
    t.check_tables()
    _free(t, [0, 1, 2, 3])
    t.check_tables()
    assert int(t.pages.refs.abs().sum()) == 0 and int(t.pages.lens.sum()) == 0
    _compact(t)
    t.check_tables()


@pytest.mark.parametrize("n_pages,n_seqs,max_pages,page", [(1, 2, 1, 16), (37, 11, 6, 16), (1000, 60, 40, 32), (5000, 300, 30, 64), (70001, 1500, 100, 16)])
def test_a_life_of_pages(n_pages, n_seqs, max_pages, page):
    """Random grows, forks, frees and compactions over one state, tables compared after each."""
    rng = np.random.default_rng(n_pages)
    t = Both(1, page, 1, 1, 1, 16)
    t.pages, t.ref = hb.Kv8Pages(n_pages, page, n_seqs, max_pages), type(t.ref)(n_pages, page, n_seqs, max_pages)
    t.caches, t.pools = [], []
    for step in range(12):
        n = int(rng.integers(1, n_seqs + 1))
        kind = step % 4
        some = [int(s) for s in rng.integers(-1, n_seqs + 1, n)]
        if kind == 0:
            t.grow(some, [int(x) for x in rng.integers(-1, max(2, max_pages * page // 3), n)])
        elif kind == 1:
            _fork(t, some, [int(s) for s in rng.integers(-1, n_seqs + 1, n)])
        elif kind == 2:
            _free(t, some[:max(1, n // 2)])
        else:
            _compact(t)
        t.check_tables()


def test_forks_share_and_part():
    """Sequences that share pages grow apart: contents of all of them against the oracle after every step."""
    rng = np.random.default_rng(7)
    H, d, page = 2, 64, 32
    t = Both(64, page, 12, 8, H, d, layers=2)

    def write(seqs, n):
        t.grow(seqs, n)
        for layer in range(2):
            t.append(half(rng, sum(n), 2 * H, d), half(rng, sum(n), H, d), seqs, n, layer=layer)

    def check():
        t.check_tables()
        for layer in range(2):
            t.check_pools(layer)

    write([5, 1], [70, 64])
    _fork(t, [5, 5, 1, 5], [0, 2, 3, 4])
    check()
    write([0, 2, 3, 4, 5, 1], [1, 30, 1, 40, 3, 1])
    check()
    _fork(t, [4, 2], [7, 8])
    _free(t, [5, 2])
    write([7, 8], [1, 1])
    check()
    _compact(t)
    check()
    write([0, 1, 3, 4, 7, 8], [1] * 6)
    check()
    used = int((t.pages.refs > 0).sum())
    assert (t.pages.refs[:used] > 0).all()


def test_largest_tables():
    """As many sequences and requests as there may be, and refs of more pages than a workgroup ranks in one step."""
    S = 16384
    pages = hb.Kv8Pages(1 << 17, 16, S, 8)
    seqs = torch.randperm(S, generator=torch.Generator().manual_seed(1)).int().cuda()
    ok = hb.hgf_kv8_pages_grow(pages, seqs, torch.full((S,), 100, dtype=torch.int32, device="cuda"))
    assert ok.all() and (pages.lens == 100).all() and int(pages.refs.sum()) == 7 * S
    order = pages.table[seqs.long(), :7].flatten()
    assert torch.equal(order, torch.arange(7 * S, dtype=torch.int32, device="cuda"))
    gone = seqs[::2].contiguous()
    hb.hgf_kv8_pages_free(pages, gone)
    pairs, count, moved = hb.hgf_kv8_pages_compact(pages)
    live = 7 * S // 2
    assert int((pages.refs[:live] == 1).sum()) == live and not pages.refs[live:].any()
    assert torch.equal(pages.table[pages.lens > 0][:, :7].flatten().sort().values, torch.arange(live, dtype=torch.int32, device="cuda"))
    n = count.item()
    assert (pairs[:n, 0] >= live).all() and (pairs[:n, 1] < live).all() and (pairs[n:] == -1).all()
    stay = seqs[1::2].contiguous()
    pairs, ok = hb.hgf_kv8_pages_fork(pages, stay, gone)
    assert ok.all() and torch.equal(pairs[:, 1], torch.arange(live, live + S // 2, dtype=torch.int32, device="cuda"))
    assert torch.equal(pages.table[gone.long(), :6], pages.table[stay.long(), :6]) and int(pages.refs.sum()) == 7 * S
