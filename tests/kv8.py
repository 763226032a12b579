"""Shared by the tests of the paged 8-bit cache and of the attention over prompts: the same state for the library and for
the oracle, and the tolerances."""
import numpy as np
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def half(rng, *shape, scale=1.0):
    x = rng.standard_normal(shape) * scale
    x[..., ::7] *= 3.0
    return x.astype(np.float16)


class Both:
    """A cache and its pages, on the GPU and in the oracle."""

    def __init__(self, n_pages, page, n_seqs, max_pages, H, d, layers=1):
        self.H, self.d, self.page = H, d, page
        self.pages, self.ref = hb.Kv8Pages(n_pages, page, n_seqs, max_pages), ko.Pages(n_pages, page, n_seqs, max_pages)
        self.caches = [hb.Kv8Cache(n_pages, page, H, d) for _ in range(layers)]
        self.pools = [(ko.Pool(n_pages, page, 2 * H, d), ko.Pool(n_pages, page, H, d)) for _ in range(layers)]

    def place(self, lens, shuffle=None):
        """Pages for sequences 0 .. of these lengths, in a shuffled order if a generator is given."""
        order = np.arange(len(self.ref.refs))
        if shuffle is not None:
            shuffle.shuffle(order)
        at = 0
        for s, n in enumerate(lens):
            k = (n + self.page - 1) // self.page
            self.ref.table[s, :k] = order[at:at + k]
            self.ref.refs[order[at:at + k]] = 1
            self.ref.lens[s] = n
            at += k
        self.push()

    def push(self):
        for name in ("table", "lens", "refs"):
            getattr(self.pages, name).copy_(ints(getattr(self.ref, name)))

    def grow(self, seqs, new):
        ok = hb.hgf_kv8_pages_grow(self.pages, ints(seqs), ints(new))
        assert np.array_equal(ok.cpu().numpy(), self.ref.grow(seqs, new))

    def append(self, k, v, seqs, n, cu=True, layer=0):
        cu_new = ints(np.cumsum([0] + list(n))) if cu else None
        hb.hgf_kv8_append(dev(k), dev(v), self.caches[layer], self.pages, cu_new=cu_new, seqs=ints(seqs))
        at = 0
        for s, m in zip(seqs, n):
            if 0 <= s < len(self.ref.lens):
                length = min(max(int(self.ref.lens[s]), 0), self.ref.table.shape[1] * self.page)
                for pool, x in zip(self.pools[layer], (k, v)):
                    pool.write(self.ref.table[s], length - m, x[at:at + m])
            at += m

    def fill(self, rng, scale=1.0, layer=0):
        """Random contents for all sequences."""
        seqs = [s for s in range(len(self.ref.lens)) if self.ref.lens[s] > 0]
        n = [int(self.ref.lens[s]) for s in seqs]
        self.append(half(rng, sum(n), 2 * self.H, self.d, scale=scale), half(rng, sum(n), self.H, self.d), seqs, n, layer=layer)

    def check_tables(self):
        for name in ("table", "lens", "refs"):
            assert np.array_equal(getattr(self.pages, name).cpu().numpy(), getattr(self.ref, name)), name

    def check_pools(self, layer=0):
        """Every code and scale of the pool, written or not."""
        c = self.caches[layer]
        n, H, nb, d = c.n_pages, self.H, self.page // 16, self.d
        k = c.k_codes.cpu().numpy().transpose(0, 1, 2, 4, 3, 5).reshape(n, 2 * H, self.page, d)
        v = c.v_codes.cpu().numpy().transpose(0, 1, 2, 4, 3).reshape(n, H, self.page, d)
        for got, scale, pool in ((k, c.k_scale, self.pools[layer][0]), (v, c.v_scale, self.pools[layer][1])):
            assert np.array_equal(scale.cpu().numpy().astype(np.float64), pool.scale)
            assert np.array_equal(got, pool.codes)


def close(got, ref, vmax, lam, rounded_weights, what=""):
    """fp16 results against fp64: half a step of the result (2^-11 of it, 2^-25 below the normal numbers); scores of up to 32 in
    fp32 (a dozen roundings of 2^-24 each: 2.3e-5 of every weight, in the sum and in its divisor); and where the weights are
    rounded to fp16, 2^-11 of each, in the sum and in its divisor.  Both branches, halved: (1 + lam) / 2 times 2."""
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref)
    weight = (2.3e-5 + (2.0 ** -11 if rounded_weights else 0.0)) * vmax * (1.0 + abs(lam))
    err = np.abs(got - ref)
    bound = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + weight
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), f"{what}: {(err / bound).max():.3f} of the bound at {np.unravel_index((err / bound).argmax(), err.shape)}"
