"""The decode step over the 8-bit cache, rows that see no position: they are zero whatever the query holds."""
import numpy as np
import pytest
import torch

from paper_2602_05269_amd import binding as hb
from kv8 import Both, dev, half

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("max_pages", [8, 80])                # one part of a sequence, and several with a merge
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_queries_that_are_no_numbers_over_nothing(d, max_pages, bad):
    rng = np.random.default_rng(d + max_pages)
    H, page, lens = 2, 32, [200, 100, 64, 0]
    t = Both(16, page, 4, max_pages, H, d)
    assert (hb.hgf_diff_attention_kv8_workspace_bytes(4, t.pages, H, d) > 0) == (max_pages == 80)
    t.place(lens, rng)
    t.fill(rng)
    t.ref.table[1], t.ref.table[2] = -1, 16                   # (a length, and no page; pages that there are not)
    t.push()
    q = half(rng, 4, 2 * H, d)
    for softcap in (0.0, 30.0):
        clean = hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, 0.8, softcap=softcap)
        odd = q.copy()
        odd[1, 0, 3], odd[1, 2 * H - 1, d - 1], odd[2], odd[3, 1, 0] = bad, bad, bad, bad
        out = hb.hgf_diff_attention_decode_kv8(dev(odd), t.caches[0], t.pages, 0.8, softcap=softcap)
        assert torch.equal(out[0], clean[0]) and bool(clean[0].any())
        assert not clean[1:].any() and torch.equal(out[1:], torch.zeros_like(out[1:]))
