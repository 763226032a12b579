"""Capped scores where the two forms of the tanh meet, a little below and above 0.3 of the cap: two groups of keys, one on
either side, whose values are 1 and -1 and whose weights nearly balance, so that the output shows an error of the scores'
difference that fp16 would hide otherwise.

Bound of that difference: tanh from the hardware's exponential and reciprocal, 1 ulp each, is within 1.9e-7 at 0.3 and above;
a series in fp32 within 4e-8 below; and eight roundings of 2^-24 of the score on the way (argument, constants, product with the cap, in
both groups).  A group's share is the logistic function of that difference, whose slope is 1/4 at most, and
the output, half the difference of two shares that add up to one, moves as a share does."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko
from paper_2602_05269_amd import binding as hb
from kv8 import Both, dev, half, ints

pytestmark = pytest.mark.gpu


def _counts(ratio):
    """Numbers of keys whose quotient is nearly `ratio`, together at most 200."""
    best = min((abs(a / (b * ratio) - 1.0), a, b) for b in range(1, 100) for a in [max(1, round(b * ratio))] if a + b <= 200)
    return best[1:]


def _bound(cap, ref, rounded_weights):
    scores = cap * (1.9e-7 + 4e-8) + 0.31 * cap * 8 * 2.0 ** -24 + (2.0 ** -11 if rounded_weights else 0.0)
    return 0.25 * scores + 2.0 ** -11 * np.abs(ref) + 2.0 ** -25


@pytest.mark.parametrize("cap", [50.0, 200.0, 600.0, 1000.0])
@pytest.mark.parametrize("d", [16, 128])
def test_cached_decode(cap, d):
    """Codes 126 and 127 are the two groups, q puts 0.3 of the cap between them."""
    scale = 2.0 ** np.ceil(np.log2(np.sqrt(0.3 * cap * np.sqrt(d)) / 127))
    q0 = float(np.float16(0.3 * cap * np.sqrt(d) / (126.5 * scale)))
    x = q0 * np.array([126.0, 127.0]) * scale / np.sqrt(d)
    assert 0.295 * cap < x[0] < 0.3 * cap < x[1] < 0.305 * cap
    s = cap * np.tanh(x / cap)
    below, above = _counts(np.exp(s[1] - s[0]))
    n = below + above
    k, v = np.zeros((n, 2, d), dtype=np.float16), np.zeros((n, 1, d), dtype=np.float16)
    k[:, 0, 0] = np.where(np.arange(n) < below, 126, 127) * scale
    k[n - 1, 0, 1] = k[0, 0, 1] = 127 * scale                  # (columns that q does not see give every block the scale)
    k[::16, 0, 2] = 127 * scale
    v[:, 0] = np.where(np.arange(n) < below, 1.0, -1.0)[:, None]
    t = Both(16, 16, 1, 16, 1, d)
    t.place([n])
    t.append(k, v, [0], [n])
    assert (t.pools[0][0].scale[t.ref.table[0, :(n + 15) // 16], 0] == scale).all()
    q = np.zeros((1, 2, d), dtype=np.float16)
    q[0, 0, 0] = q0
    ref = ko.decode(q, *t.pools[0], t.ref.table, t.ref.lens, [0], 0.0, cap)
    out = hb.hgf_diff_attention_decode_kv8(dev(q), t.caches[0], t.pages, 0.0, softcap=cap).cpu().numpy().astype(np.float64)
    err, bound = np.abs(out - ref), _bound(cap, ref, False)
    print(f"cap {cap}, d {d}: {below} + {above} keys, {(err / bound).max():.3f} of the bound")
    assert np.abs(ref).max() < 0.01 and (err <= bound).all()


@pytest.mark.parametrize("cap", [2.0 ** 11, 2.0 ** 14, 2.0 ** 17])
@pytest.mark.parametrize("d", [16, 64])
def test_prompts(cap, d):
    """Scores half a unit below and above 0.3 of the cap.  Weights are rounded to fp16, so only large caps show it."""
    q0, k0 = 2.0 ** np.floor(np.log2(np.sqrt(0.3 * cap * np.sqrt(d)))), 0.0
    k0 = float(np.float16(0.3 * cap * np.sqrt(d) / q0))
    at = 0.3 * cap * np.sqrt(d)
    rest = float(np.float16(at - q0 * k0))                    # (what fp16 leaves of the product goes through a second column)
    off = np.float16(0.5 * np.sqrt(d))
    x = (q0 * k0 + rest + np.array([-1.0, 1.0]) * off) / np.sqrt(d)
    assert 0.295 * cap < x[0] < 0.3 * cap < x[1] < 0.305 * cap
    s = cap * np.tanh(x / cap)
    below, above = _counts(np.exp(s[1] - s[0]))
    n = below + above
    order = np.random.default_rng(int(cap)).permutation(n) < below
    q, k, v = np.zeros((1, 2, d), dtype=np.float16), np.zeros((n, 2, d), dtype=np.float16), np.zeros((n, 1, d), dtype=np.float16)
    q[0, 0, :3] = q0, 1.0, 1.0
    k[:, 0, 0], k[:, 0, 1], k[:, 0, 2] = k0, rest, np.where(order, -off, off)
    v[:, 0] = np.where(order, 1.0, -1.0)[:, None]
    ref = ko.prefill(q, k, v, [0, 1], 0.0, cu_k=[0, n], softcap=cap)
    out = hb.hgf_diff_attention_prefill(dev(q), dev(k), dev(v), ints([0, 1]), 0.0, cu_k=ints([0, n]), softcap=cap).cpu().numpy().astype(np.float64)
    err, bound = np.abs(out - ref), _bound(cap, ref, True)
    print(f"cap {cap}, d {d}: {below} + {above} keys, {(err / bound).max():.3f} of the bound")
    assert np.abs(ref).max() < 0.01 and (err <= bound).all()
