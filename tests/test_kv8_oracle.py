"""CPU pins of the oracle of the 8-bit cache and the attention over prompts: hand-made values, the attention decode
oracle it has to agree with, and properties that the definitions promise."""
import numpy as np
import pytest

from oracle import hgf_oracle as orc
from oracle import kv8_oracle as ko


def test_block_exponent():
    assert ko.block_exponent(0.0) == -30 and ko.block_exponent(127.0) == 0 and ko.block_exponent(127.5) == 1
    assert ko.block_exponent(2.0 ** -24) == -30 and ko.block_exponent(65504.0) == 10 and ko.block_exponent(1.0) == -6
    for amax in (0.03, 0.9921875, 0.9926, 1.7, 300.0):
        e = ko.block_exponent(amax)
        assert 127 * 2.0 ** e >= amax > 127 * 2.0 ** (e - 1)


def test_codes_are_off_by_less_than_a_step_however_the_tokens_came():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((40, 2, 16)) * np.exp2(rng.integers(-6, 6, (40, 1, 1)))).astype(np.float16)
    whole, single = ko.Pool(3, 16, 2, 16), ko.Pool(3, 16, 2, 16)
    row = [2, 0, 1]
    whole.write(row, 0, x)
    for i in range(40):
        single.write(row, i, x[i:i + 1])
    assert np.array_equal(whole.scale, single.scale)
    for pool, bound in ((whole, 0.5), (single, 1.0)):
        err = np.abs(pool.read(row, range(40)) - x.astype(np.float64))
        step = np.stack([pool.scale[row[p // 16], :, 0] for p in range(40)])[:, :, None]
        assert (err <= bound * step).all()
    assert not np.array_equal(whole.codes, single.codes)


def test_what_int8_cannot_hold():
    pool = ko.Pool(1, 16, 1, 16)
    x = np.zeros((2, 1, 16), dtype=np.float16)
    x[0, 0, 0], x[0, 0, 1], x[1, 0, 2] = np.nan, np.inf, -np.inf
    pool.write([0], 0, x)
    got = pool.read([0], [0, 1, 2, -1])
    assert got[0, 0, 0] == 0 and got[0, 0, 1] == 65536 and got[1, 0, 2] == -65536 and not got[2:].any()


def test_prefill_of_the_last_row_is_the_decode_step():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal(s).astype(np.float16) for s in ((9, 4, 16), (9, 4, 16), (9, 2, 16)))
    full = ko.prefill(q, k, v, [0, 9], 0.3)
    step = orc.diff_attention_decode(q[8:9], k[None], v[None], [9], 0.3)
    assert np.allclose(full[8], step[0], rtol=1e-12, atol=1e-13)
    first = orc.diff_attention_decode(q[:1], k[None], v[None], [1], 0.3)
    assert np.allclose(full[0], first[0]) and np.allclose(full[0], 0.5 * (1 - 0.3) * v[0].astype(np.float64))
    # documents cut the sequence, a prefix opens it
    cut = ko.prefill(q, k, v, [0, 9], 0.3, doc_q=[5] * 4 + [2] * 5, doc_k=[5] * 4 + [2] * 5)
    two = ko.prefill(q, k, v, [0, 4, 9], 0.3)
    assert np.allclose(cut, two)
    assert np.allclose(ko.prefill(q, k, v, [0, 9], 0.3, prefix=[9]), ko.prefill(q, k, v, [0, 9], 0.3, causal=False))
    assert not ko.prefill(q, k, v, [0, 9], 0.3, doc_q=[-1] * 9, doc_k=[-1] * 9).any()
    # a large cap changes nothing, a small one levels the scores; a steep bias leaves the row itself
    assert np.allclose(ko.prefill(q, k, v, [0, 9], 0.3, softcap=1e6), full, atol=1e-9)
    assert np.allclose(ko.prefill(q, k, v, [0, 9], 0.3, slopes=[1e4] * 4), 0.5 * 0.7 * v.astype(np.float64))


def test_pages():
    p = ko.Pages(6, 16, 4, 4)
    assert list(p.grow([0, 1], [20, 16])) == [1, 1]
    assert p.table[0].tolist() == [0, 1, -1, -1] and p.table[1].tolist() == [2, -1, -1, -1] and p.refs.tolist() == [1, 1, 1, 0, 0, 0]
    pairs, ok = p.fork([0, 1], [2, 3])
    assert ok.tolist() == [1, 1] and pairs.tolist() == [[1, 3], [-1, -1]]
    assert p.table[2].tolist() == [0, 3, -1, -1] and p.refs.tolist() == [2, 1, 2, 1, 0, 0]
    # not enough pages for the second request and what follows; a request that needs none; one named twice; too long
    assert list(p.grow([0, 1, 2, 3, 3], [17, 33, 1, 1, 1])) == [1, 0, 1, 0, 0]
    assert list(p.grow([1], [64])) == [0] and list(p.grow([7, -1], [1, 1])) == [0, 0]
    p.free([0, 0, 9])
    assert p.refs.tolist() == [1, 0, 2, 1, 0, 0] and p.lens[0] == 0
    pairs, n, moved = p.compact()
    assert n == 1 and pairs.tolist() == [[3, 1], [-1, -1], [-1, -1]] and moved.tolist() == [0, -1, 2, 1, -1, -1]
    assert p.table[2].tolist() == [0, 1, -1, -1] and p.refs.tolist() == [1, 1, 2, 0, 0, 0]


@pytest.mark.parametrize("seed", [3, 4])
def test_moving_pages_moves_no_content(seed):
    rng = np.random.default_rng(seed)
    p, pool = ko.Pages(20, 16, 6, 5), ko.Pool(20, 16, 1, 16)
    p.grow([0, 1, 2, 3], [30, 17, 48, 5])
    for s in range(4):
        pool.write(p.table[s], 0, rng.standard_normal((p.lens[s], 1, 16)))
    before = {s: pool.read(p.table[s], range(p.lens[s])) for s in (1, 3)}
    p.free([0, 2])
    pairs, n, _ = p.compact()
    pool.copy(pairs[:n])
    for s in (1, 3):
        assert np.array_equal(pool.read(p.table[s], range(p.lens[s])), before[s])
