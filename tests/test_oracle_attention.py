"""Pins of the attention and paged-row oracle (no GPU): closed forms of the softmax,
the byte order of a page, and the coding's own error."""

import numpy as np
import pytest

from oracle import attention as at


def test_equal_scores_average_what_is_seen():
    q = np.zeros((3, 2, 4))
    k = np.random.default_rng(0).normal(size=(5, 1, 4))
    v = np.arange(20.0).reshape(5, 1, 4)
    r = at.attend(q, k, v, 0.5)
    for i in range(3):  # row i of 3 sees the first i + 3 of 5 keys
        assert np.allclose(r["out"][i, 0], v[:i + 3, 0].mean(0))
        assert np.allclose(r["lse"][i], np.log(i + 3))


def test_one_far_key_takes_all_and_empty_rows_are_zero():
    q = np.ones((2, 1, 4))
    k = np.zeros((2, 1, 4))
    k[1] = 100.0
    v = np.array([[[1.0] * 4], [[2.0] * 4]])
    r = at.attend(q, k, v, 1.0, causal=False)
    assert np.array_equal(r["out"][0, 0], [2.0] * 4) and np.isclose(r["lse"][0, 0], 400.0)
    r = at.attend(np.ones((3, 1, 4)), k[:1], v[:1], 1.0)   # three rows, one key: two see none
    assert np.array_equal(r["out"][:2], np.zeros((2, 1, 4)))
    assert np.all(np.isneginf(r["lse"][:2])) and np.array_equal(r["out"][2, 0], [1.0] * 4)


@pytest.mark.parametrize("d,P", [(64, 32), (128, 64)])
def test_page_order_is_a_permutation_and_comes_back(d, P):
    assert sorted(at.key_nibble(d, np.arange(d))) == list(range(d))
    got = sorted(at.value_nibble(d, t, e) for t in range(32) for e in range(d))
    assert got == list(range(32 * d))
    rng = np.random.default_rng(1)
    H = 3
    c = rng.integers(0, 16, size=(2, P, H, d))
    s = at._bf16(rng.random((2, P, H, d // 32)))
    o = at._bf16(rng.normal(size=(2, P, H, d // 32)))
    page = at.pack_page(c, s, o, H, d, P)
    assert page.size == at.page_bytes(H, d, P)
    c2, s2, o2 = at.unpack_page(page, H, d, P)
    assert np.array_equal(c, c2) and np.array_equal(s, s2) and np.array_equal(o, o2)


def test_codes_by_hand():
    x = np.zeros((32,), np.float32)
    x[:16] = np.arange(16)          # spread 15: s = 1, o = 0
    x[16] = 2.5                     # halfway: the even code
    x[17] = 3.5
    c, s, o = at.quantise(x)
    assert s[0] == 1 and o[0] == 0
    assert list(c[:16]) == list(range(16)) and c[16] == 2 and c[17] == 4
    c, s, o = at.quantise(np.full(32, -7.0, np.float32))
    assert s[0] == 0 and o[0] == -7 and not c.any()
    x[3] = np.nan
    c, s, o = at.quantise(x)
    assert np.isnan(s[0]) and np.isnan(o[0]) and not c.any()
    x[3] = np.inf
    assert np.isnan(at.quantise(x)[1][0])


def test_coding_error_is_half_a_step():
    x = np.random.default_rng(2).normal(size=(50, 128)).astype(np.float32)
    c, s, o = at.quantise(x)
    g = x.reshape(50, 4, 32)
    lo, hi = g.min(-1), g.max(-1)
    # half a step, and at the ends what the rounding of o and s leaves
    lim = s / 2 + 2.0 ** -8 * (np.abs(lo) + (hi - lo)) * (1 + 2.0 ** -20)
    err = np.abs(at.dequantise(c, s, o).reshape(50, 4, 32) - g)
    assert (err <= lim[..., None]).all()
