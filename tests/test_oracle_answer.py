"""The fp64 definitions of the weights of keys, the choice and the sampling, by hand."""

import numpy as np
import pytest

from oracle import answer, attention as at


@pytest.mark.parametrize("causal", [True, False])
def test_weights_are_the_attention_s_softmax(causal):
    """With the lse of the same rows the weights of a row sum to 1, and times the values they
    are the attention's result."""
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    ref = at.attend(q, k, v, 0.3, causal)
    r = answer.key_weights(q, k, ref["lse"], 0.3, causal)
    np.testing.assert_allclose(r["w"].sum(1), 3 * 2, rtol=1e-12)   # 3 rows, 2 heads of a group
    one = answer.key_weights(q[:, :1], k[:, :1], ref["lse"][:, :1], 0.3, causal)["w"][0]
    np.testing.assert_allclose(one @ v[:, 0], ref["out"][:, 0].sum(0), rtol=1e-12)


def test_weights_of_prior_and_masks():
    q, k = np.zeros((1, 1, 4)), np.zeros((3, 1, 4))
    r = answer.key_weights(q, k, np.full((1, 1), np.log(2.0)), 1.0, True, seen=[True, False, True],
                           prior=np.array([[1.0, 2.0, 4.0]]), decay=0.5)
    np.testing.assert_allclose(r["w"], [[1.0, 1.0, 2.5]])
    r = answer.key_weights(np.zeros((3, 1, 4)), k[:1], np.zeros((3, 1)), 1.0)   # two rows see no key
    np.testing.assert_allclose(r["w"], [[1.0]])


def test_choice():
    w = [0.5, np.nan, 2.0, -0.0, 0.0, 2.0, np.inf, -1.0]
    pick = lambda *a: list(answer.evict_select(np.array(w), *a))  # noqa: E731
    assert pick(8) == list(range(8)) and pick(0) == []
    assert pick(1) == [6] and pick(2) == [2, 6] and pick(3) == [2, 5, 6]
    assert pick(5) == [0, 2, 3, 5, 6]                     # the zeros are equal: by number
    assert pick(7) == [0, 2, 3, 4, 5, 6, 7]               # the NaN goes first
    assert pick(3, 2, 1) == [0, 1, 7] and pick(4, 2, 1) == [0, 1, 6, 7]


def test_sample():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    t = lambda u, **kw: answer.sample(x, u, **kw)  # noqa: E731
    assert [t(u)["token"] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.95)] == [1, 1, 3, 3, 2, 0]
    assert t(0.5)["logprob"] == pytest.approx(np.log(0.3))
    assert list(t(0.0, top_k=2)["kept"]) == [1, 3] and t(0.0, top_k=2)["logprob"] == pytest.approx(np.log(4 / 7))
    assert list(t(0.0, top_p=0.5)["kept"]) == [1, 3] and list(t(0.0, top_p=0.0)["kept"]) == [1]
    assert list(t(0.0, min_p=0.6)["kept"]) == [1, 3] and list(t(0.0, min_p=9.0)["kept"]) == [1]
    assert t(0.99, temperature=0.0)["token"] == 1 and t(0.99, temperature=0.0)["logprob"] == 0
    assert answer.sample([1.0, 1.0], 0.6)["token"] == 1 and answer.sample([-np.inf, 0.0], 0.0)["token"] == 1
    for bad in ([np.nan, 1.0], [-np.inf, -np.inf]):
        assert answer.sample(bad, 0.5)["token"] == -1
    assert t(0.5, temperature=np.inf)["token"] == -1 and t(2.0)["token"] == 0 and t(np.nan)["token"] == 1
