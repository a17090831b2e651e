"""The comparison of attention_model.py on the CPU: what it lets pass and what it refuses."""
import numpy as np
import pytest

import attention_model as A


def case(T=5, L=9, H=4, Hkv=2, d=8, seed=0):
    r = np.random.default_rng(seed)
    q, k, v = r.standard_normal((T, H, d)), r.standard_normal((L, Hkv, d)), r.standard_normal((L, Hkv, d))
    return q, k, v, np.full((L, Hkv), 2.0 ** -7)


@pytest.mark.parametrize("causal", [True, False])
def test_accepts_the_definition(causal):
    q, k, v, s = case()
    a = A.attention(q, k, v, s, causal)
    t, h = 3, 2
    n = 9 - 5 + t + 1 if causal else 9
    x = np.exp(k[:n, 1] @ q[t, h] / np.sqrt(8.0))
    assert np.allclose(a["out"][t, h], x @ v[:n, 1] / x.sum(), rtol=1e-12)
    assert np.isclose(a["lse"][t, h], np.log(x.sum()), rtol=1e-12)
    A.check(a["out"], a["lse"], q, k, v, s, causal)


@pytest.mark.parametrize("bad", [np.nan, np.inf, 9.0])
@pytest.mark.parametrize("which", ["out", "lse"])
def test_refuses_what_is_wrong_or_no_number(which, bad):
    q, k, v, s = case()
    a = A.attention(q, k, v, s, True)
    x = dict(out=a["out"].copy(), lse=a["lse"].copy())
    x[which].reshape(-1)[7] = bad
    with pytest.raises(AssertionError):
        A.check(x["out"], x["lse"], q, k, v, s, True)


def test_rows_that_see_nothing():
    q, k, v, s = case(T=5, L=3)
    a = A.attention(q, k, v, s, True)
    assert np.all(a["out"][:2] == 0) and np.all(a["lse"][:2] == -np.inf) and np.isfinite(a["lse"][2:]).all()
    A.check(a["out"], a["lse"], q, k, v, s, True)
    a["out"][0] = 1e-3
    with pytest.raises(AssertionError):
        A.check(a["out"], a["lse"], q, k, v, s, True)


def test_a_hidden_key_widens_nothing():
    q, k, v, s = case()
    was = A.bounds(A.attention(q, k, v, s, True), 8, 9)[0]
    v, s, k = v.copy(), s.copy(), k.copy()
    v[-1] *= 2.0 ** 40
    s[-1] *= 2.0 ** 40
    k[-1] *= 100.0
    now = A.bounds(A.attention(q, k, v, s, True), 8, 9)[0]
    assert np.array_equal(was[:-1], now[:-1]) and (now[-1] > was[-1]).any()
