"""The 64-bit forms of the token-sequence operators against differences, special cases and each other (no GPU)."""
import numpy as np
import pytest

from tests import sequence_oracle as S


@pytest.mark.parametrize("causal,nq,nk", [(False, 5, 7), (True, 6, 6), (True, 3, 7), (True, 7, 3)])
def test_gradients_match_differences(causal, nq, nk):
    rng = np.random.default_rng(3)
    q, k, v, do = (rng.standard_normal((n, 5)) for n in (nq, nk, nk, nq))
    scale = 0.7
    r = S.attention(q, k, v, scale, causal, "f32", do)
    h = 1e-5

    def loss(q, k, v):
        return float((S.attention(q, k, v, scale, causal, "f32")["out"][0] * do).sum())

    for name, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        x = [q, k, v]
        for _ in range(3):
            step = rng.standard_normal(x[i].shape)
            up, down = list(x), list(x)
            up[i], down[i] = x[i] + h * step, x[i] - h * step
            # central differences: h^2 / 6 of the third derivative (below 1e3 here) and 2^-52 of the loss over h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - float((r[name][0] * step).sum())) < 1e-7


def test_rows_that_see_nothing_and_masked_values():
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((n, 4)) for n in (5, 2, 2))
    r = S.attention(q, k, v, 1.0, True, "f32", rng.standard_normal((5, 4)))
    assert np.all(r["out"][0][:3] == 0) and np.all(np.isneginf(r["lse"][0][:3])) and np.all(r["dq"][0][:3] == 0)
    assert np.allclose(r["out"][0][3], v[0])
    v2 = v.copy()
    v2[1] = np.nan  # only the last row sees it
    r2 = S.attention(q, k, v2, 1.0, True, "f32")
    assert np.allclose(r2["out"][0][:4], r["out"][0][:4]) and np.isnan(r2["out"][0][4]).all()


def test_rotary_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(5)
    f = S.frequencies([4])
    x, y = rng.standard_normal((2, 1, 1, 10))
    for inter in (False, True):
        dots = []
        for shift in (0, 1000):
            a = S.rotary(x, np.array([[3 + shift]]), [4], f, inter)
            b = S.rotary(y, np.array([[11 + shift]]), [4], f, inter)
            assert np.isclose(np.linalg.norm(a), np.linalg.norm(x)) and np.array_equal(a[..., 8:], x[..., 8:])
            dots.append((a * b).sum())
        assert np.isclose(dots[0], dots[1])
        back = S.rotary(S.rotary(x, np.array([[7]]), [4], f, inter), np.array([[7]]), [4], f, inter, backward=True)
        assert np.allclose(back, x)
