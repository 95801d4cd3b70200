"""The plain routing and 8-bit layer against their definitions slot by slot,
and their gradients against differences."""
import numpy as np
import pytest

import oracle.experts as ox


def _case(n, k, E, W, seed=0):
    rng = np.random.default_rng(seed)
    e = rng.integers(-1, E + 1, (n, k))                     # E and -1: dropped
    return rng, e, rng.standard_normal((n, W)), rng.random((n, k))


@pytest.mark.parametrize("n,k,E", [(1, 1, 1), (7, 2, 3), (40, 3, 5), (5, 4, 9)])
def test_plan_is_a_stable_sort(n, k, E):
    _, e, _, _ = _case(n, k, E, 1)
    off, rows, pos = ox.plan(e, E)
    flat = e.reshape(-1)
    kept = [s for s in range(n * k) if 0 <= flat[s] < E]
    want = sorted(kept, key=lambda s: (flat[s], s))
    assert list(rows[:off[E]]) == want and (rows[off[E]:] == -1).all()
    for s in range(n * k):
        r = pos.reshape(-1)[s]
        assert (rows[r] == s and off[flat[s]] <= r < off[flat[s] + 1]) if s in kept else r == -1


def test_combine_brings_back_what_gather_sent():
    _, e, x, w = _case(30, 3, 4, 6)
    off, rows, pos = ox.plan(e, 4)
    y, _ = ox.combine(ox.gather(x, rows, 3), pos, w)
    np.testing.assert_allclose(y, x * (w * (pos >= 0)).sum(1)[:, None], rtol=1e-14)


def test_gradients_against_differences():
    rng, e, x, w = _case(9, 2, 3, 5, seed=3)
    off, rows, pos = ox.plan(e, 3)
    z, dy = rng.standard_normal((18, 5)), rng.standard_normal((9, 5))
    value = lambda z, w: float((ox.combine(z, pos, w)[0] * dy).sum())
    dz, dw, _ = ox.combine_backward(z, dy, rows, pos, w)
    h = 1e-6
    for a, d in ((z, dz), (w, dw)):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = value(z, w)
            a[i] = keep - h
            down = value(z, w)
            a[i] = keep
            assert abs((up - down) / (2 * h) - d[i]) < 1e-8
    # the gather's gradient is the combine without weights
    g = rng.standard_normal((18, 5))
    dx, _ = ox.combine(g, pos)
    sent = lambda x: float((ox.gather(x, rows, 2) * g).sum())
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = sent(x)
        x[i] = keep - h
        down = sent(x)
        x[i] = keep
        assert abs((up - down) / (2 * h) - dx[i]) < 1e-8


def test_codes_are_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 33)) * np.exp(4 * rng.standard_normal((50, 1)))
    x[3] = 0
    x[4] *= 1e-35
    x[5, 7] = np.inf
    x[6, 2] = np.nan
    q, s = ox.codes(x)
    assert s[3] == 0 and s[4] == 0 and np.isnan(s[5]) and np.isnan(s[6]) and not q[[3, 4, 5, 6]].any()
    ok = np.r_[0:3, 7:50]
    assert (np.abs(q[ok]).max(1) == 127).all()
    assert (np.abs(q[ok] * s[ok, None].astype(float) - x[ok]) <= s[ok, None] * 0.50001).all()


def test_product_of_codes_by_loops():
    rng = np.random.default_rng(2)
    qx, qw = rng.integers(-127, 128, (5, 9)), rng.integers(-128, 128, (2, 4, 9))
    sx, sw, b = rng.random(5), rng.random((2, 4)), rng.standard_normal((2, 4))
    groups = np.array([0, 1, 1, -1, 0])
    y, _ = ox.product(qx, sx, qw, sw, b, groups)
    for r in range(5):
        for c in range(4):
            g = groups[r]
            want = 0.0 if g < 0 else sum(int(qx[r, i]) * int(qw[g, c, i]) for i in range(9)) * sx[r] * sw[g, c] + b[g, c]
            assert abs(y[r, c] - want) <= 1e-14 * abs(want)
