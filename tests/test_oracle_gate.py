"""The plain choice of experts, vectors of ids and 4-bit codes against closed
forms, differences and brute force (no GPU)."""
import itertools

import numpy as np
import pytest

import oracle.gate as og
import oracle.mx4 as om


def test_choice_by_hand():
    z = np.log(np.array([[1.0, 2.0, 4.0, 3.0], [1.0, 1.0, 1.0, 1.0]]))
    e, w = og.choose(z, 2)
    np.testing.assert_array_equal(e, [[2, 3], [0, 1]])
    np.testing.assert_allclose(w, [[0.4, 0.3], [0.25, 0.25]], rtol=1e-15)
    e, w = og.choose(z, 2, renorm=True, scale=7.0)
    np.testing.assert_allclose(w, [[4.0, 3.0], [3.5, 3.5]], rtol=1e-15)
    # the bias chooses and does not weigh
    e, w = og.choose(z, 1, bias=[1.0, 0, 0, 0])
    np.testing.assert_array_equal(e, [[0], [0]])
    np.testing.assert_allclose(w, [[0.1], [0.25]], rtol=1e-15)


def test_groups_by_hand():
    s = np.array([[0.9, 0.1, 0.6, 0.5, 0.55, 0.2]])
    z = np.log(s / (1 - s))
    # groups (0.9 0.1) (0.6 0.5) (0.55 0.2): best two sum to 1.0, 1.1, 0.75
    e, _ = og.choose(z, 2, "sigmoid", groups=3, keep=1, best=2)
    np.testing.assert_array_equal(e, [[2, 3]])
    e, _ = og.choose(z, 3, "sigmoid", groups=3, keep=2, best=2)
    np.testing.assert_array_equal(e, [[0, 2, 3]])
    e, _ = og.choose(z, 2, "sigmoid", groups=3, keep=1, best=1)
    np.testing.assert_array_equal(e, [[0, 1]])
    # closed experts do not count; a group without an open one is never kept
    z[0, [1, 2, 3]] = -np.inf
    e, w = og.choose(z, 3, "sigmoid", groups=3, keep=2, best=2)
    np.testing.assert_array_equal(e, [[0, 4, 5]])
    e, w = og.choose(np.full((1, 4), -np.inf), 3)
    assert (e == -1).all() and (w == 0).all()


@pytest.mark.parametrize("kind,renorm", itertools.product(("softmax", "sigmoid"), (False, True)))
def test_gradient_of_weights_against_differences(kind, renorm):
    rng = np.random.default_rng(3)
    z = rng.standard_normal((5, 7))
    z[1, 2] = -np.inf
    e, _ = og.choose(z, 3, kind)
    d = rng.standard_normal(e.shape)

    def total(z):
        s = og.scores(z, kind)
        w = np.take_along_axis(s, e, 1)
        if renorm:
            w = w / w.sum(1, keepdims=True)
        return 1.7 * (d * w).sum()

    dz, mag = og.choose_backward(z, e, d, kind, renorm, 1.7)
    assert (np.abs(dz) <= mag * (1 + 1e-12) + 1e-300).all()
    for t, i in itertools.product(range(5), range(7)):
        if z[t, i] == -np.inf:
            assert dz[t, i] == 0
            continue
        h, up, dn = 1e-6, z.copy(), z.copy()
        up[t, i] += h
        dn[t, i] -= h
        # truncation h^2 and rounding 2^-53 / h of values around 5
        assert abs((total(up) - total(dn)) / (2 * h) - dz[t, i]) < 5e-9


def test_lookup_and_its_gradient():
    rng = np.random.default_rng(0)
    table, ids = rng.standard_normal((4, 3)), np.array([2, 0, -1, 2, 4, 3])
    y = og.lookup(table, ids, 2.0)
    np.testing.assert_array_equal(y, [2 * table[2], 2 * table[0], np.zeros(3), 2 * table[2], np.zeros(3), 2 * table[3]])
    dy = rng.standard_normal((6, 3))
    d, _ = og.lookup_backward(ids, dy, 4, 2.0)
    # linear: <dy, lookup(v)> = <lookup_backward(dy), v>
    v = rng.standard_normal((4, 3))
    np.testing.assert_allclose((dy * og.lookup(v, ids, 2.0)).sum(), (d * v).sum(), rtol=1e-13)
    assert not d[1].any()


def test_codes_are_the_nearest_values():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, 70)) * np.exp(4 * rng.standard_normal((9, 1)))
    q, e = om.quantise(x)
    assert q.shape == (9, 256) and e.shape == (9, 8) and not q[:, 70:].any() and not e[:, 3:].any()
    v = om.values(q, e)[:, :70]
    x = x.astype(np.float32).astype(np.float64)
    for b in range(3):
        part, got = x[:, 32 * b:32 * b + 32], v[:, 32 * b:32 * b + 32]
        a = np.abs(part).max(1)
        scale = 2.0 ** (e[:, b] - 127.0)
        assert ((a / scale >= 3.5) & (a / scale < 7.0)).all()
        near = np.abs(np.abs(part)[:, :, None] - om.VALUES * scale[:, None, None]).min(2)
        np.testing.assert_allclose(np.abs(got - part), near, rtol=1e-12, atol=1e-300)


def test_codes_at_ties_and_ends():
    block = np.zeros((1, 32))
    block[0, :16] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -2.5, 6.9, 0.24, 0.26, -6.0, 3.0]
    q, e = om.quantise(block)
    assert e[0, 0] == 127
    np.testing.assert_array_equal(om.values(q, e)[0, :16],
                                  [4, 0, 1, 1, 2, 2, 4, 4, 0, -1, -2, 6, 0, 0.5, -6, 3])
    for a, want in ((7.0, 128), (np.nextafter(np.float32(7), np.float32(0)), 127), (3.5, 127), (3.4999998, 126),
                    (2.0 ** -100, 25), (np.nextafter(np.float32(2.0 ** -100), np.float32(0)), 0), (3.4e38, 253),
                    (1e39, 255), (np.nan, 255), (-np.inf, 255), (0.0, 0)):
        block[:] = 0
        block[0, 5] = a
        q, e = om.quantise(block)
        assert e[0, 0] == want, a
        if want in (0, 255):
            assert not q.any()
    codes, scales = om.pack(*om.quantise(np.arange(600.0)[None] + 1))
    assert codes.shape == (1, 384) and scales.shape == (3, 1, 8)
