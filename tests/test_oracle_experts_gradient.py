"""What the product of codes is as a layer's gradient: not the derivative of the
layer at fixed codes of its weights, but within the stated share of the norm."""
import numpy as np
import pytest

import oracle.experts as ox


def _back(W, dy):
    """Products of the codes of dy [m, n] and of the transposed weights W [n, k], and the derivative at W's codes."""
    qd, sd = ox.codes(dy)
    qt, st = ox.codes(W.T)
    qw, sw = ox.codes(W)
    return ox.product(qd, sd, qt[None], st[None])[0], dy @ (qw * sw[:, None].astype(np.float64))


@pytest.mark.parametrize("n,k", [(240, 240), (240, 1600), (1024, 1024)])
def test_the_product_approximates_the_derivative(n, k):
    # a code of a normal row is off by s / sqrt(12), about 0.7 to 0.9% of the row's root mean square for rows of
    # 240 to 1,600: the codes of dy, of W and of its transpose each once, 1.2 to 1.5% together
    rng = np.random.default_rng(n + k)
    W, dy = rng.standard_normal((n, k)) / np.sqrt(k), rng.standard_normal((200, n))
    got, derivative = _back(W, dy)
    err = np.linalg.norm(got - derivative) / np.linalg.norm(derivative)
    assert 0.008 < err < 0.02
    # output channels of different sizes: a row of the transposed codes has one scale for all of them
    got, derivative = _back(W * np.exp(rng.standard_normal((n, 1))), dy)
    assert err < np.linalg.norm(got - derivative) / np.linalg.norm(derivative) < 0.06
