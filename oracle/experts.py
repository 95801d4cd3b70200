"""Routing of tokens to experts and back, and layers in 8-bit codes: the
definitions written out in numpy, in float64 (the codes' own float32 roundings
are part of their definition)."""
import numpy as np


def plan(expert, nexpert):
    """(offsets [E + 1], rows [n * k], pos [n, k]) of the choices expert [n, k]."""
    flat = np.asarray(expert).reshape(-1).astype(np.int64)
    offsets = np.zeros(nexpert + 1, np.int64)
    rows, pos = np.full(len(flat), -1, np.int64), np.full(len(flat), -1, np.int64)
    first = 0
    for e in range(nexpert):
        slots = np.flatnonzero(flat == e)
        rows[first:first + len(slots)] = slots
        pos[slots] = first + np.arange(len(slots))
        first += len(slots)
        offsets[e + 1] = first
    return offsets, rows, pos.reshape(np.asarray(expert).shape)


def gather(x, rows, topk, weight=None):
    """[n * k, W]: weight of the slot times the row of its token; zeros without a slot."""
    y = np.zeros((len(rows), x.shape[1]))
    live = rows >= 0
    y[live] = x[rows[live] // topk]
    if weight is not None:
        y[live] *= weight.reshape(-1)[rows[live]][:, None]
    return y


def combine(x, pos, weight=None):
    """([n, W] sums, [n, W] sums of magnitudes) over the kept slots of a token."""
    n, k = pos.shape
    y, mag = np.zeros((n, x.shape[1])), np.zeros((n, x.shape[1]))
    for j in range(k):
        t = np.flatnonzero(pos[:, j] >= 0)
        part = x[pos[t, j]] * (1.0 if weight is None else weight[t, j][:, None])
        y[t] += part
        mag[t] += np.abs(part)
    return y, mag


def combine_backward(x, dy, rows, pos, weight=None):
    """dE/dx [n * k, W]; dE/dweight [n, k] and the sums of magnitudes behind it."""
    n, k = pos.shape
    dw, mag = np.zeros((n, k)), np.zeros((n, k))
    for j in range(k):
        t = np.flatnonzero(pos[:, j] >= 0)
        part = dy[t] * x[pos[t, j]]
        dw[t, j], mag[t, j] = part.sum(1), np.abs(part).sum(1)
    return gather(dy, rows, k, weight), dw, mag


def codes(x):
    """(codes int8 [n, K], scales float32 [n]) of the rows of x."""
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        x = np.asarray(x).astype(np.float32)
        a = np.abs(x).max(1).astype(np.float32) if x.shape[1] else np.zeros(len(x), np.float32)
        finite = np.isfinite(x).all(1)
        live = finite & (a >= np.float32(2.0 ** -100))
        one27 = np.float32(127.0)
        u = np.where(live, one27 / a, np.float32(0)).astype(np.float32)
        q = np.rint(np.where(live[:, None], x, np.float32(0)) * u[:, None]).astype(np.int8)
        scale = np.where(live, a / one27, np.where(finite, np.float32(0), np.float32(np.nan))).astype(np.float32)
    return q, scale


def product(qx, sx, qw, sw, bias=None, groups=None):
    """y [m, n] in float64 of codes qx [m, k], qw [G, n, k], and a bound on the
    magnitudes that its rounding goes by; groups [m]: -1 gives a row of zeros."""
    m, n = len(qx), qw.shape[1]
    groups = np.zeros(m, np.int64) if groups is None else groups
    y, mag = np.zeros((m, n)), np.zeros((m, n))
    for g in np.unique(groups[groups >= 0]):
        at = np.flatnonzero(groups == g)
        # float64 holds these sums exactly
        s = qx[at].astype(np.float64) @ qw[g].astype(np.float64).T
        part = s * sx[at].astype(np.float64)[:, None] * sw[g].astype(np.float64)
        b = 0.0 if bias is None else bias[g].astype(np.float64)
        y[at], mag[at] = part + b, np.abs(part) + np.abs(b)
    return y, mag
