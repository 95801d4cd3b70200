"""The choice of experts and vectors of ids: the definitions written out in
numpy, in float64."""
import numpy as np


def scores(z, kind):
    """Softmax over the open experts (z > -inf) or sigmoids; [n, E] float64."""
    z = np.asarray(z, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "sigmoid":
            return 1.0 / (1.0 + np.exp(-z))
        top = z.max(1, keepdims=True)
        p = np.exp(z - np.where(top == -np.inf, 0.0, top))
        total = p.sum(1, keepdims=True)
        return p / np.where(total == 0, 1.0, total)


def choose(z, topk, kind="softmax", bias=None, groups=1, keep=1, best=1, renorm=False, scale=1.0):
    """(expert [n, k], weight [n, k]) token by token, the best expert first."""
    z = np.asarray(z, np.float64)
    n, E = z.shape
    s = scores(z, kind)
    expert, weight = np.full((n, topk), -1), np.zeros((n, topk))
    per = E // groups
    for t in range(n):
        # with neither bias nor groups the order is that of the logits (whose scores may round to equal numbers)
        c = z[t] if bias is None and groups == 1 else s[t] + (0.0 if bias is None else np.asarray(bias, np.float64))
        if np.isnan(c + s[t]).any():
            expert[t], weight[t] = np.arange(topk), np.nan
            continue
        open_ = (z[t] != -np.inf) & (c != -np.inf)
        if groups > 1:
            value = []
            for g in range(groups):
                mine = sorted(c[g * per:(g + 1) * per][open_[g * per:(g + 1) * per]], reverse=True)[:best]
                value.append(sum(mine) if mine else -np.inf)
            order = sorted((g for g in range(groups) if value[g] > -np.inf), key=lambda g: (-value[g], g))[:keep]
            open_ &= np.isin(np.arange(E) // per, order)
        chosen = sorted(np.flatnonzero(open_), key=lambda e: (-c[e], e))[:topk]
        w = s[t, chosen]
        if renorm:
            w = w / w.sum() if w.sum() > 0 else np.zeros_like(w)
        expert[t, :len(chosen)], weight[t, :len(chosen)] = chosen, scale * w
    return expert, weight


def choose_backward(z, expert, dweight, kind="softmax", renorm=False, scale=1.0):
    """(dlogits, magnitudes that its terms have) [n, E] of sum(dweight * weight) at the given experts."""
    z, d = np.asarray(z, np.float64), np.asarray(dweight, np.float64)
    n, E = z.shape
    s = scores(z, kind)
    dz, mag = np.zeros((n, E)), np.zeros((n, E))
    for t in range(n):
        live = [j for j in range(expert.shape[1]) if 0 <= expert[t, j] < E]
        e = expert[t, live]
        mine, g = s[t, e], scale * d[t, live]
        size = np.abs(g)
        if renorm:
            S = mine.sum()
            if not S > 0:
                continue
            g, size = (g - (g * mine).sum() / S) / S, (size + (size * mine).sum() / S) / S
        ds, ms = np.zeros(E), np.zeros(E)
        np.add.at(ds, e, g)
        np.add.at(ms, e, size)
        if kind == "sigmoid":
            dz[t], mag[t] = ds * s[t] * (1 - s[t]), ms * s[t]
        else:
            dz[t], mag[t] = s[t] * (ds - (g * mine).sum()), s[t] * (ms + (size * mine).sum())
        dz[t, z[t] == -np.inf] = 0.0
    return dz, mag


def lookup(table, ids, scale=1.0):
    """[n, W]; zeros for an id that is none."""
    live = (ids >= 0) & (ids < len(table))
    return np.where(live[:, None], scale * table[np.where(live, ids, 0)], 0.0)


def lookup_backward(ids, dy, nid, scale=1.0):
    """(dtable [nid, W], magnitudes): scale times the sum over each id's tokens."""
    d, mag = np.zeros((nid, dy.shape[1])), np.zeros((nid, dy.shape[1]))
    live = (ids >= 0) & (ids < nid)
    np.add.at(d, ids[live], dy[live])
    np.add.at(mag, ids[live], np.abs(dy[live]))
    return scale * d, abs(scale) * mag
