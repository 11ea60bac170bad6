"""Routing by scores and its gradient in 64 bits, one token at a time (host,
numpy), from the definition."""
from __future__ import annotations

import numpy as np


def scores(z, sigmoid):
    z = np.asarray(z, np.float64)
    if sigmoid:
        e = np.exp(-np.abs(z))
        return np.where(z >= 0, 1 / (1 + e), e / (1 + e))
    top = z.max()
    if top == -np.inf:
        return np.zeros_like(z)
    with np.errstate(invalid="ignore"):
        e = np.exp(z - top)
    return e / e.sum()


def route_token(z, bias, k, sigmoid, groups, top_groups, pair, renorm, scale):
    """(ids, weights) of one token's logits z."""
    z = np.asarray(z, np.float64)
    E = len(z)
    s = scores(z, sigmoid)
    broken = np.isnan(z).any() or (not sigmoid and (z == np.inf).any())
    if broken:
        order = np.where(np.isnan(z), np.inf, z)
        left = [e for e in range(E) if order[e] > -np.inf]
    else:
        with np.errstate(invalid="ignore"):
            c = s + (0 if bias is None else np.asarray(bias, np.float64))
        on = (z > -np.inf) & (c > -np.inf)
        order = z if bias is None else c
        left = [e for e in range(E) if on[e]]
        if groups > 1:
            size = E // groups
            value = []
            for g in range(groups):
                mine = sorted((c[e] for e in range(g * size, (g + 1) * size) if on[e]),
                              reverse=True)
                value.append(-np.inf if not mine else sum(mine[:2]) if pair else mine[0])
            kept = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
            left = [e for e in left if e // size in kept]
    ids = sorted(left, key=lambda e: (-order[e], e))[:k]
    if broken:
        w = np.full(len(ids), np.nan)
    elif not renorm:
        w = s[ids]
    elif sigmoid:  # in logarithms: no sum of 0
        lg = np.array([-np.logaddexp(0.0, -z[e]) for e in ids])
        w = np.exp(lg - lg.max()) if len(ids) else lg
        w = w / w.sum()
    else:
        w = scores(z[ids], False) if len(ids) else np.zeros(0)
    fill = k - len(ids)
    out = np.concatenate([w * scale, np.full(fill, np.nan if broken else 0.0)])
    return np.array(ids + [-1] * fill, np.int32), out


def route(z, bias, k, **rules):
    got = [route_token(row, bias, k, **rules) for row in z]
    return (np.array([g[0] for g in got]).reshape(-1, k),
            np.array([g[1] for g in got]).reshape(-1, k))


def weights_of(z, ids, sigmoid, renorm, scale):
    """The weights of given experts as a function of z (what the gradient is of)."""
    s = scores(z, sigmoid)[ids]
    return scale * (s / s.sum() if renorm else s)


def route_backward(z, ids, dw, sigmoid, renorm, scale):
    """dz [T][E] through the Jacobian of each step."""
    z = np.asarray(z, np.float64)
    dz = np.zeros_like(z)
    for t in range(len(z)):
        on = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < z.shape[1]]
        if not on:
            continue
        at = ids[t, on]
        g = np.asarray(dw, np.float64)[t, on] * scale
        s = scores(z[t], sigmoid)
        if renorm:
            total = s[at].sum()
            g = (np.eye(len(on)) / total - np.outer(np.ones(len(on)), s[at]) / total ** 2) @ g
        ds = np.zeros(z.shape[1])
        np.add.at(ds, at, g)
        dz[t] = ds * s * (1 - s) if sigmoid else s * ds - s * (s @ ds)
    return dz
