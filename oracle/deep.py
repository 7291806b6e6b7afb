"""CPU oracle of deep estimators (test infrastructure only; numpy, fp64 throughout): residual layers with a norm in front, and
rows kept in 8 bits for the reverse pass.

    h_1 = [x | means of x] W_0 + b_0
    u_l = act((h_l - mu) r * gamma_l + beta_l), mu and r = 1 / sqrt(var + eps) per graph and group of columns
    h_{l+1} = h_l + [u_l | means of u_l] W_l + b_l
    sum over the rows of each graph, regression network and loss as in oracle/train.py.

The gradient is the hand-derived reverse pass of these formulas.  With `kept` the reverse pass sees every layer's input h_l
(l >= 1) as rounded to 8 bits: what the matrix of layer l and its norm read is formed again from those values.
Pins (tests/test_oracle_deep.py): central differences of the loss for every parameter tensor, closed forms of the norm.
"""
from __future__ import annotations

import math

import numpy as np

from .train import Params, _edges, _mean_of_neighbours, loss_of

ACTS = ("none", "relu", "gelu", "silu")


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z


def act_slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


_erf = np.vectorize(math.erf, otypes=[np.float64])


def keep(x):
    """x as it reads back from 8 bits: per row and 32 columns the smallest power of two whose 127 steps reach the largest value."""
    out = np.zeros_like(x)
    for c in range(0, x.shape[1], 32):
        v = x[:, c:c + 32]
        m = np.abs(v).max(axis=1)
        with np.errstate(divide="ignore"):
            e = np.where(m > 0, np.ceil(np.log2(m / 127.0)), -126.0)
        e = np.clip(np.where((m > 0) & (m <= 127.0 * np.exp2(e - 1)), e - 1, e), -126, 121)
        step = np.exp2(e)[:, None]
        q = np.clip(np.rint(v / step), -127, 127)
        q = np.where((q == 0) & (v != 0), np.sign(v), q)
        out[:, c:c + 32] = q * step
    return out


def norm(h, off, groups, gamma, beta, eps, name):
    """(u, xh, r): r per row and group column as wide as h."""
    n, C = h.shape
    xh, r = np.zeros_like(h), np.zeros_like(h)
    w = C // groups
    for g in range(len(off) - 1):
        lo, hi = int(off[g]), int(off[g + 1])
        if hi == lo:
            continue
        for k in range(groups):
            v = h[lo:hi, k * w:(k + 1) * w]
            s = 1.0 / math.sqrt(v.var() + eps)
            xh[lo:hi, k * w:(k + 1) * w] = (v - v.mean()) * s
            r[lo:hi, k * w:(k + 1) * w] = s
    return act(xh * gamma + beta, name), xh, r


def norm_back(du, xh, r, off, groups, gamma, beta, name):
    """(dh, dgamma, dbeta)"""
    dz = du * act_slope(xh * gamma + beta, name)
    u = dz * gamma
    dh = np.zeros_like(du)
    w = du.shape[1] // groups
    for g in range(len(off) - 1):
        lo, hi = int(off[g]), int(off[g + 1])
        for k in range(groups):
            s = (slice(lo, hi), slice(k * w, (k + 1) * w))
            if hi > lo:
                dh[s] = r[s] * (u[s] - u[s].mean() - xh[s] * (u[s] * xh[s]).mean())
    return dh, (dz * xh).sum(0), dz.sum(0)


def _means(h, c):
    n = h.shape[0]
    return _mean_of_neighbours(h, *c["pin"], n), _mean_of_neighbours(h, *c["pout"], n)


def forward(batch, p: Params, gamma, beta, groups, eps, name):
    """(y [B], cache); gamma, beta [L - 1, H]"""
    n, B = batch.ntot, batch.n_cand
    off = np.asarray(batch.node_off, np.int64)
    c = dict(pin=_edges(batch.in_rowptr, batch.in_col, n), pout=_edges(batch.out_rowptr, batch.out_col, n), off=off)
    x = np.asarray(batch.Xc[:n], np.float64)
    h = np.concatenate([x, *_means(x, c)], axis=1) @ p.W[0] + p.b[0]
    hs = [x, h]
    for l in range(1, len(p.W)):
        u, _, _ = norm(h, off, groups, gamma[l - 1], beta[l - 1], eps, name)
        h = h + np.concatenate([u, *_means(u, c)], axis=1) @ p.W[l] + p.b[l]
        hs.append(h)
    gid = np.repeat(np.arange(B), np.diff(off))
    r = np.zeros((B, h.shape[1]))
    np.add.at(r, gid, h)
    z1 = np.maximum(r @ p.W1 + p.b1, 0.0)
    z2 = np.maximum(z1 @ p.W2 + p.b2, 0.0)
    c.update(hs=hs, gid=gid, r=r, z1=z1, z2=z2)
    return z2 @ p.w3 + p.b3[0], c


def loss_and_gradients(batch, target, p: Params, gamma, beta, groups, eps, name, kept=False, floor=1e-6):
    """(loss, y, gradient as Params, dgamma, dbeta)"""
    y, c = forward(batch, p, gamma, beta, groups, eps, name)
    t = np.asarray(target, np.float64)
    B, n, L = batch.n_cand, batch.ntot, len(p.W)
    yc = np.maximum(y, floor)
    dy = np.where(y > floor, 2.0 / max(B, 1) * (np.log(yc) - np.log(t)) / yc, 0.0)
    dz2 = np.outer(dy, p.w3) * (c["z2"] > 0)
    dz1 = (dz2 @ p.W2.T) * (c["z1"] > 0)
    dh = (dz1 @ p.W1.T)[c["gid"]]
    gW, gb = [None] * L, [None] * L
    dgamma, dbeta = np.zeros_like(np.asarray(gamma, np.float64)), np.zeros_like(np.asarray(beta, np.float64))
    pin, pout = c["pin"], c["pout"]
    indeg = np.maximum(np.bincount(pin[0], minlength=n), 1).astype(np.float64)
    outdeg = np.maximum(np.bincount(pout[0], minlength=n), 1).astype(np.float64)
    for l in range(L - 1, -1, -1):
        h = c["hs"][l]
        if l > 0:
            h = keep(h) if kept else h
            u, xh, r = norm(h, c["off"], groups, gamma[l - 1], beta[l - 1], eps, name)
        else:
            u = h
        gW[l] = np.concatenate([u, *_means(u, c)], axis=1).T @ dh
        gb[l] = dh.sum(axis=0)
        if l == 0:
            break
        d = h.shape[1]
        dA = dh @ p.W[l].T
        du = dA[:, :d].copy()
        np.add.at(du, pin[1], (dA[:, d:2 * d] / indeg[:, None])[pin[0]])
        np.add.at(du, pout[1], (dA[:, 2 * d:] / outdeg[:, None])[pout[0]])
        back, dgamma[l - 1], dbeta[l - 1] = norm_back(du, xh, r, c["off"], groups, gamma[l - 1], beta[l - 1], name)
        dh = dh + back
    g = Params(gW, gb, c["r"].T @ dz1, dz1.sum(0), c["z1"].T @ dz2, dz2.sum(0), c["z2"].T @ dy, np.array([dy.sum()]))
    return loss_of(y, t, floor), y, g, dgamma, dbeta
