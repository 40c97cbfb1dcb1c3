"""fp64 CPU oracle of the operators on an 8-bit head.

Test infrastructure: plain restatements of the formulas in numpy, sharing no code with the CUDA path.  Whole T x V matrices are
formed, so it is for small sizes.

  quantize      rows as integers and scales, by whole numbers where the inputs allow it
  product       z[t, v] = sx[t] sw[v] sum_i xq[t, i] wq[v, i] + bias[v]
  product_grad  dX = (dY sw) Wq
  cross_entropy nll, lse, 1 - p of the label;   cross_entropy_grad  dX of sum(g nll) and the terms it is summed from
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

__all__ = ["nearest", "quantize", "product", "product_grad", "cross_entropy", "cross_entropy_grad"]


def nearest(x: float, most: float) -> int:
    """127 x / most to the nearest integer, halves to the even one, in exact arithmetic."""
    return round(127 * Fraction(x) / Fraction(most))        # Python rounds fractions half to even


def quantize(X):
    """(xq int64 [rows, d], scale float64 [rows], rounded to binary32)."""
    X = np.asarray(X, np.float64)
    q = np.zeros(X.shape, np.int64)
    scale = np.zeros(X.shape[0])
    for r, x in enumerate(X):
        if not np.all(np.isfinite(x)):
            scale[r] = np.nan
            continue
        most = np.abs(x).max()
        if most == 0.0:
            continue
        scale[r] = np.float64(np.float32(most) / np.float32(127.0))
        t = 127.0 * x / most
        q[r] = np.rint(t)
        for i in np.flatnonzero(np.abs(np.abs(t - np.floor(t)) - 0.5) < 1e-9):
            q[r, i] = nearest(float(x[i]), float(most))
    return q, scale


def product(xq, sx, wq, sw, bias=None):
    # whole numbers below 2^53, whatever the order of the sum: exact
    z = (xq.astype(np.float64) @ wq.astype(np.float64).T) * sx[:, None] * sw[None, :]
    return z if bias is None else z + bias


def product_grad(dY, wq, sw):
    return (dY * sw) @ wq.astype(np.float64)


def _on(labels, valid, T, V):
    live = np.ones(T, bool) if valid is None else np.asarray(valid).astype(bool)
    return live, live & (labels >= 0) & (labels < V)


def cross_entropy(z, labels, valid=None):
    """dict(nll, lse, rest): rest = 1 - p of the label, from the other tokens' sum."""
    T, V = z.shape
    live, ok = _on(labels, valid, T, V)
    nll, lse, rest = np.zeros(T), np.zeros(T), np.zeros(T)
    for r in np.flatnonzero(live):
        m = z[r].max()
        lse[r] = m + np.log(np.exp(z[r] - m).sum())
        if ok[r]:
            others = np.delete(z[r], labels[r]) - z[r, labels[r]]
            if others.size:
                m = others.max()
                o = m + np.log(np.exp(others - m).sum())
                nll[r] = np.logaddexp(0.0, o)
                rest[r] = 1.0 / (1.0 + np.exp(-o))
    return dict(nll=nll, lse=lse, rest=rest, live=live, ok=ok)


def cross_entropy_grad(z, labels, valid, g, wq, sw):
    """(dX, terms): terms [T, V] = dz sw, whose product with wq dX is."""
    T, V = z.shape
    r = cross_entropy(z, labels, valid)
    dz = np.zeros((T, V))
    for t in np.flatnonzero(r["ok"]):
        y = labels[t]
        others = np.array(z[t])
        others[y] = -np.inf
        if V > 1:
            e = np.exp(others - others.max())
            dz[t] = r["rest"][t] * e / e.sum()
            dz[t, y] = -r["rest"][t]
        dz[t] *= g[t]
    terms = dz * sw
    return terms @ wq.astype(np.float64), terms
