"""fp64 CPU oracle of the LM-head operators beside the CAT loss.

Test infrastructure, like cat_oracle: plain restatements of the formulas in numpy float64, sharing no code with the CUDA
path.  Whole T x V matrices are formed, so it is for small sizes.

  logprob_forward    log-sum-exp, log probability of a given token, entropy, top alternatives of softmax(H W^T)
  logprob_backward   gradients of sum(gl * logp) + sum(ge * entropy)
  topk_kd            CAT-weighted beta * CE + KD against a teacher's stored top lists, and its gradients
"""
from __future__ import annotations

import numpy as np

from .cat_oracle import _as_f64, _as_i64, cat_weights, fixed_decay_weights

__all__ = ["logprob_forward", "logprob_backward", "topk_kd"]


def _mask(valid, T):
    if valid is None:
        return np.ones(T, bool)
    v = valid.detach().to("cpu").numpy() if hasattr(valid, "detach") else np.asarray(valid)
    return v.astype(bool)


def _logits(H, W, on):
    """Logits of the rows that take part; the others may hold anything and get zeros."""
    H, W = _as_f64(H).copy(), _as_f64(W)
    H[~on] = 0.0
    return H, W, H @ W.T


def _log_softmax(z):
    m = z.max(axis=1, keepdims=True)
    lse = m + np.log(np.exp(z - m).sum(axis=1, keepdims=True))
    return lse[:, 0], z - lse


def logprob_forward(H, W, labels=None, valid=None, k=0):
    T, V = H.shape[0], W.shape[0]
    on = _mask(valid, T)
    _, _, z = _logits(H, W, on)
    lse, lp = _log_softmax(z)
    p = np.exp(lp)
    out = dict(z=z, lse=np.where(on, lse, 0.0), entropy=np.where(on, -(p * lp).sum(axis=1), 0.0), on=on)
    if labels is not None:
        y = _as_i64(labels)
        known = on & (y >= 0) & (y < V)
        out["logp"] = np.where(known, lp[np.arange(T), np.clip(y, 0, V - 1)], 0.0)
        out["known"] = known
    ids, tl = np.full((T, k), -1, np.int64), np.full((T, k), -np.inf)
    for r in range(T):
        if on[r]:
            order = np.lexsort((np.arange(V), -z[r]))[:k]       # falling logit, then rising id
            ids[r, :len(order)], tl[r, :len(order)] = order, lp[r, order]
    out["top_ids"], out["top_logp"] = ids, tl
    return out


def logprob_backward(H, W, labels, valid, gl=None, ge=None):
    """(dH, dW, terms, coef): for error bounds, terms[r, v] is the sum of the absolute values of what makes up dz[r, v], and
    coef[r, v] = |ge| p what multiplies the difference log p + entropy, whose error is absolute."""
    T, V = H.shape[0], W.shape[0]
    on = _mask(valid, T)
    Hd, Wd, z = _logits(H, W, on)
    _, lp = _log_softmax(z)
    p = np.exp(lp)
    dz, terms, coef = np.zeros_like(z), np.zeros_like(z), np.zeros_like(z)
    if gl is not None:
        y = _as_i64(labels)
        known = on & (y >= 0) & (y < V)
        g = np.where(known, _as_f64(gl), 0.0)
        dz -= g[:, None] * p
        terms += np.abs(g)[:, None] * p
        dz[np.arange(T), np.clip(y, 0, V - 1)] += g
        terms[np.arange(T), np.clip(y, 0, V - 1)] += np.abs(g)
    if ge is not None:
        g = np.where(on, _as_f64(ge), 0.0)
        ent = -(p * lp).sum(axis=1)
        dz -= g[:, None] * p * (lp + ent[:, None])
        terms += np.abs(g)[:, None] * p * (np.abs(lp) + ent[:, None])
        coef += np.abs(g)[:, None] * p
    return dz @ Wd, dz.T @ Hd, terms, coef


def topk_kd(H, W, labels, valid, K, top_ids, top_logp, block_start=None, beta=0.1, renormalize=True, conf_ext=None, g=1.0,
            fixed_decay_gamma=None):
    T, V = H.shape[0], W.shape[0]
    ids, tl = _as_i64(top_ids), _as_f64(top_logp)
    L = ids.shape[0]
    y = _as_i64(labels)
    pos = np.arange(T) if block_start is None else (_as_i64(block_start)[:, None] + np.arange(K)).reshape(-1)
    ok = _mask(valid, T) & (y >= 0) & (y < V) & (pos >= 0) & (pos < L)
    Hd, Wd, z = _logits(H, W, ok)
    lse, lq = _log_softmax(z)
    ce, kd = np.zeros(T), np.zeros(T)
    dz, terms = np.zeros((T, V)), np.zeros((T, V))
    for r in np.nonzero(ok)[0]:
        entries = [(int(i), float(t)) for i, t in zip(ids[pos[r]], tl[pos[r]]) if 0 <= i < V and t > -np.inf]
        if renormalize and entries:
            t = np.array([e[1] for e in entries])
            t = t - (t.max() + np.log(np.exp(t - t.max()).sum()))
            entries = [(e[0], float(x)) for e, x in zip(entries, t)]
        ce[r] = -lq[r, y[r]]
        mass = sum(np.exp(t) for _, t in entries)
        kd[r] = sum(np.exp(t) * (t - lq[r, i]) for i, t in entries)
        dz[r] = (beta + mass) * np.exp(lq[r])
        terms[r] = dz[r]
        dz[r, y[r]] -= beta
        terms[r, y[r]] += beta
        for i, t in entries:
            dz[r, i] -= np.exp(t)
            terms[r, i] += np.exp(t)
    conf = np.where(ok, np.exp(-ce) if conf_ext is None else _as_f64(conf_ext), 1.0)
    weight = cat_weights(conf, ok, K) if fixed_decay_gamma is None else fixed_decay_weights(fixed_decay_gamma, ok, K)
    n = max(1, int(ok.sum()))
    a, b = float((weight * ce).sum() / n), float((weight * kd).sum() / n)
    scale = (g * weight / n)[:, None]
    dz *= scale
    terms *= np.abs(scale)
    return dict(loss=beta * a + b, loss_ce=a, loss_kd=b, lse=lse, conf=conf, weight=weight, ok=ok, n_valid=int(ok.sum()), z=z, ce=ce,
                kd=kd, dH=dz @ Wd, dW=dz.T @ Hd, terms=terms)
