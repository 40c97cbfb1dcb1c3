"""Inputs and error bounds of the 8-bit head's GPU tests, from the arithmetic of the kernels.

u = 2^-24 is half a step of binary32 relative to the value, e = 2^-8 of bfloat16, h = 2^-11 of half precision.
  logits   the integer sum is exact; its conversion and two scales are three roundings: 3 u |z|; the bias one more of the result.
  lse      of the other tokens: exponents a (t sx) with one more rounding and that of log2 e's constant, 5 u |z|; V exponentials of 4 u each added in
           chains of V / 16 + 64, in units of the running sum; the exponent's own rounding, u times its size: tol_l = u (V / 16 + 64 + 4 spread).
  nll      d nll / d logits sums to 1 - p_y on either side: (1 - p_y) (err of lse + 5 u |z_y|), and its own rounding.
  dX       terms exp(z - o) sw: relative h + the exponent's error (that of the logits, of o, which comes from lse and nll in binary32, 4 u (|lse| + 1)
           + 2 u / rest-free), or half a step of the smallest half precision number, 2^-25, in units where the largest scale is 2^14; the fp32 sum of
           the contraction 2 u per addition (16 products each); the result e.
"""
import numpy as np
import torch

U, E, H16 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11


def np64(t):
    return t.detach().cpu().double().numpy()


def head(V, d, seed=0, spread=1.0):
    """Integers and scales as a checkpoint holds them (with -128 among them), scales over `spread` powers of ten."""
    g = torch.Generator().manual_seed(seed)
    q = (40.0 * torch.randn(V, d, generator=g)).round().clamp(-128, 127).to(torch.int8)
    scale = (0.02 / 40.0) * 10.0 ** (spread * (torch.rand(V, generator=g) - 0.5))
    return q, scale


def tokens(T, d, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, d, generator=g) * (0.5 + torch.rand(T, 1, generator=g))).to(dtype)


def sure(X, q, scale, y, most, seed=2):
    """Rows of X whose label's logit is raised by up to `most`."""
    g = torch.Generator().manual_seed(seed)
    W = q.float() * scale.unsqueeze(1)
    Wy = W[y.clamp(0, q.shape[0] - 1)]
    amount = most * torch.rand(X.shape[0], generator=g) * (torch.rand(X.shape[0], generator=g) < 0.6)
    return (X.float() + Wy * (amount / (Wy * Wy).sum(1).clamp(min=1e-6)).unsqueeze(1)).to(X.dtype)


def check_ce(nll, lse, z, ref):
    live, ok = ref["live"], ref["ok"]
    V = z.shape[1]
    zl = np.where(live[:, None], z, 0.0)
    big = np.abs(zl).max(axis=1)
    tol = U * (5 * big + V / 16 + 64 + 4 * (zl.max(axis=1) - zl.min(axis=1)))
    assert np.all(np.abs(lse - ref["lse"])[live] <= (tol + 2 * U * np.abs(ref["lse"]))[live])
    assert not lse[~live].any() and not nll[~ok].any()
    assert np.all(np.abs(nll - ref["nll"])[ok] <= (ref["rest"] * (1.01 * tol + 5 * U * big) + 2 * U * ref["nll"])[ok] + 2.0 ** -149)


def check_ce_grad(dX, z, ref, terms, want, g, q, scale):
    q, V, d = q.astype(np.float64), q.shape[0], q.shape[1]
    ok = ref["ok"]
    big = np.where(ok, np.abs(np.where(ok[:, None], z, 0.0)).max(axis=1), 0.0)
    tol = U * (10 * big + V / 8 + 128 + 8 * 2 * big + 8 * (np.abs(ref["lse"]) + 1))
    mag = np.abs(terms) @ np.abs(q)
    factor = np.abs(np.where(ok, g, 0.0)) * ref["rest"]
    floor = (factor * np.abs(scale).max() * 2.0 ** -38)[:, None] * np.abs(q).sum(axis=0)
    off = (1.01 * tol[:, None] + 1.01 * H16 + 2 * U * (V / 16 + 24)) * mag + floor
    bound = off + E * (np.abs(want) + off) + 2.0 ** -126
    err = np.abs(dX - want)
    assert np.all(err <= bound), (float((err / bound).max()), np.unravel_index(int((err / bound).argmax()), err.shape))
    assert not dX[~ok].any()
    if np.linalg.norm(want) > 0:
        assert np.linalg.norm(err) <= E * np.linalg.norm(want) + np.linalg.norm(off)
