"""Gradients of rows that are sure of a token, in every form of the backward pass: few rows (dz in two terms), more, several slabs."""
import math

import numpy as np
import pytest
import torch

from head_ops_util import U, tolerances
from paper_2605_08632_b200.api import TokenLogProb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().cpu().double().numpy()


def sure_rows(T, d, V, dtype, seed, rest):
    """Rows one token of which has all but about `rest` of the probability."""
    g = torch.Generator().manual_seed(seed)
    W = (0.02 * torch.randn(V, d, generator=g)).to(dtype)
    token = torch.randint(0, V, (T,), generator=g)
    Wy = W[token].float()
    H = 0.3 * torch.randn(T, d, generator=g)
    up = math.log(V / rest) - (H * Wy).sum(1)
    return (H + Wy * (up / (Wy * Wy).sum(1)).unsqueeze(1)).to(dtype), W, token


FORMS = [(6, 128, 2500, BF, 0), (100, 512, 1111, BF, 0), (200, 256, 3001, BF, 0), (1100, 128, 2500, BF, 0), (600, 128, 2500, BF, 1), (1030, 192, 5003, BF, 3),
         (6, 96, 700, F32, 0), (300, 96, 2500, F32, 1), (130, 320, 3001, F32, 1)]


@pytest.mark.parametrize("T,d,V,dtype,slab_mib", FORMS)
@pytest.mark.parametrize("rest", [1e-2, 1e-5, 1e-6])
@pytest.mark.parametrize("which", ["logp", "entropy", "both"])
def test_gradient_of_sure_rows(T, d, V, dtype, slab_mib, rest, which):
    """dH of each row by itself: its size is that of 1 - p, so what may be off is a share of 1 - p.

    With x_v = log p_v, off by e_x = tol_z (its logit) + tol_l + 8 U |lse| (lse), an entry v other than the sure token's,
    -gl p_v - ge p_v (x_v + entropy), is off by e_x of itself and by |ge| p_v (e_x + e_h), e_h = 4 (1 + log V) (tol_z + tol_l) the
    entropy's error.  The sure token's entry is minus their sum: off by the sum of that, and by V U of the sum of their sizes for the addition.
    A label that is not the sure token has gl more, which no rounding touches but that of the sum with its p.  dH is dz W: the errors times |W|,
    (V + 16) U of the products' sizes for the sum, for bf16 the rounding of dz (2^-16 of each entry in two terms; 2^-8 above 128 rows) and of
    the result (2^-8).
    """
    H, W, token = sure_rows(T, d, V, dtype, 3, rest)
    g = torch.Generator().manual_seed(1)
    y = torch.where(torch.arange(T) % 5 == 4, torch.randint(0, V, (T,), generator=g), token)          # some are sure of another token
    gl = (torch.randn(T, generator=g)) if which != "entropy" else None
    ge = (torch.randn(T, generator=g)) if which != "logp" else None
    bf16 = dtype == BF
    e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=dtype, slab_mib=slab_mib)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    e.forward(dev(H), dev(W), dev(y))
    dH, dW = e.backward(dev(H), dev(W), dev(y) if gl is not None else None, None, dev(gl), dev(ge))
    assert e.bwd_status() == 0
    Hd, Wd = np64(H), np64(W)
    z = Hd @ Wd.T
    m = z.max(1, keepdims=True)
    lse = m[:, 0] + np.log(np.exp(z - m).sum(1))
    x = z - lse[:, None]
    sure = np.arange(T), token.numpy()
    others = np.exp(x)
    others[sure] = 0.0
    left = others.sum(1)
    # what the bounds below need of the inputs: the token has most of the row (its probability is 1 - left)
    assert (left < 0.35).all() and (left > 0).all() and np.median(left) < 50 * rest
    x[sure] = np.log1p(-left)
    p = others.copy()
    p[sure] = 1.0 - left
    h = -(p * x).sum(1)
    a = np.zeros(T) if gl is None else np64(gl)
    b = np.zeros(T) if ge is None else np64(ge)
    dz = -p * (a[:, None] + b[:, None] * (x + h[:, None]))
    terms = p * (np.abs(a)[:, None] + np.abs(b)[:, None] * (np.abs(x) + h[:, None]))
    lab = np.arange(T), y.numpy()
    if gl is not None:
        dz[lab] += a
    terms[lab] += np.abs(a)
    dz[sure] = 0.0
    dz[sure] = -dz.sum(1)
    terms[sure] = 0.0
    tol_z, tol_l = tolerances(Hd, Wd, np.ones(T, bool), z, bf16)
    e_x = tol_z + tol_l + 8 * U * np.abs(lse)[:, None]
    e_h = 4 * (1 + math.log(V)) * (tol_z + tol_l)
    err = e_x * p * (np.abs(a)[:, None] + np.abs(b)[:, None] * (np.abs(x) + h[:, None])) + np.abs(b)[:, None] * p * (e_x + e_h)
    err[lab] += 2 * U * np.abs(a)
    err[sure] = 0.0
    err[sure] = err.sum(1) + V * U * terms.sum(1)
    size = np.abs(dz)
    # the unrounded label entry of 129 to 1024 rows is no worse than the rounded one
    rounding = 0.0 if not bf16 else 2.0 ** -16 if T <= 128 else 2.0 ** -8
    want = dz @ Wd
    tol = (1.02 * err + (rounding + (V + 16) * U) * size) @ np.abs(Wd)
    tol = tol * 1.01 + (2.0 ** -8 if bf16 else 2 * U) * np.abs(want) + 2.0 ** -126
    assert np.all(np.abs(np64(dH) - want) <= tol), float((np.abs(np64(dH) - want) / tol).max())
    # and dW, whose rows sum over the rows of H
    want = dz.T @ Hd
    tol = ((1.02 * err + (rounding + (T + 16) * U) * size).T @ np.abs(Hd)) * 1.01 + (2.0 ** -8 if bf16 else 2 * U) * np.abs(want) + 2.0 ** -126
    assert np.all(np.abs(np64(dW) - want) <= tol), float((np.abs(np64(dW) - want) / tol).max())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_slabs_change_roundings_only(dtype):
    """Rows of every certainty, masked ones and labels that are no tokens, in one slab and in several."""
    T, d, V = 1100, 64, 3000
    H, W, token = sure_rows(T, d, V, dtype, 9, 1.0)
    g = torch.Generator().manual_seed(2)
    H = (H.float() * (0.2 + 1.2 * torch.rand(T, 1, generator=g))).to(dtype)
    y = torch.where(torch.rand(T, generator=g) < 0.1, torch.full_like(token, -100), token).to(DEV)
    valid = (torch.rand(T, generator=g) < 0.8).to(DEV)
    H[(valid == 0).cpu()] = float("nan")
    gl, ge = torch.randn(T, generator=g).to(DEV), torch.randn(T, generator=g).to(DEV)
    out = []
    for slab in (0, 2):
        e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=dtype, slab_mib=slab)
        e.forward(H.to(DEV), W.to(DEV), y, valid)
        out.append([np64(t) for t in e.backward(H.to(DEV), W.to(DEV), y, valid, gl, ge)])
        again = e.backward(H.to(DEV), W.to(DEV), y, valid, gl, ge)
        assert all(np.array_equal(np64(t), o) for t, o in zip(again, out[-1]))
    for a, b in zip(*out):
        assert np.isfinite(a).all()
        assert np.linalg.norm(a - b) <= (2.0 ** -7 if dtype == BF else 1e-5) * np.linalg.norm(a)
    assert not out[0][0][(valid == 0).cpu().numpy()].any()


@pytest.mark.parametrize("dtype,dW_dtype,d,pitch", [(BF, F32, 72, 0), (BF, F32, 64, 8), (BF, BF, 64, 0), (F32, F32, 33, 0), (F32, F32, 64, 4), (F32, F32, 64, 3)])
def test_accumulation_over_slabs(dtype, dW_dtype, d, pitch):
    """An fp32 dW that is added to takes the whole of what the slabs give in one addition; its gaps stay as they are."""
    from paper_2605_08632_b200 import binding as B
    T, V = 700, 2500
    H, W, token = sure_rows(T, d, V, dtype, 4, 1e-2)
    g = torch.Generator().manual_seed(8)
    gl = torch.randn(T, generator=g).to(DEV)
    old = torch.randn(V, d + pitch, generator=g).to(dW_dtype).to(DEV)
    code = {BF: B.CAT_BF16, F32: B.CAT_F32}
    wide = torch.zeros(V, d + pitch, dtype=dtype, device=DEV)
    wide[:, :d] = W.to(DEV)
    shape = B.make_shape(T, d, V, 1, code[dtype], code[dW_dtype], ldW=d + pitch, slab_mib=1)
    e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=dW_dtype)
    r = e.forward(H.to(DEV), W.to(DEV), token.to(DEV))
    n = B.cat_logprob_workspace_bytes(shape, 0, 1)
    ws, dH = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV), torch.empty(T, d, dtype=dtype, device=DEV)
    out = []
    for add in (False, True):
        dW = old.clone()
        B.cat_logprob_bwd(shape, H.to(DEV), wide, token.to(DEV), None, r.lse, None, gl, None, dH, dW, add, ws[:n])
        out.append(dW)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xA5).all()) and int(ws[:4].view(torch.int32)) == 0
    assert all(torch.equal(o[:, d:], old[:, d:]) for o in out)
    if dW_dtype == F32:
        assert torch.equal(out[1][:, :d], old[:, :d] + out[0][:, :d])
    else:      # rounded once; out[0], the same sum without the addend, carries a rounding of its own
        want = np64(old) + np64(out[0])
        assert np.all(np.abs(np64(out[1]) - want) <= 2.0 ** -8 * 1.01 * (np.abs(want) + np.abs(np64(out[0]))))
