"""Top-list distillation where draft and teacher are both sure of a token: dz is then a difference of what is left, 1 - q and 1 - p."""
import math

import numpy as np
import pytest
import torch

from head_ops_util import U, tolerances
from paper_2605_08632_b200.api import CatLoss
from test_logprob_sure_rows_gpu import sure_rows

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("T,d,V,dtype,slab_mib", [(6, 128, 2500, BF, 0), (200, 256, 3001, BF, 0), (600, 128, 2500, BF, 1), (6, 96, 700, F32, 0), (300, 96, 2500, F32, 1)])
@pytest.mark.parametrize("rest", [1e-5, 1e-6])
@pytest.mark.parametrize("teacher", ["label alone", "nearly sure", "of another"])
def test_gradient_of_sure_rows(T, d, V, dtype, slab_mib, rest, teacher):
    """Weights 1 (conf_ext, K = 1), so dz = (1/N) ((beta + mass) q - beta [y] - sum p_i [id_i]).

    An entry other than the sure token's is off by the share e = tol_z + tol_l + 8 U |lse| of its softmax, for bf16 above 0 with the steps' 2^-10
    (1.01), and by 16 U of its list probability (exp and the sum of k terms); the sure token's, minus their sum, by the sum of that and V U of their
    sizes.  Where the teacher is sure of another token the label's entry is no small difference, and 16 U of its terms are off.  dH is dz W, as in
    the test of the log probabilities.
    """
    H, W, token = sure_rows(T, d, V, dtype, 3, rest)
    bf16, beta, k = dtype == BF, 0.25, 4
    g = torch.Generator().manual_seed(6)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(T)])
    clash = (ids == token[:, None])
    ids[clash] = (ids[clash] + 1) % V
    tl = torch.full((T, k), math.log(rest / 8))
    if teacher == "label alone":
        ids[:, 0], tl[:, 0] = token, 0.0
        ids[:, 1:] = -1
    else:
        if teacher == "nearly sure":
            ids[:, 2] = token
        tl[:, 2] = math.log1p(-rest)
    eng = CatLoss(T, d, V, 1, dtype=dtype, dW_dtype=dtype, slab_mib=slab_mib)
    loss3, dH, _ = eng.topk_kd_forward_backward(H.to(DEV), W.to(DEV), token.to(DEV), None, ids.to(DEV), tl.to(DEV), beta=beta, renormalize=False,
                                                conf_ext=torch.ones(T, device=DEV))
    assert eng.topk_kd_status() == 0
    z = np64(H) @ np64(W).T
    m = z.max(1, keepdims=True)
    lse = m[:, 0] + np.log(np.exp(z - m).sum(1))
    sure = np.arange(T), token.numpy()
    q = np.exp(z - lse[:, None])
    q[sure] = 0.0
    left = q.sum(1)
    assert (left < 2.0 ** -10).mean() > 0.9 and (left > 0).all()
    p = np.where(ids.numpy() >= 0, np.exp(np64(tl)), 0.0)
    mass = p.sum(1)
    lists = np.zeros((T, V))
    for i in range(k):
        np.add.at(lists, (np.arange(T), np.where(ids.numpy()[:, i] >= 0, ids.numpy()[:, i], 0)), p[:, i])
    dz = (beta + mass)[:, None] * q - lists
    tol_z, tol_l = tolerances(np64(H), np64(W), np.ones(T, bool), z, bf16)
    e = tol_z + tol_l + 8 * U * np.abs(lse)[:, None] + (1.01 * 2.0 ** -10 if bf16 else 0.0)
    err = e * (beta + mass)[:, None] * q + 16 * U * lists
    dz[sure] = 0.0
    dz[sure] = -dz.sum(1)
    err[sure] = 0.0
    err[sure] = err.sum(1) + V * U * (np.abs(dz).sum(1))
    # rows with more left than 2^-10 keep the difference itself, off by the error of lse and 16 U of its terms
    far = left >= 2.0 ** -10 * 0.98
    direct = (e.max(1) - (1.01 * 2.0 ** -10 if bf16 else 0.0) + 16 * U) * (2 * beta + 2 * mass)
    err[sure] = np.where(far, np.maximum(err[sure], direct), err[sure])
    rounding = 0.0 if not bf16 else 2.0 ** -16 if T <= 128 else 2.0 ** -8
    want = dz @ np64(W) / T
    tol = (1.02 * err + (rounding + (V + 16) * U) * np.abs(dz)) @ np.abs(np64(W)) / T
    tol = tol * 1.01 + (2.0 ** -8 if bf16 else 4 * U) * np.abs(want) + 2.0 ** -126
    off = np.abs(np64(dH) - want)
    assert np.all(off <= tol), float((off / tol).max())
