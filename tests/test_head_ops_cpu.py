"""The LM-head operators without a GPU: the oracle against hand examples and differences, argument refusals before any launch,
workspace sizes, the binding's structure layout."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import head_ops_oracle as O
from oracle.cat_oracle import cat_forward_backward
from paper_2605_08632_b200 import api
from paper_2605_08632_b200 import binding as B

P = ctypes.c_void_p
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------------------ the oracle
def test_forward_hand_example():
    # two tokens with logits log 3 and 0: probabilities 3/4 and 1/4; a third row masked
    H = np.array([[1.0], [2.0], [np.nan]])
    W = np.array([[np.log(3.0)], [0.0]])
    r = O.logprob_forward(H, W, np.array([1, 0, 0]), np.array([1, 1, 0]), k=3)
    assert np.allclose(r["logp"], [np.log(0.25), np.log(0.9), 0.0])
    assert np.allclose(r["entropy"][0], -(0.75 * np.log(0.75) + 0.25 * np.log(0.25)))
    assert np.allclose(r["lse"], [np.log(4.0), np.log(10.0), 0.0])
    assert r["top_ids"].tolist() == [[0, 1, -1], [0, 1, -1], [-1, -1, -1]]
    assert np.isneginf(r["top_logp"][0, 2]) and np.isneginf(r["top_logp"][2]).all()


def test_ties_go_to_the_lower_id():
    r = O.logprob_forward(np.zeros((1, 2)), np.ones((5, 2)), k=4)
    assert r["top_ids"].tolist() == [[0, 1, 2, 3]] and np.allclose(r["entropy"], np.log(5.0))


@pytest.mark.parametrize("use_l,use_e", [(True, False), (False, True), (True, True)])
def test_backward_against_differences(use_l, use_e):
    rng = np.random.default_rng(0)
    T, d, V = 4, 5, 7
    H, W = rng.normal(size=(T, d)), rng.normal(size=(V, d))
    y, valid = np.array([2, -100, 6, 0]), np.array([1, 1, 1, 0])
    gl, ge = (rng.normal(size=T) if use_l else None), (rng.normal(size=T) if use_e else None)

    def f(H, W):
        r = O.logprob_forward(H, W, y, valid)
        return (gl @ r["logp"] if use_l else 0.0) + (ge @ r["entropy"] if use_e else 0.0)

    dH, dW, *_ = O.logprob_backward(H, W, y, valid, gl, ge)
    for X, D in ((H, dH), (W, dW)):
        for i in np.ndindex(X.shape):
            old, h = X[i], 1e-6
            X[i] = old + h
            up = f(H, W)
            X[i] = old - h
            down = f(H, W)
            X[i] = old
            assert abs((up - down) / (2 * h) - D[i]) < 1e-7
    assert not dH[3].any()


@pytest.mark.parametrize("renorm", [False, True])
def test_topk_kd_against_differences_with_frozen_weights(renorm):
    rng = np.random.default_rng(1)
    K, d, V, k, L = 3, 4, 9, 4, 5
    T = 9
    H, W = rng.normal(size=(T, d)), rng.normal(size=(V, d))
    y = rng.integers(0, V, T)
    ids = rng.integers(0, V, (L, k))
    ids[1, 2:] = -1                          # a short list
    ids[2] = [3, 3, y[2], 3]                 # the same id three times
    ids[3] = -1                              # an empty one
    tl = np.log(rng.dirichlet(np.ones(k), L)) - 0.2
    start = np.array([0, 3, 1])              # block 1 runs past the last position
    args = (y, np.ones(T), K, ids, tl, start, 0.3, renorm)
    base = O.topk_kd(H, W, *args)
    assert base["n_valid"] == 8 and not base["dH"][5].any()
    w, n = base["weight"], base["n_valid"]

    def f(H, W):
        r = O.topk_kd(H, W, *args)
        return float((w * (0.3 * r["ce"] + r["kd"])).sum() / n)

    assert abs(f(H, W) - base["loss"]) < 1e-12
    for X, D in ((H, base["dH"]), (W, base["dW"])):
        for i in np.ndindex(X.shape):
            old, h = X[i], 1e-6
            X[i] = old + h
            up = f(H, W)
            X[i] = old - h
            down = f(H, W)
            X[i] = old
            assert abs((up - down) / (2 * h) - D[i]) < 1e-7


def test_topk_kd_of_a_full_sorted_list_is_the_full_distillation():
    """With every token in the list the two normalisations agree and the loss is Eq. 12's."""
    from oracle.cat_oracle import cat_kd_forward_backward
    rng = np.random.default_rng(2)
    T, K, d, V = 8, 4, 6, 11
    H, W, Ht = rng.normal(size=(T, d)), rng.normal(size=(V, d)), rng.normal(size=(T, d))
    y = rng.integers(0, V, T)
    r = O.logprob_forward(Ht, W, k=V)
    ref, dH, dW = cat_kd_forward_backward(H, W, y, None, K, Ht, W, np.arange(0, T, K), 0.2, conf_source="draft")
    for renorm in (False, True):
        got = O.topk_kd(H, W, y, None, K, r["top_ids"], r["top_logp"], None, 0.2, renorm)
        assert np.isclose(got["loss"], ref["loss"]) and np.allclose(got["dH"], dH) and np.allclose(got["dW"], dW)


def test_topk_kd_without_entries_is_beta_times_cat():
    rng = np.random.default_rng(3)
    H, W, y = rng.normal(size=(6, 4)), rng.normal(size=(7, 4)), rng.integers(0, 7, 6)
    got = O.topk_kd(H, W, y, None, 3, np.full((6, 2), -1), np.zeros((6, 2)), None, 0.5)
    ref, dH, dW = cat_forward_backward(H, W, y, None, 3, g=0.5)
    assert np.isclose(got["loss"], 0.5 * ref["loss"]) and got["loss_kd"] == 0.0
    assert np.allclose(got["dH"], dH) and np.allclose(got["dW"], dW)


# ------------------------------------------------------------------------------ refusals and sizes
OK = P(4096)         # never dereferenced: validation fails first


def _lp_fwd(s, H=OK, W=OK, labels=OK, k=4, logp=OK, lse=OK, entropy=OK, ids=OK, tl=OK, ws=OK, n=1 << 40):
    return B.lib().cat_logprob_fwd(ctypes.byref(s) if s is not None else None, H, W, labels, None, k, logp, lse, entropy, ids, tl, ws, n, None)


def _lp_bwd(s, H=OK, labels=OK, lse=OK, entropy=OK, gl=OK, ge=OK, dH=OK, dW=OK, ws=OK, n=1 << 40):
    return B.lib().cat_logprob_bwd(ctypes.byref(s) if s is not None else None, H, OK, labels, None, lse, entropy, gl, ge, dH, dW, 0, ws, n, None)


def _kd(s, desc, H=OK, labels=OK, ids=OK, tl=OK, start=None, loss=OK, dH=OK, dW=OK, ws=OK, n=1 << 40):
    return B.lib().cat_topk_kd_loss_fwd_bwd(ctypes.byref(s) if s is not None else None, ctypes.byref(desc) if desc is not None else None, H, OK, labels,
                                            None, ids, tl, start, None, None, loss, OK, OK, OK, None, dH, dW, 0, ws, n, None)


def test_logprob_refusals():
    s = B.make_shape(60, 128, 500, 7, B.CAT_BF16)           # T % K != 0: K is not this operator's business
    need = B.cat_logprob_workspace_bytes(s, 4, 0)
    assert need > 0
    assert _lp_fwd(None) == -1 and _lp_fwd(s, H=None) == -1 and _lp_fwd(s, lse=None) == -1 and _lp_fwd(s, ids=None) == -1
    assert _lp_fwd(s, labels=None) == -1 and _lp_fwd(s, logp=None) == -1            # both or neither
    assert _lp_fwd(s, k=-1) == -2 and _lp_fwd(s, k=B.CAT_TOPK_MAX + 1) == -2
    assert _lp_fwd(s, H=P(4104)) == -4 and _lp_fwd(s, ids=P(4100)) == -4 and _lp_fwd(s, entropy=P(4098)) == -4
    assert _lp_fwd(s, n=need - 1) == -5 and _lp_fwd(s, ws=None) == -5 and _lp_fwd(s, ws=P(4096 + 16)) == -5
    assert _lp_fwd(B.make_shape(0, 128, 500, 1, B.CAT_BF16)) == -2
    assert _lp_fwd(B.make_shape(60, 132, 500, 1, B.CAT_BF16)) == -4
    assert _lp_fwd(B.make_shape(60, 128, 500, 1, 5)) == -3
    assert _lp_bwd(None) == -1 and _lp_bwd(s, lse=None) == -1 and _lp_bwd(s, dW=None) == -1
    assert _lp_bwd(s, labels=None) == -1 and _lp_bwd(s, entropy=None) == -1          # needed by the gradient given
    assert _lp_bwd(s, ge=P(4098)) == -4 and _lp_bwd(s, dW=P(4100)) == -4
    assert _lp_bwd(s, n=B.cat_logprob_workspace_bytes(s, 0, 1) - 1) == -5
    for k, which in ((-1, 0), (B.CAT_TOPK_MAX + 1, 0), (0, 2)):
        assert B.cat_logprob_workspace_bytes(s, k, which) == 0


def test_topk_kd_refusals():
    s = B.make_shape(64, 128, 500, 8, B.CAT_BF16)
    desc = B.make_topk_kd_desc(20, 4, 0.1)
    need = B.cat_topk_kd_workspace_bytes(s, desc)
    assert need > 0
    assert _kd(None, desc) == -1 and _kd(s, None) == -1 and _kd(s, desc, H=None) == -1 and _kd(s, desc, ids=None) == -1
    assert _kd(s, desc, labels=None) == -1 and _kd(s, desc, loss=None) == -1
    assert _kd(B.make_shape(60, 128, 500, 8, B.CAT_BF16), desc) == -2
    bad = [dict(L=0, k=4, beta=0.1), dict(L=20, k=0, beta=0.1), dict(L=20, k=B.CAT_TOPK_MAX + 1, beta=0.1), dict(L=20, k=4, beta=-1.0),
           dict(L=20, k=4, beta=float("nan")), dict(L=20, k=4, beta=float("inf")), dict(L=20, k=4, beta=0.1, ld=3), dict(L=1 << 31, k=4, beta=0.1)]
    for kw in bad:
        d = B.make_topk_kd_desc(**kw)
        assert _kd(s, d) == -2 and B.cat_topk_kd_workspace_bytes(s, d) == 0, kw
    d = B.make_topk_kd_desc(20, 4, 0.1)
    d.renormalize = 2
    assert _kd(s, d) == -2
    assert _kd(s, desc, ids=P(4100)) == -4 and _kd(s, desc, start=P(4100)) == -4 and _kd(s, desc, dH=P(4104)) == -4
    assert _kd(s, desc, n=need - 1) == -5 and _kd(s, desc, ws=P(4097)) == -5


def test_workspaces_stay_bounded():
    assert ctypes.sizeof(B.cat_topk_kd_desc) == 32
    big = B.make_shape(65536, 2048, 128256, 8, B.CAT_BF16)
    logits = 65536 * 128256 * 2
    assert B.cat_logprob_workspace_bytes(big, 0, 0) < 64 << 20                       # no alternatives: no slab
    assert B.cat_logprob_workspace_bytes(big, 20, 0) < 0.25 * logits
    assert B.cat_topk_kd_workspace_bytes(big, B.make_topk_kd_desc(8199, 64, 0.1)) < 0.25 * logits
    one = B.make_shape(1, 2048, 128256, 1, B.CAT_BF16)
    assert B.cat_logprob_workspace_bytes(one, 20, 0) < 1 << 20
    small = B.make_shape(65536, 2048, 128256, 8, B.CAT_BF16, slab_mib=256)
    assert B.cat_logprob_workspace_bytes(small, 20, 0) < 300 << 20


@pytest.mark.parametrize("pair", ["0", "1"])
def test_one_slab_has_room_for_dz_in_two_terms(pair):
    """Up to 128 rows, dz stands in the slab (and H in its copy) as two sets of rows, each rounded up to 32; the kernels without CTA
    pairs plan in tiles of 128 rows, so that a slab of one tile would be too low.  A slab is no taller than its batch otherwise."""
    code = ("from paper_2605_08632_b200 import binding as B\n"
            "for T, K in ((1, 1), (66, 33), (70, 1), (128, 8), (128, 128)):\n"
            "    s = B.make_shape(T, 512, 20000, K, B.CAT_BF16, B.CAT_BF16)\n"
            "    print(T, B.cat_topk_kd_workspace_bytes(s, B.make_topk_kd_desc(T, 4, 0.1)), B.cat_logprob_workspace_bytes(s, 0, 1))\n")
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, CAT_LOSS_CTA_PAIR=pair), capture_output=True, text=True, check=True)
    for line in out.stdout.splitlines():
        T, kd, bwd = (int(x) for x in line.split())
        rows = 2 * ((T + 31) // 32 * 32)
        need = rows * (20000 * 2 + 512 * 2) + rows * 512 * 4           # slab, copy of H, dH's parts
        assert need <= kd < need + (40 << 20), line
        assert need <= bwd < need + (40 << 20), line


def test_python_layer_refuses_what_the_kernels_would_misread():
    dev = torch.device("cpu")
    x = torch.zeros(4, 8)
    api._check("x", x, (4, 8), torch.float32, dev)
    with pytest.raises(TypeError):
        api._check("x", x, (4, 8), torch.bfloat16, dev)
    with pytest.raises(ValueError):
        api._check("x", x, (4, 9), torch.float32, dev)
    with pytest.raises(ValueError):
        api._check("x", x, (4, 8), torch.float32, torch.device("cuda", 0))
    with pytest.raises(ValueError):
        api._check("x", x.t(), (8, 4), torch.float32, dev, rows_only=True)
    wide = torch.zeros(4, 16)[:, :8]
    api._check("x", wide, (4, 8), torch.float32, dev, rows_only=True)
    with pytest.raises(ValueError):
        api._check("x", wide, (4, 8), torch.float32, dev)
    with pytest.raises(ValueError):
        api._check("x", torch.zeros(8).expand(4, 8), (4, 8), torch.float32, dev, rows_only=True)
    assert api._mask(torch.ones(3, dtype=torch.bool)).dtype == torch.uint8
    assert api._pitch(torch.zeros(1, 16)[:, :8]) == 8
