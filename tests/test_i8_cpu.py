"""The 8-bit head without a GPU: the oracle against hand examples and differences, refusals before any launch, workspace sizes, layouts."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import i8_oracle as O
from paper_2605_08632_b200 import api
from paper_2605_08632_b200 import binding as B

P = ctypes.c_void_p
OK = P(4096)            # never dereferenced: what is tested fails first


# ------------------------------------------------------------------------------ the oracle
def test_quantize_hand_examples():
    q, s = O.quantize(np.array([[127.0, 0.5, 1.5, -2.5, -127.0], [1.0, 0.5, -0.5, 0.25, 0.0], [0.0] * 5, [1.0, np.inf, 0, 0, 0], [np.nan, 1, 0, 0, 0]]))
    assert q[0].tolist() == [127, 0, 2, -2, -127] and s[0] == 1.0           # halves to the even integer
    assert q[1].tolist() == [127, 64, -64, 32, 0]                             # 63.5 -> 64, 31.75 -> 32
    assert s[2] == 0.0 and not q[2:].any() and np.isnan(s[3:]).all()


def test_quantize_is_within_half_a_step():
    rng = np.random.default_rng(0)
    X = rng.normal(size=(20, 50)).astype(np.float32)
    q, s = O.quantize(X)
    assert np.all(np.abs(q) <= 127) and np.all(np.abs(q).max(axis=1) == 127)
    for r in range(20):
        most = Fraction(float(np.abs(X[r]).max()))
        assert all(abs(127 * Fraction(float(x)) / most - int(n)) <= Fraction(1, 2) for x, n in zip(X[r], q[r]))


def test_cross_entropy_hand_example():
    z = np.array([[np.log(3.0), 0.0], [np.log(3.0), 0.0], [0.0, 800.0], [5.0, 5.0]])
    r = O.cross_entropy(z, np.array([0, 1, 1, -100]), np.array([1, 1, 1, 1]))
    assert np.allclose(r["nll"], [np.log(4 / 3), np.log(4.0), 0.0, 0.0]) and np.allclose(r["lse"], [np.log(4.0)] * 2 + [800.0, 5 + np.log(2.0)])
    assert np.allclose(r["rest"], [0.25, 0.75, 0.0, 0.0])
    assert O.cross_entropy(z, np.array([0, 0, 0, 0]), np.array([0, 0, 0, 0]))["lse"].tolist() == [0.0] * 4


def test_gradients_against_differences():
    """With the tokens' values X in the place of scale * integers, as the straight-through gradient takes them."""
    rng = np.random.default_rng(1)
    T, d, V = 4, 5, 7
    X, wq, sw = rng.normal(size=(T, d)), rng.integers(-128, 128, size=(V, d)), rng.random(V) * 0.02
    y, valid, g = np.array([2, -100, 6, 0]), np.array([1, 1, 1, 0]), rng.normal(size=T)
    dY = rng.normal(size=(T, V))

    def logits(X):
        return X @ (wq * sw[:, None]).T

    for f, D in ((lambda X: g @ O.cross_entropy(logits(X), y, valid)["nll"], O.cross_entropy_grad(logits(X), y, valid, g, wq, sw)[0]),
                 (lambda X: (dY * logits(X)).sum(), O.product_grad(dY, wq, sw))):
        for i in np.ndindex(X.shape):
            old, h = X[i], 1e-6
            X[i] = old + h
            up = f(X)
            X[i] = old - h
            down = f(X)
            X[i] = old
            assert abs((up - down) / (2 * h) - D[i]) < 1e-6


# ------------------------------------------------------------------------------ refusals
def shape(**kw):
    base = dict(T=64, d=128, V=512)
    base.update(kw)
    return B.make_i8_shape(**base)


BAD = [(dict(T=0), -2), (dict(d=0), -2), (dict(V=0), -2), (dict(d=65544), -2), (dict(ldX=127), -2), (dict(ldW=120), -2), (dict(slab_mib=-1), -2),
       (dict(x_dtype=7), -3), (dict(ldW=136), -4)]
BAD_LINEAR = [(dict(ldY=511), -2), (dict(ldY=513), -4), (dict(ldY=516), -4), (dict(y_dtype=5), -3), (dict(ldY=514, y_dtype=B.CAT_F32), -4)]
BAD_BACK = [(dict(x_dtype=B.CAT_F32), -3), (dict(lddX=127), -2), (dict(lddX=132), -4), (dict(d=124, lddX=128), -4)]


def calls(s, n):
    L = B.lib()
    a = ctypes.byref(s)
    return [lambda: L.cat_i8_linear_fwd(a, OK, OK, OK, OK, OK, OK, n, None), lambda: L.cat_i8_linear_bwd(a, OK, OK, OK, OK, OK, n, None),
            lambda: L.cat_i8_ce_fwd(a, OK, OK, OK, OK, OK, OK, OK, OK, n, None), lambda: L.cat_i8_ce_bwd(a, *[OK] * 9, OK, n, None)]


@pytest.mark.parametrize("which,kw,code", [(w, kw, c) for w in range(4) for kw, c in BAD] + [(w, kw, c) for w in (0, 1) for kw, c in BAD_LINEAR]
                         + [(w, kw, c) for w in (1, 3) for kw, c in BAD_BACK] + [(1, dict(y_dtype=B.CAT_F32), -3)])
def test_bad_shapes_are_refused_on_the_host(which, kw, code):
    s = shape(**kw)
    assert B.cat_i8_workspace_bytes(s, which) == 0
    assert calls(s, 1 << 40)[which]() == code


def test_shapes_that_only_other_passes_refuse():
    assert B.cat_i8_workspace_bytes(shape(ldY=511), 2) > 0 and B.cat_i8_workspace_bytes(shape(d=124, lddX=124), 0) > 0
    assert B.cat_i8_workspace_bytes(shape(d=13), 2) > 0 and B.cat_i8_workspace_bytes(shape(), 4) == 0 == B.cat_i8_workspace_bytes(shape(), -1)


def test_null_alignment_and_workspace_errors():
    L, s = B.lib(), shape()
    a = ctypes.byref(s)
    entries = [(L.cat_i8_linear_fwd, 5, {3}, {0: 2, 1: 16, 2: 4, 3: 4, 4: 16}), (L.cat_i8_linear_bwd, 4, set(), {0: 16, 1: 16, 2: 4, 3: 16}),
               (L.cat_i8_ce_fwd, 7, {4}, {0: 2, 1: 16, 2: 4, 3: 8, 5: 4, 6: 4}),
               (L.cat_i8_ce_bwd, 9, {4}, {0: 2, 1: 16, 2: 4, 3: 8, 5: 4, 6: 4, 7: 4, 8: 16})]
    for which, (f, n, optional, aligned) in enumerate(entries):
        need = B.cat_i8_workspace_bytes(s, which)
        for i in range(n):
            args = [OK] * n
            args[i] = None
            if i not in optional:
                assert f(a, *args, OK, need, None) == -1
            if i in aligned:
                args[i] = P(4096 + aligned[i] // 2)
                assert f(a, *args, OK, need, None) == -4
        assert f(None, *[OK] * n, OK, need, None) == -1
        assert f(a, *[OK] * n, OK, need - 1, None) == -5
        assert f(a, *[OK] * n, None, need, None) == -5
        assert f(a, *[OK] * n, P(4096 + 128), need, None) == -5
    q = L.cat_i8_quantize
    assert q(None, 0, 4, 8, 8, OK, 8, OK, None) == -1 and q(OK, 0, 4, 8, 8, None, 8, OK, None) == -1 and q(OK, 0, 4, 8, 8, OK, 8, None, None) == -1
    assert q(OK, 0, 0, 8, 8, OK, 8, OK, None) == -2 and q(OK, 0, 4, 0, 8, OK, 8, OK, None) == -2
    assert q(OK, 0, 4, 8, 7, OK, 8, OK, None) == -2 and q(OK, 0, 4, 8, 8, OK, 7, OK, None) == -2 and q(OK, 0, 1 << 31, 8, 8, OK, 8, OK, None) == -2
    assert q(OK, 2, 4, 8, 8, OK, 8, OK, None) == -3 and q(P(4097), 0, 4, 8, 8, OK, 8, OK, None) == -4
    assert q(P(4098), 1, 4, 8, 8, OK, 8, OK, None) == -4 and q(OK, 0, 4, 8, 8, OK, 8, P(4098), None) == -4


def test_workspaces_stay_bounded():
    big = B.make_i8_shape(16384, 2048, 128256)
    assert B.cat_i8_workspace_bytes(big, 0) < 16384 * 2064 + (1 << 20)
    assert B.cat_i8_workspace_bytes(big, 3) < (3 << 30) + 2 * 128256 * 2048 + 16384 * 2064 + (300 << 20)      # never T x V
    small = B.make_i8_shape(16384, 2048, 128256, slab_mib=256)
    assert B.cat_i8_workspace_bytes(small, 3) < (256 << 20) + 2 * 128256 * 2048 + 16384 * 2064 + (300 << 20)


def test_struct_layout():
    assert ctypes.sizeof(B.cat_i8_shape) == 72


def test_cpu_tensors_are_refused():
    with pytest.raises(ValueError):
        api.quantize_rows(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        api.Int8Head(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        api.Int8Head.from_quantized(torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3))
    with pytest.raises(TypeError):
        api.quantize_rows(torch.zeros(3, 4, dtype=torch.float64))
    with pytest.raises(ValueError):
        api.quantize_rows(torch.zeros(3))
