"""The 8-bit head at the ends of its ranges, against the fp64 oracle; bounds in i8_util."""
import numpy as np
import pytest
import torch

from i8_util import check_ce, head, np64, tokens
from oracle import i8_oracle as O
from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import Int8Head
from test_i8_gpu import BF, DEV, F32, check_logits, check_problem, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [12, 200])
def test_rows_whose_scale_rounds_to_zero(T):
    """Largest values of 1e-45 to 8e-44: their 127th is no binary32 number but 0, their integers are up to 127; logits are 0."""
    d, V = 48, 2000
    q, scale = head(V, d)
    X = tokens(T, d, F32)
    for i, size in enumerate((1e-45, 1e-44, 3e-44, 8e-44, 9.5e-44, 2e-43)):
        X[i] = torch.where(torch.arange(d) % 3 == 0, -size, size)
    xq, xs = O.quantize(np64(X))
    assert not xs[:4].any() and xs[4] > 0 and (np.abs(xq[:4]).max(axis=1) == 127).all()
    y = torch.arange(T) * 7 % V
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_logits(h(X.to(DEV)), X, q, scale, None, F32)
    nll, lse = h.loss_forward(X.to(DEV), y.to(DEV))
    z = O.product(xq, xs, q.numpy(), np64(scale))
    check_ce(np64(nll), np64(lse), z, O.cross_entropy(z, y.numpy()))


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("size", [1e7, 1e10, 1e28])
@pytest.mark.parametrize("sign", [-1.0, 1.0, 0.0])
def test_logits_of_any_size(T, size, sign):
    """All below -size, all above size, or on both sides: what rounding leaves of the largest logit's own exponent, many units above 1e9, is cut off."""
    d, V = 64, 3000
    g = torch.Generator().manual_seed(T)
    q = torch.randint(1, 128, (V, d), generator=g)
    if sign == 0.0:
        q = torch.where(torch.rand(V, d, generator=g) < 0.5, q, -q)
    q = q.to(torch.int8)
    scale = (0.02 / 40.0) * (1.0 + torch.rand(V, generator=g))
    X = ((sign or 1.0) * size * (1.0 + torch.rand(T, d, generator=g))).to(BF)
    y = torch.randint(0, V, (T,), generator=g)
    y[0] = -100
    nll, lse = Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).loss_forward(X.to(DEV), y.to(DEV))
    xq, xs = O.quantize(np64(X))
    z = O.product(xq, xs, q.numpy(), np64(scale))
    assert sign == 0.0 or (sign * z).min() > size           # 64 products of 1 .. 2 sizes with 5e-4 .. 0.13
    check_ce(np64(nll), np64(lse), z, O.cross_entropy(z, y.numpy()))


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("size", [1e32, 3e34])
def test_rows_whose_logits_are_all_far_below_zero(T, size):
    """No fixed number stands for "no logit yet"."""
    test_logits_of_any_size(T, size, -1.0)


@pytest.mark.parametrize("T", [60, 120, 300])
def test_gradients_of_huge_logits_stay_finite(T):
    """Logits of 1e8, where lse's own rounding is several units: the terms exp(z - lse) are cut off at half precision's largest value whatever the number of rows."""
    d, V = 64, 1000
    q, scale = (t.to(DEV) for t in head(V, d, spread=0.0))
    X = (tokens(T, d, F32) * 3e8).to(BF).to(DEV)
    y = (torch.arange(T) * 7 % V).to(DEV)
    h = Int8Head.from_quantized(q, scale)
    nll, lse = h.loss_forward(X, y)
    assert bool(nll.isfinite().all()) and float(nll.max()) > 1e7
    dX = h.loss_backward(X, y, None, torch.ones(T, device=DEV), nll, lse)
    assert bool(dX.isfinite().all())


# ------------------------------------------------------------------------------ the largest sizes of rows to integers
def quantize_large(rows, d, pitch, at):
    """Zeros but for one value in each of the places `at`."""
    X = torch.zeros(rows, d, dtype=BF, device=DEV)
    q = torch.full((rows, pitch), 9, dtype=torch.int8, device=DEV)
    s = torch.full((rows,), 7.0, device=DEV)
    for n, (r, i) in enumerate(at):
        X[r, i] = float(n + 1)
    B.cat_i8_quantize(X, B.CAT_BF16, rows, d, d, q, pitch, s)
    return q, s


def test_quantize_of_the_most_rows():
    rows = 2 ** 31 - 1
    at = [(0, 0), (5, 0), (2 ** 30 + 1, 0), (rows - 9, 0), (rows - 1, 0)]
    q, s = quantize_large(rows, 1, 8, at)
    for n, (r, _) in enumerate(at):
        assert int(q[r, 0]) == 127 and float(s[r]) == float(torch.tensor((n + 1) / 127.0))
        s[r] = 0.0
        q[r, 0] = 0
    assert int(torch.count_nonzero(s)) == 0
    for i in range(0, rows, 1 << 28):
        assert not bool(q[i:i + (1 << 28), 0].any()) and bool((q[i:i + (1 << 28), 1:] == 9).all())


def test_quantize_of_the_longest_row():
    d = 2 ** 31 - 1
    q, s = quantize_large(1, d, d, [(0, 0), (0, 255), (0, 2 ** 30), (0, d - 300), (0, d - 1)])
    assert float(s[0]) == float(torch.tensor(5 / 127.0))
    for i, n in ((0, 25), (255, 51), (2 ** 30, 76), (d - 300, 102), (d - 1, 127)):          # 25.4, 50.8, 76.2, 101.6
        assert int(q[0, i]) == n
    assert int(torch.count_nonzero(q)) == 5


# ------------------------------------------------------------------------------ heads that lie in wider rows
@pytest.mark.parametrize("T", [5, 200, 600])
@pytest.mark.parametrize("d,pitch", [(64, 96), (64, 64), (72, 208), (56, 64)])
def test_a_head_is_used_where_it_is(T, d, pitch):
    V = 1500
    q, scale, X, y, valid, g = problem(T, d, V)
    wide = torch.full((V, pitch), 99, dtype=torch.int8, device=DEV)
    wide[:, :d] = q.to(DEV)
    h = Int8Head.from_quantized(wide[:, :d], scale.to(DEV))
    assert h.q.data_ptr() == wide.data_ptr() and h.q.stride(0) == pitch
    check_problem(h, q, scale, X, y, valid, g)
    check_logits(h(X.to(DEV)), X, q, scale, None, BF)
    dY = torch.randn(T, V + 4, device=DEV).to(BF)[:, :V]
    same = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    assert torch.equal(h.logits_backward(dY), same.logits_backward(dY))
    assert torch.equal(h.to("cpu").to(DEV)(X.to(DEV)), same(X.to(DEV)))
    assert bool((wide[:, d:] == 99).all())


def test_other_layouts_are_copied():
    V, d = 300, 64
    q, scale = (t.to(DEV) for t in head(V, d))
    X = tokens(9, d, BF).to(DEV)
    want = Int8Head.from_quantized(q, scale)(X)
    for pitch, shift in ((72, 0), (80, 8), (64, 4)):
        flat = torch.zeros(V * pitch + 16, dtype=torch.int8, device=DEV)
        at = flat[shift:shift + V * pitch].view(V, pitch)[:, :d]
        at.copy_(q)
        h = Int8Head.from_quantized(at, scale)
        assert h.q.data_ptr() != at.data_ptr() and h.q.data_ptr() % 16 == 0 and torch.equal(h(X), want)


# ------------------------------------------------------------------------------ row slabs and the gradient that widens the head on its way
@pytest.mark.parametrize("T,d,V,mib", [(300, 1024, 9001, 1), (500, 2056, 25001, 20), (700, 2056, 50001, 48)])
def test_slabs_of_a_few_rows(T, d, V, mib):
    q, scale, X, y, valid, g = problem(T, d, V)
    need = B.cat_i8_workspace_bytes(B.make_i8_shape(T, d, V, slab_mib=mib), 3)
    assert need < B.cat_i8_workspace_bytes(B.make_i8_shape(T, d, V), 3) and need < 2 * d * V + (mib << 20)          # several slabs, no widened copy
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV), slab_mib=mib)
    nll, lse, dX = check_problem(h, q, scale, X, y, valid, g)
    for _ in range(3):
        assert torch.equal(h.loss_backward(X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV), nll, lse), dX)


# ------------------------------------------------------------------------------ one outlier among the scales
@pytest.mark.parametrize("T", [20, 200])
@pytest.mark.parametrize("power", [12, 14, 16])
def test_one_large_scale_beside_flat_rows(T, power):
    """Every term of a row whose probabilities are all about 1 / V is so small then that it is off by up to 2^-39 of the largest scale."""
    d, V = 128, 40000
    q, scale, X, y, valid, g = problem(T, d, V, spread=0.0, most=0.0)
    scale[123] *= 2.0 ** power
    X = (X.float() * 2.0 ** (-power - 4)).to(BF)
    check_problem(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)), q, scale, X, y, valid, g)
