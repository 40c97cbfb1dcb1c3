"""cat_i8_quantize, cat_i8_linear_fwd / _bwd and cat_i8_ce_fwd / _bwd against the fp64 oracle, through the public classes; bounds in i8_util."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from i8_util import E, U, check_ce, check_ce_grad, head, np64, sure, tokens
from oracle import i8_oracle as O
from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import CatLoss, Int8Head, quantize_rows

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------ rows to integers
def check_rows(X):
    q, s = quantize_rows(X.to(DEV))
    want_q, want_s = O.quantize(np64(X))
    assert q.shape == X.shape and q.dtype == torch.int8
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(np64(s), want_s, equal_nan=True)


@pytest.mark.parametrize("rows,d,dtype", [(1, 1, BF), (1, 1, F32), (3, 7, BF), (5, 16, F32), (129, 1003, F32), (300, 1024, BF), (7, 4099, BF), (33, 264, F32),
                                          (2, 70001, BF), (1000, 8, BF)])
def test_quantize_equals_the_definition(rows, d, dtype):
    g = torch.Generator().manual_seed(rows + d)
    check_rows((torch.randn(rows, d, generator=g) * (0.1 + torch.rand(rows, 1, generator=g))).to(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_on_halves_and_at_the_ends_of_the_range(dtype):
    """Values that lie on a half or next to one, rows of tiny, huge, equal and missing values."""
    g = torch.Generator().manual_seed(3)
    most = (1.0 + torch.rand(64, 1, generator=g)).to(dtype).float()
    halves = (torch.arange(255) - 127).float() / 254.0            # of the largest value: odd multiples lie on halves or round to beside them
    X = torch.cat([most, (most * halves), most * 0.5], 1).to(dtype)
    check_rows(X)
    check_rows(torch.nextafter(X.float(), torch.zeros(())).to(dtype))
    check_rows(torch.cat([torch.full((1, 1), 127.0), torch.arange(-126, 127).float().unsqueeze(0) + 0.5], 1).to(dtype))
    odd = torch.zeros(12, 40)
    odd[1, 5] = 1e-45
    odd[2] = torch.randn(40, generator=g) * 1e-41
    odd[3] = torch.randn(40, generator=g) * 3e-38
    odd[4] = torch.randn(40, generator=g) * 1e38
    odd[5] = 3.0
    odd[6, 39] = float("inf")
    odd[7, 0] = float("-inf")
    odd[8, 20] = float("nan")
    odd[9] = torch.randn(40, generator=g) * 2e-30
    odd[10] = torch.finfo(dtype).max
    odd[11] = -0.0
    check_rows(odd.to(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_of_rows_that_lie_apart(dtype):
    X = tokens(50, 300, dtype)
    check_rows(X[:, 1:264])                # rows at odd addresses
    check_rows(X[::3, :256])
    check_rows(X[:1, 3:4])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shift", range(8))
def test_quantize_at_every_address(dtype, shift):
    """Rows whose first value lies anywhere in 16 bytes, pitches that move it from row to row, lengths around whole eights; what lies around the matrix is NaN."""
    for rows, d, pitch in ((1, 1, 1), (3, 7, 9), (5, 8, 8), (4, 9, 11), (2, 23, 23), (9, 31, 40), (6, 33, 33), (40, 257, 257), (3, 2050, 2051), (2, 8191, 8191)):
        flat = torch.full((shift + rows * pitch + 16,), float("nan"))
        X = flat[shift:shift + rows * pitch].view(rows, pitch)[:, :d]
        X.copy_(torch.randn(rows, d, generator=torch.Generator().manual_seed(d + shift)))
        on = flat.to(dtype).to(DEV)
        view = on[shift:shift + rows * pitch].view(rows, pitch)[:, :d]
        q, s = quantize_rows(view)
        want_q, want_s = O.quantize(np64(X.to(dtype)))
        assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(np64(s), want_s)
        padded = torch.full((rows, (d + 7) // 8 * 8 + 8), 99, dtype=torch.int8, device=DEV)
        B.cat_i8_quantize(view, B.CAT_BF16 if dtype == BF else B.CAT_F32, rows, d, pitch, padded, padded.shape[1], s)
        assert bool((padded[:, d:] == 99).all()) and np.array_equal(padded[:, :d].cpu().numpy(), want_q)


def test_quantize_leaves_what_is_not_its_own():
    X = tokens(20, 37, BF).to(DEV)
    q = torch.full((20, 48), 99, dtype=torch.int8, device=DEV)
    s = torch.full((24,), 7.0, device=DEV)
    B.cat_i8_quantize(X, B.CAT_BF16, 20, 37, 37, q, 48, s)
    assert bool((q[:, 37:] == 99).all()) and bool((s[20:] == 7.0).all())
    assert np.array_equal(q[:, :37].cpu().numpy(), O.quantize(np64(X))[0])


# ------------------------------------------------------------------------------ product
def check_logits(Y, X, q, scale, bias, dtype):
    xq, xs = O.quantize(np64(X))
    z = O.product(xq, xs, q.numpy(), np64(scale))
    want = z if bias is None else z + np64(bias)
    tol = 3.01 * U * np.abs(z) + (U * (np.abs(want) + np.abs(z)) if bias is not None else 0.0)
    got = np64(Y)
    assert got.shape == want.shape and Y.dtype == dtype
    bound = tol + (E * (np.abs(want) + tol) if dtype == BF else 0.0) + 2.0 ** -149
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())


SIZES = [(1, 64, 1), (1, 2048, 3000), (2, 1, 7), (3, 17, 64), (5, 128, 257), (16, 1000, 1000), (17, 513, 4097), (67, 1024, 9473), (32, 96, 19001),
         (100, 260, 5000), (128, 128, 40007), (129, 200, 700), (255, 65, 513), (300, 1024, 2056), (511, 640, 1031), (1025, 48, 300), (4, 65536, 33)]


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("x,y,bias", [(BF, BF, False), (BF, F32, True), (F32, BF, True)])
def test_logits_match_oracle(T, d, V, x, y, bias):
    q, scale = head(V, d, seed=T + V)
    X = tokens(T, d, x, seed=d)
    b = torch.randn(V, generator=torch.Generator().manual_seed(9)) if bias else None
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV), None if b is None else b.to(DEV))
    check_logits(h.logits(X.to(DEV), y), X, q, scale, b, y)


@pytest.mark.parametrize("T,V", [(200, 3), (300, 31), (129, 33), (140, 8), (600, 1)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_narrow_outputs_of_many_rows(T, V, dtype):
    d = 72
    q, scale = head(V, d)
    X = tokens(T, d, BF)
    b = torch.randn(V, generator=torch.Generator().manual_seed(9))
    check_logits(Int8Head.from_quantized(q.to(DEV), scale.to(DEV), b.to(DEV)).logits(X.to(DEV), dtype), X, q, scale, b, dtype)


def test_extreme_integers_add_up_exactly():
    """Every token and weight at the ends of their range, so that the sums are the largest there are."""
    d = 65536
    q = torch.full((40, d), -128, dtype=torch.int8)
    q[1::2] = 127
    X = torch.ones(18, d)
    X[1::2] = -1.0
    scale = torch.full((40,), 2.0 ** -20)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_logits(h(X.to(DEV)), X, q, scale, None, F32)


@pytest.mark.parametrize("T", [1, 40, 200])
def test_head_from_weights_and_rows_that_lie_apart(T):
    d, V = 200, 3001
    W = (0.02 * torch.randn(V, d + 24, generator=torch.Generator().manual_seed(1))).to(BF)[:, :d]
    X = tokens(T, d + 9, BF)[:, 9:]
    h = Int8Head(W.to(DEV))
    q, s = O.quantize(np64(W))
    assert np.array_equal(h.q[:, :d].cpu().numpy(), q) and np.array_equal(np64(h.scale), s)
    check_logits(h(X.to(DEV)), X, torch.from_numpy(q.astype(np.int8)), h.scale.cpu(), None, BF)
    y = h(X.to(DEV), F32)
    assert y.shape == (T, V) and y.stride(0) % 8 == 0


@pytest.mark.parametrize("T", [3, 150])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_logits_leave_what_lies_past_the_vocabulary(T, dtype):
    d, V, ld = 64, 1003, 1024
    q, scale = head(V, d)
    X = tokens(T, d, BF).to(DEV)
    code = B.CAT_BF16 if dtype == BF else B.CAT_F32
    shape = B.make_i8_shape(T, d, V, ldY=ld, y_dtype=code)
    Y = torch.full((T + 2, ld), 77.0, dtype=dtype, device=DEV)
    n = B.cat_i8_workspace_bytes(shape, 0)
    ws = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    B.cat_i8_linear_fwd(shape, X, q.to(DEV), scale.to(DEV), None, Y, ws[:n])
    assert bool((Y[T:] == 77.0).all()) and bool((Y[:, V:] == 77.0).all()) and bool((ws[n:] == 0x5A).all())
    assert int(ws[:4].view(torch.int32).item()) == 0
    check_logits(Y[:T, :V], X, q, scale, None, dtype)


def test_logits_past_31_bits():
    T, d, V = 17001, 16, 128256
    q, scale = head(V, d)
    X = tokens(T, d, BF)
    Y = Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).logits(X.to(DEV))
    rows = [0, 1, 255, 8371, 8372, 16742, 16743, 16744, 17000]
    check_logits(Y[rows], X[rows], q, scale, None, BF)


def test_nothing_finite_in_a_row_or_channel():
    for T in (5, 200):
        d, V = 48, 300
        q, scale = head(V, d)
        scale[7], scale[9] = float("nan"), 0.0
        X = tokens(T, d, BF)
        X[1, 3], X[2, 5], X[3] = float("inf"), float("nan"), 0.0
        Y = np64(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).logits(X.to(DEV), F32))
        bad = np.zeros((T, V), bool)
        bad[[1, 2]], bad[:, 7] = True, True
        assert np.array_equal(np.isnan(Y), bad)
        assert not Y[3][~bad[3]].any() and not Y[:, 9][~bad[:, 9]].any()


@pytest.mark.parametrize("T,d,V", [(1, 8, 1), (1, 2048, 5000), (3, 64, 100), (40, 200, 3001), (130, 264, 20000), (300, 1024, 2056), (700, 72, 513), (257, 512, 777), (400, 72, 513),
                                   (480, 256, 70000), (336, 128, 70001), (129, 520, 1003)])
def test_logits_gradient_matches_oracle(T, d, V):
    q, scale = head(V, d, seed=V)
    g = torch.Generator().manual_seed(T)
    ld = (V + 7) // 8 * 8 + 8
    dY = torch.full((T, ld), float("nan")).to(BF)
    dY[:, :V] = torch.randn(T, V, generator=g).to(BF)
    dX = np64(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).logits_backward(dY.to(DEV)[:, :V]))
    dY = np64(dY[:, :V])
    want = O.product_grad(dY, q.numpy(), np64(scale))
    mag = np.abs(dY * np64(scale)) @ np.abs(q.numpy().astype(np.float64))
    off = (E + 2 * U * (V / 16 + 24)) * mag
    assert np.all(np.abs(dX - want) <= off + E * (np.abs(want) + off) + 2.0 ** -126)
    assert np.linalg.norm(dX - want) <= 2 * E * np.linalg.norm(want) + 2.0 ** -100


# More rows than one pass over the head takes, heads so large that no widened copy is made: two passes that share the parts' workspace.
@pytest.mark.parametrize("T,d,V", [(449, 2048, 25001), (513, 2056, 25003), (895, 4104, 25000)])
def test_logits_gradient_in_two_passes(T, d, V):
    test_logits_gradient_matches_oracle(T, d, V)


# ------------------------------------------------------------------------------ cross entropy
def problem(T, d, V, masked=0.2, spread=1.0, most=40.0):
    q, scale = head(V, d, seed=T + V, spread=spread)
    g = torch.Generator().manual_seed(T)
    y = torch.randint(0, V, (T,), generator=g)
    X = sure(tokens(T, d, BF, seed=d), q, scale, y, most)
    valid = (torch.rand(T, generator=g) >= masked).to(torch.uint8)
    y = torch.where(torch.rand(T, generator=g) < 0.05, torch.where(torch.rand(T, generator=g) < 0.5, V, -100), y)
    return q, scale, X, y, valid, torch.randn(T, generator=g)


def check_problem(h, q, scale, X, y, valid, g):
    nll, lse = h.loss_forward(X.to(DEV), y.to(DEV), None if valid is None else valid.to(DEV))
    dX = h.loss_backward(X.to(DEV), y.to(DEV), None if valid is None else valid.to(DEV), g.to(DEV), nll, lse)
    off = valid is not None and not bool(valid.all())
    Xs = np64(X)
    if off:
        Xs = Xs * valid.numpy()[:, None].astype(float) if np.isfinite(Xs).all() else np.where(valid.numpy()[:, None] != 0, Xs, 0.0)
    xq, xs = O.quantize(Xs)
    z = O.product(xq, xs, q.numpy(), np64(scale))
    v = None if valid is None else valid.numpy()
    ref = O.cross_entropy(z, y.numpy(), v)
    check_ce(np64(nll), np64(lse), z, ref)
    want, terms = O.cross_entropy_grad(z, y.numpy(), v, np64(g), q.numpy(), np64(scale))
    check_ce_grad(np64(dX), z, ref, terms, want, np64(g), q.numpy(), np64(scale))
    return nll, lse, dX


CE_SIZES = [(1, 8, 1), (1, 64, 2), (1, 2048, 5003), (2, 8, 33), (3, 72, 256), (5, 128, 257), (37, 256, 8191), (130, 136, 20011), (257, 256, 12000),
            (600, 128, 3000), (64, 1024, 9473), (300, 1024, 2056), (1025, 48, 300), (128, 2048, 19000), (17, 64, 30000), (400, 72, 513), (450, 1032, 9000), (33, 1288, 700)]


@pytest.mark.parametrize("T,d,V", CE_SIZES)
def test_loss_and_gradient_match_oracle(T, d, V):
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_problem(h, q, scale, X, y, valid, g)
    check_problem(h, q, scale, X, y, None, g)


@pytest.mark.parametrize("T", [20, 300])
def test_rows_that_are_very_sure_or_very_wrong(T):
    """Label probabilities from 1 - 1e-30 down to 1e-60, losses and gradients of each to their own size."""
    d, V = 256, 2000
    q, scale = head(V, d, spread=0.3)
    g = torch.Generator().manual_seed(5)
    y = torch.randint(0, V, (T,), generator=g)
    W = q.float() * scale.unsqueeze(1)
    Wy = W[y]
    amount = torch.linspace(-140.0, 80.0, T)
    X = (tokens(T, d, F32) + Wy * (amount / (Wy * Wy).sum(1)).unsqueeze(1)).to(BF)
    nll, _, dX = check_problem(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)), q, scale, X, y, None, torch.ones(T))
    assert float(nll.max()) > 60 and 0 < float(nll.min()) < 1e-15
    assert bool((dX != 0).any(1).all())


@pytest.mark.parametrize("spread", [0.0, 3.0, 5.0])
def test_scales_far_apart(spread):
    T, d, V = 150, 128, 3000
    q, scale, X, y, valid, g = problem(T, d, V, spread=spread, most=10.0)
    X = (X.float() * 10.0 ** (-spread / 2)).to(BF)
    check_problem(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)), q, scale, X, y, valid, g)


def test_rows_and_channels_of_zeros():
    T, d, V = 140, 64, 1000
    q, scale, X, y, valid, g = problem(T, d, V)
    X[::3] = 0.0
    scale[::7] = 0.0
    q[::11] = 0
    check_problem(Int8Head.from_quantized(q.to(DEV), scale.to(DEV)), q, scale, X, y, valid, g)
    zero = Int8Head.from_quantized(q.to(DEV), torch.zeros(V, device=DEV))
    nll, lse = zero.loss_forward(X.to(DEV), y.to(DEV))
    ok = ((y >= 0) & (y < V)).to(DEV)
    assert torch.allclose(lse, torch.full_like(lse, float(np.log(V)))) and torch.allclose(nll[ok], lse[ok])
    assert not bool(zero.loss_backward(X.to(DEV), y.to(DEV), None, g.to(DEV), nll, lse).any())


@pytest.mark.parametrize("T", [30, 300])
def test_masked_rows_may_hold_anything_and_others_may_not(T):
    d, V = 64, 3000
    q, scale, X, y, valid, g = problem(T, d, V, masked=0.5)
    off = (valid == 0).nonzero().flatten()
    X[off[0::4]], X[off[1::4], 3], X[off[2::4]] = float("nan"), float("inf"), 0.0
    g[off[0]], y[off[1]] = float("nan"), 1 << 40
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_problem(h, q, scale, X, y, valid, g)
    check_problem(h, q, scale, X, y, torch.zeros_like(valid), g)
    on = (valid != 0).nonzero().flatten()
    X[on[0], 5], y[on[0]] = float("nan"), 4
    nll, lse = h.loss_forward(X.to(DEV), y.to(DEV), valid.to(DEV))
    dX = h.loss_backward(X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV), nll, lse)
    assert bool(nll[on[0]].isnan()) and bool(lse[on[0]].isnan()) and bool(dX[on[0]].isnan().all())
    rest = torch.ones(T, dtype=torch.bool)
    rest[on[0]] = False
    assert bool(nll[rest].isfinite().all()) and bool(dX[rest].isfinite().all())


@pytest.mark.parametrize("T,d,V,mib", [(700, 64, 3000, 1), (1500, 128, 9000, 4), (513, 2048, 20000, 6)])
def test_slabs_change_nothing(T, d, V, mib):
    q, scale, X, y, valid, g = problem(T, d, V)
    a = Int8Head.from_quantized(q.to(DEV), scale.to(DEV), slab_mib=mib)
    assert B.cat_i8_workspace_bytes(B.make_i8_shape(T, d, V, slab_mib=mib), 3) < B.cat_i8_workspace_bytes(B.make_i8_shape(T, d, V), 3)
    check_problem(a, q, scale, X, y, valid, g)


@pytest.mark.parametrize("T", [449, 601])
def test_loss_gradient_in_two_passes(T):
    d, V = 2048, 25001
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_problem(h, q, scale, X, y, valid, g)
    args = [t.to(DEV) for t in (X, y, valid, g)]
    nll, lse = h.loss_forward(*args[:3])
    dX = h.loss_backward(*args, nll, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = h.loss_backward(*args, nll, lse)
    again.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, dX)


def test_loss_takes_fp32_tokens():
    T, d, V = 70, 100, 2000
    q, scale, _, y, valid, _ = problem(T, d, V)
    X = tokens(T, d, F32)
    nll, lse = Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).loss_forward(X.to(DEV), y.to(DEV), valid.bool().to(DEV))
    xq, xs = O.quantize(np64(X))
    z = O.product(xq, xs, q.numpy(), np64(scale))
    check_ce(np64(nll), np64(lse), z, O.cross_entropy(z, y.numpy(), valid.numpy()))


def test_gradient_follows_differences_of_the_loss():
    """Along a direction of X: the loss over the head as it is in 64 bits (no rounding of the tokens) against the kernels' gradient."""
    T, d, V = 40, 128, 500
    q, scale, X, y, valid, g = problem(T, d, V, most=6.0)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    nll, lse = h.loss_forward(X.to(DEV), y.to(DEV), valid.to(DEV))
    dX = np64(h.loss_backward(X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV), nll, lse))
    xq, xs = O.quantize(np64(X))
    W, X0 = q.numpy().astype(np.float64) * np64(scale)[:, None], xq * xs[:, None]
    along = np.random.default_rng(0).normal(size=X0.shape)

    def f(t):
        return float(np64(g) @ O.cross_entropy((X0 + t * along) @ W.T, y.numpy(), valid.numpy())["nll"])

    step = 1e-5
    slope = (f(step) - f(-step)) / (2 * step)
    # the gradient's entries are off by a rounding to bf16 and by h of their terms, and add up along the direction
    assert abs((dX * along).sum() - slope) <= 2 * E * np.linalg.norm(dX) * np.sqrt(np.log(dX.size)) + 1e-6 * abs(slope)


# ------------------------------------------------------------------------------ as they are used together
def test_a_run_from_weights_to_a_weighted_loss():
    """A target's head quantised, its confidences as the weights of the draft's CAT loss, the draft trained through the same frozen head."""
    T, K, d, V = 256, 8, 128, 3000
    W = (0.05 * torch.randn(V, d, generator=torch.Generator().manual_seed(0))).to(BF)
    q, scale, X, y, valid, _ = problem(T, d, V)
    y, X = y.clamp(0, V - 1), X.to(DEV)
    head8 = Int8Head(W.to(DEV))
    nll, _ = head8.loss_forward(X, y.to(DEV), valid.to(DEV))
    cat = CatLoss(T, d, V, K)
    loss, _, _ = cat.forward_backward(X, W.to(DEV), y.to(DEV), valid.to(DEV), conf_ext=torch.exp(-nll))
    weight = cat.weight.clone()
    h = X.clone().requires_grad_()
    (weight * head8.loss(h, y.to(DEV), valid.to(DEV))).sum().div(valid.sum().item()).backward()
    qn, sn = O.quantize(np64(W))
    xq, xs = O.quantize(np64(X))
    z = O.product(xq, xs, qn, sn)
    ref = O.cross_entropy(z, y.numpy(), valid.numpy())
    g = np64(weight) / valid.sum().item()
    want, terms = O.cross_entropy_grad(z, y.numpy(), valid.numpy(), g, qn, sn)
    check_ce_grad(np64(h.grad), z, ref, terms, want, g, qn, sn)
    conf = np.where(ref["ok"], np.exp(-ref["nll"]), 1.0).reshape(-1, K)
    before = np.concatenate([np.ones((T // K, 1)), np.cumprod(conf, axis=1)[:, :-1]], axis=1).reshape(-1)
    assert np.allclose(np64(weight), np.where(ref["ok"], before, 0.0), rtol=1e-4, atol=1e-30)
    top = head8.logits(X, F32).argmax(1)                         # the draft answers
    sure_of = np.sort(z, axis=1)[:, -1] - np.sort(z, axis=1)[:, -2] > 1e-4
    assert np.array_equal(top.cpu().numpy()[sure_of], z.argmax(axis=1)[sure_of])


def test_module_gradients():
    T, d, V = 90, 64, 1001
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    assert not list(h.parameters()) and set(h.state_dict()) == {"q", "scale"}
    wide = torch.zeros(T, d + 8, dtype=BF, device=DEV)
    wide[:, :d] = X.to(DEV)
    wide.requires_grad_()
    (h.loss(wide[:, :d], y.to(DEV), valid.bool().to(DEV)) * g.to(DEV)).sum().backward()
    nll, lse = h.loss_forward(X.to(DEV), y.to(DEV), valid.to(DEV))
    want = h.loss_backward(X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV), nll, lse)
    assert torch.equal(wide.grad[:, :d], want) and not bool(wide.grad[:, d:].any())
    for out in (BF, F32):                                        # gradients of any layout and type are laid out as the call wants them
        x = X.to(DEV).requires_grad_()
        h(x, out).float().sum().backward()
        ones = torch.ones(T, (V + 7) // 8 * 8, dtype=BF, device=DEV)[:, :V]
        assert torch.equal(x.grad, h.logits_backward(ones))
    x = X.to(DEV).requires_grad_()
    first, second = h.loss(x, y.to(DEV)), h.loss(x, y.to(DEV))
    first.detach().zero_()
    (first * 0.0 + second).sum().backward()                      # two graphs of one leaf; the first's losses written to
    assert bool(x.grad.isfinite().all())


def test_refusals():
    T, d, V = 10, 64, 100
    q, scale = head(V, d)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    X, y = tokens(T, d, BF).to(DEV), torch.zeros(T, dtype=torch.int64, device=DEV)
    nll, lse = h.loss_forward(X, y)
    for bad, error in ((lambda: h(X.half()), TypeError), (lambda: h(X[:, :32]), ValueError), (lambda: h(X.cpu()), ValueError), (lambda: h(X.t()), ValueError),
                       (lambda: h(X[0]), ValueError), (lambda: h(X[:1].expand(T, d)), ValueError), (lambda: h(X, torch.float16), TypeError),
                       (lambda: h.loss(X, y.int()), TypeError), (lambda: h.loss(X, y[:5]), ValueError), (lambda: h.loss(X, y, nll), TypeError),
                       (lambda: h.loss(X.float().requires_grad_(), y), TypeError), (lambda: h(X.float().requires_grad_()), TypeError),
                       (lambda: h.loss_backward(X.float(), y, None, nll, nll, lse), TypeError),
                       (lambda: h.loss_backward(X, y, None, nll.double(), nll, lse), TypeError),
                       (lambda: h.loss_backward(X, y, None, nll[:3], nll, lse), ValueError),
                       (lambda: h.logits_backward(torch.zeros(T, V, device=DEV)), TypeError), (lambda: h.logits_backward(torch.zeros(T, V - 1, dtype=BF, device=DEV)), ValueError),
                       (lambda: h.logits_backward(torch.zeros(T, V, dtype=BF, device=DEV)), ValueError),       # 100 entries: no whole 16 bytes
                       (lambda: Int8Head.from_quantized(q.to(DEV), scale), ValueError), (lambda: Int8Head.from_quantized(q.to(DEV).int(), scale.to(DEV)), TypeError),
                       (lambda: Int8Head.from_quantized(q.to(DEV), scale.to(DEV).bfloat16()), TypeError),
                       (lambda: Int8Head.from_quantized(q.to(DEV), scale.to(DEV), scale[:3].to(DEV)), ValueError),
                       (lambda: quantize_rows(X.unsqueeze(0)), ValueError), (lambda: quantize_rows(X[:, :0]), ValueError),
                       (lambda: Int8Head.from_quantized(q.to(DEV), scale.to(DEV)).bfloat16()(X), TypeError)):
        with pytest.raises(error):
            bad()
    odd = Int8Head.from_quantized(*(t.to(DEV) for t in head(V, 60)))
    x = X[:, :60].clone().requires_grad_()
    with pytest.raises(ValueError):                              # 60 columns: no gradient
        odd.loss(x, y).sum().backward()


def test_loss_refuses_a_head_with_a_bias():
    q, scale = head(100, 64)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV), torch.zeros(100, device=DEV))
    X, y = tokens(5, 64, BF).to(DEV), torch.zeros(5, dtype=torch.int64, device=DEV)
    n = torch.zeros(5, device=DEV)
    for call in (lambda: h.loss(X, y), lambda: h.loss(X.clone().requires_grad_(), y), lambda: h.loss_backward(X, y, None, n, n, n)):
        with pytest.raises(ValueError, match="bias"):
            call()
    assert h(X).shape == (5, 100)


def test_no_rows():
    q, scale = head(100, 64)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    X, y = torch.zeros(0, 64, dtype=BF, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV)
    assert h(X).shape == (0, 100) and h.loss(X, y).shape == (0,) and quantize_rows(X)[0].shape == (0, 64)
    assert h.logits_backward(torch.zeros(0, 104, dtype=BF, device=DEV)[:, :100]).shape == (0, 64)
    x = X.requires_grad_()
    h.loss(x, y).sum().backward()
    assert x.grad.shape == (0, 64)


@pytest.mark.parametrize("T", [1, 60, 300])
def test_runs_are_alike_bit_for_bit(T):
    d, V = 256, 20000
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    runs = []
    for _ in range(3):
        nll, lse = h.loss_forward(X.to(DEV), y.to(DEV), valid.to(DEV))
        runs.append([h(X.to(DEV)), nll, lse, h.loss_backward(X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV), nll, lse),
                     h.logits_backward(X.to(DEV)[:, :1].expand(T, V).contiguous())])
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


@pytest.mark.parametrize("T", [1, 60, 300])
def test_captured_calls_follow_new_inputs(T):
    d, V = 128, 6000
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    X, y, valid, g = X.to(DEV), y.to(DEV), valid.to(DEV), g.to(DEV)
    dY = torch.randn(T, V, device=DEV).to(BF)

    def step():
        nll, lse = h.loss_forward(X, y, valid)
        return [h.logits(X), nll, lse, h.loss_backward(X, y, valid, g, nll, lse), h.logits_backward(dY), *quantize_rows(X)]

    step()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for seed in (7, 8):
        _, _, X2, _, _, _ = problem(T, d, V, most=3.0)
        X.copy_(X2.roll(seed, 0) * (seed - 5))
        dY.copy_(dY.roll(1, 1))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("T", [1, 70, 300, 900])
def test_inputs_written_just_before_a_call(T):
    """Weights, tokens and upstream gradients that the kernel right before a call writes: the call's kernels may not start on what was there."""
    d, V, n = 512, 20000, 6
    g = torch.Generator().manual_seed(1)
    Ws = [(0.02 * torch.randn(V, d, generator=g)).to(BF).to(DEV) for _ in range(2)]
    Xs = [torch.randn(T, d, generator=g).to(BF).to(DEV) for _ in range(2)]
    dYs = [torch.randn(T, V, generator=g).to(BF).to(DEV) for _ in range(2)]
    y = torch.randint(0, V, (T,), generator=g).to(DEV)
    fresh = [Int8Head(W) for W in Ws]
    want = []
    for i in range(2):
        nll, lse = fresh[i].loss_forward(Xs[i], y)
        want.append((fresh[i].logits(Xs[i]), nll, lse, fresh[i].loss_backward(Xs[i], y, None, nll, nll, lse), fresh[i].logits_backward(dYs[i])))
    torch.cuda.synchronize()
    h = Int8Head(Ws[0])
    X, dY = Xs[0].clone(), dYs[0].clone()

    def requantise(i):
        B.cat_i8_quantize(Ws[i], B.CAT_BF16, V, d, d, h.q, d, h.scale)

    for k in range(n):
        i = k % 2
        requantise(1 - i)
        requantise(i)
        a = h.logits(Xs[i])
        requantise(1 - i)
        requantise(i)
        b = h.logits_backward(dYs[i])
        X.copy_(Xs[i])
        nll, lse = h.loss_forward(X, y)
        X.zero_()
        X.copy_(Xs[i])
        requantise(1 - i)
        requantise(i)
        c = h.loss_backward(X, y, None, nll, nll, lse)
        dY.zero_()
        dY.copy_(dYs[i])
        e = h.logits_backward(dY)
        for got, ref in zip((a, nll, lse, c, b, e), (*want[i][:4], want[i][4], want[i][4])):
            assert torch.equal(got, ref)


def test_capture_with_gradients_is_refused():
    q, scale = head(300, 64)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    X, y = tokens(20, 64, BF).to(DEV).requires_grad_(), torch.zeros(20, dtype=torch.int64, device=DEV)
    h.loss(X, y).sum().backward()
    for call in (lambda: h.loss(X, y), lambda: h(X)):
        with pytest.raises(RuntimeError, match="cannot be captured"):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                call()
    torch.cuda.synchronize()
    assert bool(h.loss(X, y).isfinite().all())


def test_two_streams_at_once():
    d, V = 128, 12000
    cases = [problem(T, d, V) for T in (40, 300)]
    heads = [Int8Head.from_quantized(c[0].to(DEV), c[1].to(DEV)) for c in cases]
    on = [[t.to(DEV) for t in c[2:]] for c in cases]

    def one(h, X, y, valid, g):
        nll, lse = h.loss_forward(X, y, valid)
        return [nll, lse, h.loss_backward(X, y, valid, g, nll, lse), h(X)]

    want = [one(h, *c) for h, c in zip(heads, on)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(one(heads[i], *on[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))


def test_without_cta_pairs():
    """The one-CTA form of the products (read once per process): a short run of its own."""
    code = """
import torch
from oracle import i8_oracle as O
import numpy as np
import sys
sys.path.insert(0, "tests")
from test_i8_gpu import check_logits, check_problem, problem, DEV, BF
from paper_2605_08632_b200.api import Int8Head
for T, d, V in ((300, 264, 3001), (700, 128, 5000)):
    q, scale, X, y, valid, g = problem(T, d, V)
    h = Int8Head.from_quantized(q.to(DEV), scale.to(DEV))
    check_problem(h, q, scale, X, y, valid, g)
    check_logits(h.logits(X.to(DEV)), X, q, scale, None, BF)
    dY = torch.ones(T, (V + 7) // 8 * 8, dtype=BF, device=DEV)[:, :V]
    want = np.tile((q.double() * scale.double()[:, None]).sum(0).numpy(), (T, 1))
    got = h.logits_backward(dY).double().cpu().numpy()
    assert np.linalg.norm(got - want) <= 2.0 ** -7 * np.linalg.norm(want)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, CAT_LOSS_CTA_PAIR="0", PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-2000:]
