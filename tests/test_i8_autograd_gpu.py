"""Gradients through Int8Head as autograd asks for them, beside what test_i8_gpu holds."""
import copy

import pytest
import torch
import torch.autograd.forward_ad as forward_ad
import torch.utils.checkpoint

from i8_util import head, tokens
from paper_2605_08632_b200.api import Int8Head
from test_i8_gpu import BF, DEV, F32, problem

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ a head that is replaced
def replace(h, how, q, scale):
    """Other weights in the module's buffers, without writing to the tensors that were there."""
    if how == "scale":
        h.scale = scale
    elif how == "q":
        h.q = q
    else:
        h.load_state_dict({"q": q, "scale": scale}, assign=True)


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("how", ["scale", "q", "assign"])
def test_backward_is_of_the_head_that_the_forward_pass_saw(T, how):
    d, V = 64, 1001
    q, scale, X, y, valid, g = (t.to(DEV) for t in problem(T, d, V))
    q2, scale2 = (t.to(DEV) for t in head(V, d, seed=77))
    dY = torch.randn(T, 1008, device=DEV).to(BF)[:, :V]
    fixed = Int8Head.from_quantized(q, scale)
    nll, lse = fixed.loss_forward(X, y, valid)
    want_logits, want_loss = fixed.logits_backward(dY), fixed.loss_backward(X, y, valid, g, nll, lse)
    h = Int8Head.from_quantized(q.clone(), scale.clone())
    for call, up, want in ((lambda x: h(x), dY, want_logits), (lambda x: h.loss(x, y, valid), g, want_loss)):
        x = X.clone().requires_grad_()
        out = call(x)
        replace(h, how, q2.clone(), 3.0 * scale2)
        out.backward(up)
        assert torch.equal(x.grad, want)
        replace(h, "assign", q.clone(), scale.clone())


@pytest.mark.parametrize("call", [lambda h, x, y: h(x), lambda h, x, y: h.loss(x, y)])
def test_a_head_written_to_in_between_is_noticed(call):
    q, scale = (t.to(DEV) for t in head(300, 64))
    for write in (lambda h: h.scale.mul_(2.0), lambda h: h.q.zero_()):
        h = Int8Head.from_quantized(q.clone(), scale.clone())
        x = tokens(20, 64, BF).to(DEV).requires_grad_()
        out = call(h, x, torch.zeros(20, dtype=torch.int64, device=DEV))
        write(h)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()


# ------------------------------------------------------------------------------ forward mode
@pytest.mark.parametrize("needs_grad", [False, True])
@pytest.mark.parametrize("T", [20, 300])
def test_tangents_are_refused_not_dropped(T, needs_grad):
    q, scale = (t.to(DEV) for t in head(300, 64))
    h, X, y = Int8Head.from_quantized(q, scale), tokens(T, 64, BF).to(DEV), torch.zeros(T, dtype=torch.int64, device=DEV)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(X.clone().requires_grad_(needs_grad), torch.ones_like(X))
        for call in (lambda: h(dual), lambda: h.loss(dual, y)):
            with pytest.raises(NotImplementedError):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError):         # which does not switch tangents off
                call()
        assert h(X).shape == (T, 300) and bool(h.loss(X, y).isfinite().all())


# ------------------------------------------------------------------------------ refusals
def test_columns_without_a_gradient_are_refused_before_the_forward_pass():
    """Heads whose rows are no whole 16 bytes of bf16."""
    q, scale = (t.to(DEV) for t in head(100, 60))
    h, y = Int8Head.from_quantized(q, scale), torch.zeros(10, dtype=torch.int64, device=DEV)
    x = tokens(10, 60, BF).to(DEV).requires_grad_()
    for call in (lambda: h(x), lambda: h.loss(x, y)):
        with pytest.raises(ValueError, match="multiple of 8"):
            call()
        with torch.no_grad():
            assert call().shape[0] == 10


# ------------------------------------------------------------------------------ fp32 logits
def test_upstream_gradients_of_fp32_logits_are_rounded_once():
    """The contraction takes bf16: fp32 upstream gradients are rounded to it, halves to even, and nothing else is."""
    T, d, V = 70, 64, 1001
    q, scale = (t.to(DEV) for t in head(V, d))
    h, x = Int8Head.from_quantized(q, scale), tokens(T, d, BF).to(DEV).requires_grad_()
    up = torch.randn(T, V, device=DEV) * torch.rand(T, 1, device=DEV)
    h(x, F32).backward(up)
    laid = torch.zeros(T, 1008, dtype=BF, device=DEV)
    laid[:, :V] = up.to(BF)
    assert torch.equal(x.grad, h.logits_backward(laid[:, :V]))


# ------------------------------------------------------------------------------ what is kept for the backward pass
def test_kept_tensors_may_be_packed_away():
    """Hooks that lay the kept tensors out anew, a head in wider rows among them, and a forward pass that is run again."""
    T, d, V = 60, 64, 1001
    q, scale, X, y, valid, g = (t.to(DEV) for t in problem(T, d, V))
    wide = torch.zeros(V, 96, dtype=torch.int8, device=DEV)
    wide[:, :d] = q
    for h in (Int8Head.from_quantized(q, scale), Int8Head.from_quantized(wide[:, :d], scale)):
        for call, up in ((lambda x: h.loss(x, y, valid), g), (lambda x: h(x), torch.randn(T, V, device=DEV).to(BF))):
            plain, packed, again = (X.clone().requires_grad_() for _ in range(3))
            call(plain).backward(up)
            with torch.autograd.graph.save_on_cpu():
                out = call(packed)
            out.backward(up)
            torch.utils.checkpoint.checkpoint(call, again, use_reentrant=False).backward(up)
            assert torch.equal(packed.grad, plain.grad) and torch.equal(again.grad, plain.grad)


def test_copies_of_a_head():
    T, d, V = 20, 60, 300
    q, scale = (t.to(DEV) for t in head(V, d))
    wide = torch.full((V, 96), 55, dtype=torch.int8, device=DEV)
    wide[:, :d] = q
    X = tokens(T, d, BF).to(DEV)
    h = Int8Head.from_quantized(wide[:, :d], scale)
    want = h(X)
    for other in (copy.deepcopy(h), Int8Head.from_quantized(torch.zeros_like(q), torch.zeros_like(scale)), Int8Head.from_quantized(h.q[:, :d], h.scale)):
        other.load_state_dict(h.state_dict())
        assert torch.equal(other(X), want)
    assert bool((wide[:, d:] == 55).all())
