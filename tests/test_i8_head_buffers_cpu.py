"""What Int8Head refuses before anything reaches the library: buffers that were replaced by others of other sizes, types or layouts."""
import pytest
import torch

from paper_2605_08632_b200 import api

V, d = 40, 60
LD = 64


@pytest.fixture
def made(monkeypatch):
    """A head in host memory (which the constructor refuses) and the calls that got as far as the library."""
    calls = []
    monkeypatch.setattr(api, "_rows", lambda name, t, dtypes, device=None: t.shape[1])
    monkeypatch.setattr(api, "_on", lambda device, call, *args: calls.append(call))
    monkeypatch.setattr(api.B, "cat_i8_workspace_bytes", lambda shape, which: 16)
    h = api.Int8Head.from_quantized(aligned(torch.zeros(V, LD, dtype=torch.int8))[:, :d], aligned(torch.ones(V)), aligned(torch.zeros(V)))
    return h, calls


def aligned(t, off=0):
    """t at `off` bytes past a 16-byte boundary."""
    flat = torch.zeros(t.numel() * t.element_size() + 32, dtype=torch.uint8)
    at = -flat.data_ptr() % 16 + off
    return flat[at:at + t.numel() * t.element_size()].view(t.dtype).view(t.shape).copy_(t)


X = torch.zeros(3, d, dtype=torch.bfloat16)
BAD = [(dict(q=torch.zeros(V - 1, LD, dtype=torch.int8)), ValueError), (dict(q=torch.zeros(V, d, dtype=torch.int8)), ValueError),
       (dict(q=torch.zeros(V, LD // 2, dtype=torch.int8)), ValueError), (dict(q=torch.zeros(V * LD, dtype=torch.int8)), ValueError),
       (dict(q=torch.zeros(LD, V, dtype=torch.int8).t()), ValueError), (dict(scale=torch.ones(V - 1)), ValueError), (dict(scale=torch.ones(())), ValueError),
       (dict(scale=torch.ones(V, 1)), ValueError), (dict(scale=torch.ones(1).expand(V)), ValueError), (dict(scale=torch.ones(2 * V)[::2]), ValueError),
       (dict(bias=torch.zeros(V + 1)), ValueError), (dict(bias=torch.zeros(2 * V)[1::2]), ValueError), (dict(q=torch.zeros(V, LD)), TypeError),
       (dict(scale=torch.ones(V).double()), TypeError), (dict(bias=torch.zeros(V).bfloat16()), TypeError),
       (dict(q=aligned(torch.zeros(V, LD, dtype=torch.int8), 8)), ValueError), (dict(scale=aligned(torch.ones(V), 4)), ValueError),
       (dict(bias=aligned(torch.zeros(V), 8)), ValueError)]


@pytest.mark.parametrize("bad,error", BAD)
def test_replaced_buffers_that_do_not_fit(made, bad, error):
    h, calls = made
    assert h.logits(X).shape == (3, V) and calls == [api.B.cat_i8_linear_fwd]
    for name, t in bad.items():
        setattr(h, name, t)
    with pytest.raises(error):
        h.logits(X)
    with pytest.raises(error):
        h.logits_backward(torch.zeros(3, V, dtype=torch.bfloat16))
    if "bias" not in bad:
        h.bias = None
        with pytest.raises(error):
            h.loss_forward(X, torch.zeros(3, dtype=torch.int64))
    assert len(calls) == 1


def test_replaced_buffers_that_fit(made):
    h, calls = made
    h.q, h.scale, h.bias = aligned(torch.ones(V, LD, dtype=torch.int8)), aligned(torch.zeros(V)), None
    h.logits(X)
    h.loss_forward(X, torch.zeros(3, dtype=torch.int64))
    assert calls == [api.B.cat_i8_linear_fwd, api.B.cat_i8_ce_fwd]
