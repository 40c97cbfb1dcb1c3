"""Gradients of few rows through the 8-bit head, many times over: every run has the bits of the first."""
import pytest
import torch

from i8_util import head
from paper_2605_08632_b200.api import Int8Head
from test_i8_gpu import BF, DEV

pytestmark = pytest.mark.gpu

# one and two passes, rows and head as M side, an odd and an even number of stages
SIZES = [(449, 2048, 25001), (601, 2048, 25001), (240, 2048, 25001), (300, 1024, 30001), (350, 1024, 30001), (100, 1024, 30001), (16, 1024, 30001)]


@pytest.mark.parametrize("T,d,V", SIZES)
def test_gradients_repeat(T, d, V):
    q, scale = (t.to(DEV) for t in head(V, d, seed=T))
    h = Int8Head.from_quantized(q, scale)
    X, y = torch.randn(T, d, device=DEV).to(BF), torch.randint(0, V, (T,), device=DEV)
    dY = torch.randn(T, (V + 7) // 8 * 8, device=DEV).to(BF)[:, :V]
    g = torch.randn(T, device=DEV)
    nll, lse = h.loss_forward(X, y)
    step = lambda: (h.loss_backward(X, y, None, g, nll, lse), h.logits_backward(dY))
    graph = torch.cuda.CUDAGraph()
    first = step()
    with torch.cuda.graph(graph):
        again = step()
    other = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(200):
        for a, b in zip(step(), first):
            other += (a != b).sum()
        graph.replay()
        for a, b in zip(again, first):
            other += (a != b).sum()
    assert int(other) == 0
