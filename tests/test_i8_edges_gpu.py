"""The 8-bit head at the ends of its ranges, against the fp64 oracle; bounds in i8_util."""
import numpy as np
import pytest
import torch

from i8_util import check_ce, head, np64, tokens
from oracle import i8_oracle as O
from paper_2605_08632_b200.api import Int8Head
from test_i8_gpu import DEV, F32, check_logits

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
