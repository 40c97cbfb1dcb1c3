"""A vocabulary of more 64-column tiles than a grid's second extent has room for (2^16 - 1)."""
import numpy as np
import pytest
import torch

from paper_2605_08632_b200.api import TokenLogProb

pytestmark = pytest.mark.gpu


def test_fp32_gradients_of_a_vocabulary_of_millions():
    T, d, V = 3, 4, 64 * 65535 + 130
    g = torch.Generator().manual_seed(0)
    H, W = torch.randn(T, d, generator=g), 0.5 * torch.randn(V, d, generator=g)
    y = torch.tensor([5, V - 1, V - 70])
    gl, ge = torch.randn(T, generator=g), torch.randn(T, generator=g)
    e = TokenLogProb(T, d, V, top_k=3, dtype=torch.float32)
    r = e.forward(H.cuda(), W.cuda(), y.cuda())
    dH, dW = e.backward(H.cuda(), W.cuda(), y.cuda(), None, gl.cuda(), ge.cuda())
    Hd, Wd = H.double().cuda(), W.double().cuda()
    z = Hd @ Wd.T
    lp = torch.log_softmax(z, 1)
    p = lp.exp()
    ent = -(p * lp).sum(1)
    dz = -gl.double().cuda()[:, None] * p - ge.double().cuda()[:, None] * p * (lp + ent[:, None])
    dz[torch.arange(T), y.cuda()] += gl.double().cuda()
    # sums of 4 million terms: in runs of 256, added up in up to 2^14 further steps of 2^-24, far from all of one sign
    for got, want in ((dH, dz @ Wd), (dW, dz.T @ Hd), (r.entropy, ent), (r.lse, z.logsumexp(1))):
        assert float((got.double() - want).norm()) <= 1e-4 * float(want.norm())
    assert torch.equal(r.top_ids, z.topk(3, 1).indices)
