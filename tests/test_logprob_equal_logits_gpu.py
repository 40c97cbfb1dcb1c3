"""Rows whose logits are all equal, at vocabularies of which a single thread block should not have to read the head row by row."""
import math

import pytest
import torch

from paper_2605_08632_b200.api import TokenLogProb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,d,V,k,dtype", [(1, 256, 128256, 20, BF), (70, 256, 128256, 5, BF), (300, 256, 128256, 64, BF), (40, 64, 40000, 20, F32),
                                           (3, 64, 300, 256, BF), (3, 64, 6, 9, F32)])
@pytest.mark.parametrize("zero", ["W", "H"])
def test_zero_operands(T, d, V, k, dtype, zero):
    """A head of zeros (as layers are initialised) or hidden states of zeros, minus zeros among them: ids 0, 1, ... and log V."""
    g = torch.Generator().manual_seed(1)
    H, W = torch.randn(T, d, generator=g), torch.randn(V, d, generator=g)
    z = H if zero == "H" else W
    z.zero_()
    z[:, ::3] = -0.0
    e = TokenLogProb(T, d, V, top_k=k, dtype=dtype)
    H, W = H.to(dtype).cuda(), W.to(dtype).cuda()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    r = e.forward(H, W)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 1000.0        # a few ms; row by row it would be many seconds
    n = min(k, V)
    assert torch.equal(r.top_ids[:, :n].cpu(), torch.arange(n).expand(T, n)) and bool((r.top_ids[:, n:] == -1).all())
    assert float((r.lse - math.log(V)).abs().max()) <= 4e-6 and float((r.entropy - math.log(V)).abs().max()) <= 4e-6
    assert float((r.top_logp[:, :n] + math.log(V)).abs().max()) <= 4e-6


@pytest.mark.parametrize("T", [2, 40, 200])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_head_that_is_almost_zero_is_not_zero(T, dtype):
    """Weights whose squares vanish in fp32: their logits differ all the same, and so does their order."""
    d, V, k = 64, 3000, 7
    g = torch.Generator().manual_seed(2)
    H, W = torch.randn(T, d, generator=g).to(dtype), (torch.randn(V, d, generator=g) * 2.0 ** -90).to(dtype)
    r = TokenLogProb(T, d, V, top_k=k, dtype=dtype).forward(H.cuda(), W.cuda())
    want = (H.double() @ W.double().T).topk(k, 1).indices
    assert torch.equal(r.top_ids.cpu(), want)
