"""Top-list distillation of rows whose own largest logits lie far above everything that the list and the label name: the rows that are most wrong."""
import pytest
import torch

import test_topk_kd_gpu as base
from paper_2605_08632_b200.api import CatLoss

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,dtype", [(96, BF), (640, BF), (96, F32)])
@pytest.mark.parametrize("renorm", [True, False])
def test_logits_past_the_range_above_the_named_ones(T, dtype, renorm):
    """One to three tokens from 60 to 250 nats above the named ones (16-bit steps from ref end at 80), the first and the last of the vocabulary
    among them, beside ordinary rows and masked ones."""
    K, d, V, k = 4, 64, 501, 3
    H, W, y, valid, ids, tl, start = base.make(T, K, d, V, k, dtype)
    g = torch.Generator().manual_seed(5)
    named = torch.cat([ids[(start[:, None] + torch.arange(K)).reshape(-1)], y[:, None]], 1)
    free = [[v for v in (0, V - 1, 8, 255, 256, 257, 300) if v not in named[r].tolist()] for r in range(T)]
    H = H.float()
    for r in range(T):
        if r % 4 == 0:
            continue
        up = 60.0 + 190.0 * float(torch.rand(1, generator=g))
        tokens = W[torch.tensor(free[r][: r % 4])].float()
        # hidden states that give each of those tokens `up` and a little more than the next
        H[r] = torch.linalg.lstsq(tokens, up + 0.5 * torch.arange(len(tokens)).float().unsqueeze(1)).solution.squeeze(1)
    H = H.to(dtype)
    x = (H, W, y, valid, ids, tl, start)
    conf = torch.full((T,), 0.9)
    eng = CatLoss(T, d, V, K, dtype=dtype)
    out = base.run(eng, *x, beta=0.2, renormalize=renorm, conf_ext=conf)
    ref = base.check(eng, out, x, K, beta=0.2, renormalize=renorm, conf_ext=conf)
    top = ref["z"].max(1)
    far = (top - ref["z"][torch.arange(T), y.numpy()]) > 90
    assert far.sum() > T // 3
