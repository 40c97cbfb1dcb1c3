"""What the engines of the LM-head operators keep between calls: workspaces that captured graphs hold, counters, autograd's buffers."""
import numpy as np
import pytest
import torch

from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import CatLoss

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def lists(L, k, V, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(L)])
    return ids.to(DEV), torch.log_softmax(torch.randn(L, k, generator=g), 1).to(DEV)


def rows(T, d, V, seed, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    H, W = torch.randn(T, d, generator=g).to(dtype), (0.05 * torch.randn(V, d, generator=g)).to(dtype)
    return H.to(DEV), W.to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step_outlives_calls_with_longer_lists(dtype):
    """Capture with short lists, call with long ones and with others, replay: the replay's workspace is still the engine's."""
    T, K, d, V = 96, 8, 64, 700
    eng = CatLoss(T, d, V, K, dtype=dtype)
    H, W, y = rows(T, d, V, 0, dtype)
    short, long = lists(T, 3, V, 1), lists(T, B.CAT_TOPK_MAX, V, 2)
    eng.topk_kd_forward_backward(H, W, y, None, *short)
    address = eng._ws_topk.data_ptr()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = eng.topk_kd_forward_backward(H, W, y, None, *short)
    eng.topk_kd_forward_backward(H, W, y, None, *long)
    eng.topk_kd_forward_backward(H, W, y, None, *lists(T, 200, V, 3))
    others = [torch.full((1 << 22,), 0x5A, dtype=torch.uint8, device=DEV) for _ in range(8)]     # would take freed memory
    assert eng._ws_topk.data_ptr() == address
    H2, W2, _ = rows(T, d, V, 7, dtype)
    H.copy_(H2), W.copy_(W2)
    graph.replay()
    torch.cuda.synchronize()
    want = CatLoss(T, d, V, K, dtype=dtype).topk_kd_forward_backward(H, W, y, None, *short)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(bool((o == 0x5A).all()) for o in others)


def test_a_captured_distillation_outlives_calls_with_more_positions():
    """kd_forward_backward's workspace grows with the target positions a slab refers to; a captured call keeps the one it was given."""
    T, K, d, V, L = 512, 8, 64, 700, 2000
    eng = CatLoss(T, d, V, K)
    H, W, y = rows(T, d, V, 0)
    Ht, Wt, _ = rows(L, d, V, 1)
    near, far = torch.arange(T // K), torch.arange(T // K) * 30
    eng.kd_forward_backward(H, W, y, None, Ht, Wt, near, 0.2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = eng.kd_forward_backward(H, W, y, None, Ht, Wt, near, 0.2)
    held = eng._ws_kd
    address, n = held.data_ptr(), held.numel()
    del held
    eng.kd_forward_backward(H, W, y, None, Ht, Wt, far, 0.2)
    assert eng._ws_kd.numel() > n
    others = [torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV) for _ in range(4)]         # would take freed memory
    assert all(o.data_ptr() != address for o in others)
    H2, W2, _ = rows(T, d, V, 7)
    H.copy_(H2), W.copy_(W2)
    graph.replay()
    torch.cuda.synchronize()
    want = CatLoss(T, d, V, K).kd_forward_backward(H, W, y, None, Ht, Wt, near, 0.2)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(bool((o == 0x5A).all()) for o in others)


def bad_labels(T, V, seed):
    """Labels of which some are no token id, some of those in masked rows; and how many rows have one and are not masked."""
    g = torch.Generator().manual_seed(seed)
    y = torch.randint(0, V, (T,), generator=g)
    where = torch.rand(T, generator=g)
    for i, value in enumerate((-100, -1, V, V + 1, 2 ** 40, -(2 ** 62))):
        y[(where >= 0.05 * i) & (where < 0.05 * (i + 1))] = value
    valid = torch.rand(T, generator=g) < 0.7
    bad = (y < 0) | (y >= V)
    assert bool((bad & valid).any()) and bool((bad & ~valid).any())
    return y.to(DEV), valid.to(DEV), bad, valid


@pytest.mark.parametrize("dtype,slab_mib", [(BF, 0), (F32, 0), (BF, 1), (F32, 1)])
def test_top_list_distillation_counts_labels_that_are_no_tokens(dtype, slab_mib):
    """stats.n_bad_labels as in cat_loss_fwd_bwd: unmasked rows whose label is outside the vocabulary, whether they have a list or not."""
    T, K, d, V, k = 600, 4, 64, 900, 5
    H, W, _ = rows(T, d, V, 0, dtype)
    y, valid, bad, mask = bad_labels(T, V, 1)
    eng = CatLoss(T, d, V, K, dtype=dtype, slab_mib=slab_mib)
    ids, tl = lists(T, k, V, 2)
    for n_lists in (T, 400):                     # the last rows are without a list
        for m in (valid, None):
            eng.topk_kd_forward_backward(H, W, y, m, ids[:n_lists], tl[:n_lists])
            on = mask if m is not None else torch.ones(T, dtype=torch.bool)
            s = eng.fwd_stats()
            assert s.n_bad_labels == int((on & bad).sum())
            assert s.n_valid == int((on & ~bad)[:n_lists].sum())
    eng.forward_backward(H, W, y, valid.to(torch.uint8))
    assert eng.fwd_stats().n_bad_labels == int((mask & bad).sum())


def test_distillation_from_a_head_counts_labels_that_are_no_tokens():
    T, K, d, V, L = 600, 4, 64, 900, 160
    H, W, _ = rows(T, d, V, 0)
    Ht, Wt, _ = rows(L, d, V, 3)
    y, valid, bad, mask = bad_labels(T, V, 1)
    start = torch.arange(T // K) + 12            # the last blocks run past the target's positions
    has = ((start[:, None] + torch.arange(K)).reshape(-1) < L)
    eng = CatLoss(T, d, V, K)
    for m in (valid.to(torch.uint8), None):
        eng.kd_forward_backward(H, W, y, m, Ht, Wt, start, 0.2)
        on = mask if m is not None else torch.ones(T, dtype=torch.bool)
        s = eng.fwd_stats()
        assert s.n_bad_labels == int((on & bad).sum())
        assert s.n_valid == int((on & ~bad & has).sum())
