"""The order of the alternatives where sums cancel: logits that are small against the products they are made of, so that the error of a
logit has nothing to do with its size.  ids must be those of the exact products all the same (include/cat_loss.h)."""
import numpy as np
import pytest
import torch

from head_ops_util import U, tolerances
from oracle import head_ops_oracle as O
from paper_2605_08632_b200.api import TokenLogProb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().cpu().double().numpy()


def check(H, W, k, **kw):
    """ids exactly those of the 64-bit products (whose own error, 1e-16 of sum |h w|, is far below any gap between two random logits);
    values within the bounds of head_ops_util: an fp32 sum of d products that passes through sum |h w|."""
    T, d = H.shape
    e = TokenLogProb(T, d, W.shape[0], top_k=k, dtype=H.dtype, **kw)
    r = e.forward(H.to(DEV), W.to(DEV))
    assert e.status() == 0
    ref = O.logprob_forward(H, W, None, None, k)
    assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"])
    tol_z, tol_l = tolerances(np64(H), np64(W), ref["on"], ref["z"], H.dtype == BF)
    tol = tol_z + tol_l + 8 * U * np.abs(ref["lse"])
    assert np.all(np.abs(np64(r.lse) - ref["lse"]) <= tol)
    there = ref["top_ids"] >= 0
    want = np.where(there, ref["top_logp"], 0.0)
    assert np.all(np.abs(np64(r.top_logp) - want)[there] <= (tol[:, None] + tol_z + 2 * U * np.abs(want))[there])


# T: the kernel for few rows in its three forms, tiles of rows with large and with small row CTAs
@pytest.mark.parametrize("T", [3, 40, 100, 200, 400])
@pytest.mark.parametrize("d,V,k,c,dtype", [
    (64, 6000, 40, 500.0, BF), (64, 6000, 40, 500.0, F32), (64, 20000, 20, 3000.0, F32), (256, 4096, 20, 1000.0, F32),
    (1024, 9000, 64, 100.0, BF), (2048, 5000, 20, 1000.0, BF), (512, 1500, 256, 3000.0, BF),
])
def test_two_channels_that_cancel(T, d, V, k, c, dtype):
    """The first and the last channel add c and take it off again; every partial sum in between is about c."""
    g = torch.Generator().manual_seed(d + k)
    W, H = 0.02 * torch.randn(V, d, generator=g), torch.randn(T, d, generator=g)
    W[:, 0] = W[:, d - 1] = 1.0
    H[:, 0], H[:, d - 1] = c, -c
    check(H.to(dtype), W.to(dtype), k)


@pytest.mark.parametrize("T,d,V,k,dtype", [(5, 1024, 600, 256, BF), (330, 1024, 600, 256, BF), (20, 768, 512, 256, F32), (130, 4096, 300, 150, BF)])
def test_kth_logit_near_zero(T, d, V, k, dtype):
    """About half the vocabulary is wanted, so the threshold lies among logits near 0."""
    g = torch.Generator().manual_seed(V)
    check(torch.randn(T, d, generator=g).to(dtype), (0.02 * torch.randn(V, d, generator=g)).to(dtype), k)


@pytest.mark.parametrize("T,dtype", [(6, BF), (350, BF), (350, F32)])
def test_outlier_channels(T, dtype):
    """A few channels of the hidden state hundreds of times as large as the others, of either sign, as trained models have them."""
    d, V, k = 1536, 7000, 32
    g = torch.Generator().manual_seed(11)
    H, W = torch.randn(T, d, generator=g), 0.02 * torch.randn(V, d, generator=g)
    at = torch.randperm(d, generator=g)[:6]
    H[:, at] *= 300.0
    W[:, at] = 0.02 * torch.sign(torch.randn(6, generator=g)) * (1 + 0.02 * torch.randn(V, 6, generator=g))
    check(H.to(dtype), W.to(dtype), k)


def test_magnitudes_whose_squares_leave_the_range():
    """Norms of rows whose squares overflow or vanish in fp32: the logits are ordinary."""
    g = torch.Generator().manual_seed(5)
    H, W = torch.randn(4, 128, generator=g), 0.1 * torch.randn(900, 128, generator=g)
    for up in (2.0 ** 70, 2.0 ** -70):
        for dtype in (BF, F32):
            check((H * up).to(dtype), (W / up).to(dtype), 12)
            check((H * up).to(dtype).repeat(80, 1), (W / up).to(dtype), 12)


def test_row_slabs_of_cancelling_sums():
    """Several slabs of rows: each takes its bound from the whole of W."""
    g = torch.Generator().manual_seed(6)
    T, d, V, k = 700, 64, 5000, 12
    W, H = 0.02 * torch.randn(V, d, generator=g), torch.randn(T, d, generator=g)
    W[:, 0] = W[:, d - 1] = 1.0
    H[:, 0], H[:, d - 1] = 900.0, -900.0
    for dtype in (BF, F32):
        check(H.to(dtype), W.to(dtype), k, slab_mib=3)
