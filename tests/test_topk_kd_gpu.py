"""cat_topk_kd_loss_fwd_bwd against the fp64 oracle, through CatLoss.topk_kd_forward_backward; bounds in head_ops_util."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from head_ops_util import U, check_grads, tolerances
from oracle import cat_oracle as C
from oracle import head_ops_oracle as O
from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import CatLoss, TokenLogProb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().cpu().double().numpy()


def make(T, K, d, V, k, dtype, seed=0, L=None, masked=0.2):
    """Lists with all that may stand in one: short and empty ones, ids outside the vocabulary, one id twice, the label, -infinity."""
    g = torch.Generator().manual_seed(seed)
    nb = T // K
    L = L or nb + K - 1
    W = (0.02 * torch.randn(V, d, generator=g)).to(dtype)
    ids = torch.randint(0, V, (L, k), generator=g)
    tl = torch.log_softmax(3 * torch.randn(L, k, generator=g), 1) - 0.1
    drop = torch.rand(L, k, generator=g)
    ids[drop < 0.1] = -1
    ids[(drop > 0.1) & (drop < 0.13)] = V
    tl[(drop > 0.13) & (drop < 0.18)] = -float("inf")
    ids[torch.rand(L, generator=g) < 0.05] = -1
    if k > 2:
        ids[:, k - 1] = torch.where(torch.rand(L, generator=g) < 0.3, ids[:, 0], ids[:, k - 1])
    start = torch.arange(nb)
    y = torch.randint(0, V, (T,), generator=g)
    pos = (start[:, None] + torch.arange(K)).reshape(-1).clamp(max=L - 1)
    y = torch.where(torch.rand(T, generator=g) < 0.5, ids[pos, 0].clamp(0, V - 1), y)
    H = torch.randn(T, d, generator=g)
    Wy = W[y].float()
    H = (H + Wy * (8 * torch.rand(T, generator=g) / (Wy * Wy).sum(1).clamp(min=1e-6)).unsqueeze(1)).to(dtype)
    valid = (torch.rand(T, generator=g) >= masked).to(torch.uint8)
    return H, W, y, valid, ids, tl, start


def run(eng, H, W, y, valid, ids, tl, start, **kw):
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    loss3, dH, dW = eng.topk_kd_forward_backward(dev(H), dev(W), dev(y), dev(valid), dev(ids), dev(tl), dev(start),
                                                 **{k: dev(v) if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
    torch.cuda.synchronize()
    assert eng.topk_kd_status() == 0 and eng.fwd_stats().device_status == 0
    return loss3, dH, dW


def check(eng, out, inputs, K, dW_bf16=False, fixed=None, **kw):
    H, W, y, valid, ids, tl, start = inputs
    loss3, dH, dW = (np64(t) for t in out)
    bf16 = H.dtype == BF
    ref = O.topk_kd(H, W, y, valid, K, ids, tl, start, fixed_decay_gamma=fixed, **kw)
    ok, V = ref["ok"], W.shape[0]
    assert eng.fwd_stats().n_valid == ref["n_valid"]
    tol_z, tol_l = tolerances(np64(H), np64(W), ok, ref["z"], bf16)
    err = tol_z + tol_l + 16 * U * (1 + np.abs(ref["z"]).max())           # of z - lse
    lse, conf, weight = np64(eng.lse), np64(eng.conf), np64(eng.weight)
    assert np.all(np.abs(lse - ref["lse"])[ok] <= err)
    assert np.all(np.abs(conf - ref["conf"])[ok] <= 1.01 * (err + 4 * U) * ref["conf"][ok]) and np.all(conf[~ok] == 1.0)
    w32 = C.cat_weights_f32(eng.conf.cpu().numpy(), ok, K) if fixed is None else C.fixed_decay_weights_f32(fixed, ok, K)
    assert eng.weight.cpu().numpy().tobytes() == w32.tobytes()
    assert np.all(np.abs(weight - ref["weight"]) <= 1.01 * K * (err + 4 * U) * ref["weight"] + 1e-37)
    # each row's term is off by err, and by K err through its weight
    n, beta = max(1, ref["n_valid"]), kw.get("beta", 0.1)
    mass = np.abs(ref["kd"]) + 2.0 * (1 + np.abs(ref["kd"]))
    for got, term in ((loss3[1], ref["ce"]), (loss3[2], ref["kd"])):
        want = float((ref["weight"] * term).sum() / n)
        slack = float((ref["weight"] * (err * (1 + mass) + 1.01 * K * (err + 4 * U) * np.abs(term))).sum() / n) + 4 * U * abs(want)
        assert abs(got - want) <= slack, (got, want, slack)
    assert abs(loss3[0] - (beta * loss3[1] + loss3[2])) <= 4 * U * (beta * abs(loss3[1]) + abs(loss3[2]))
    # dz: the stored z - ref is off by half a step of 2^-9; the weight by K err
    tol = 2 * err + 1.01 * K * (err + 4 * U) + (1.01 * 2.0 ** -10 if bf16 else 0.0)
    Hc = np.where(ok[:, None], np64(H), 0.0)
    check_grads(dH, dW, (ref["dH"], ref["dW"], ref["terms"]), np64(W), Hc, tol, bf16, dW_bf16=dW_bf16)
    assert not dH[~ok].any()
    return ref


@pytest.mark.parametrize("T,K,d,V,k,dtype", [
    (1, 1, 64, 1, 1, BF), (3, 3, 64, 2, 5, BF), (64, 8, 64, 500, 8, BF), (130, 5, 136, 3001, 16, BF), (264, 8, 128, 5003, 64, BF),
    (320, 32, 64, 1000, 256, BF), (66, 33, 72, 900, 3, BF), (128, 8, 64, 1000, 6, BF), (2, 1, 3, 5, 2, F32), (65, 5, 33, 700, 8, F32), (96, 16, 64, 2050, 64, F32),
])
@pytest.mark.parametrize("renorm", [True, False])
def test_matches_oracle(T, K, d, V, k, dtype, renorm):
    x = make(T, K, d, V, k, dtype, seed=T + k)
    eng = CatLoss(T, d, V, K, dtype=dtype)
    out = run(eng, *x, beta=0.3, renormalize=renorm)
    check(eng, out, x, K, beta=0.3, renormalize=renorm)


@pytest.mark.parametrize("dtype,dW_dtype", [(BF, F32), (BF, BF), (F32, F32)])
def test_several_slabs_scale_and_accumulation(dtype, dW_dtype):
    T, K, d, V, k = 1040, 8, 64, 3000, 6
    x = make(T, K, d, V, k, dtype)
    eng = CatLoss(T, d, V, K, dtype=dtype, dW_dtype=dW_dtype, slab_mib=2)
    conf = torch.rand(T, generator=torch.Generator().manual_seed(3)).sqrt()
    out = run(eng, *x, beta=0.0, conf_ext=conf, grad_loss=torch.tensor([0.25]))
    check(eng, out, x, K, dW_bf16=dW_dtype == BF, beta=0.0, conf_ext=conf, g=0.25)
    once = out[2].clone()
    run(eng, *x, beta=0.0, conf_ext=conf, grad_loss=torch.tensor([0.25]), accumulate_dW=True)
    big = float(once.float().abs().max())
    assert torch.allclose(eng.dW.float(), 2 * once.float(), rtol=2 ** -6 if dW_dtype == BF else 2 ** -20, atol=2 ** -20 * big)


def test_fixed_decay_positions_outside_and_unsorted_starts():
    T, K, d, V, k = 120, 4, 64, 600, 5
    H, W, y, valid, ids, tl, start = make(T, K, d, V, k, BF)
    start = torch.randperm(T // K, generator=torch.Generator().manual_seed(1)) - 2      # some before the first, some past the last position
    ids, tl = ids[:25], tl[:25]
    x = (H, W, y, valid, ids, tl, start)
    eng = CatLoss(T, d, V, K, fixed_decay_gamma=0.8)
    ref = check(eng, run(eng, *x, beta=0.5), x, K, fixed=0.8, beta=0.5)
    assert 0 < ref["n_valid"] < int(valid.sum())


def test_without_block_start_every_row_has_its_own_list():
    T, K, d, V, k = 64, 8, 64, 600, 5
    H, W, y, valid, ids, tl, _ = make(T, K, d, V, k, BF, L=50)      # the last 14 rows have none
    x = (H, W, y, valid, ids, tl, None)
    eng = CatLoss(T, d, V, K)
    ref = check(eng, run(eng, *x), x, K)
    assert not ref["ok"][50:].any()


def test_logits_far_from_the_named_ones():
    """Rows whose largest logit is up to 70 nats above all that the list and the label name, and rows with all others 60 and more below."""
    T, K, d, V, k = 160, 4, 64, 500, 3
    H, W, y, valid, ids, tl, start = make(T, K, d, V, k, BF, masked=0.0)
    far = torch.arange(T) % 2 == 0
    named = torch.cat([ids[(start[:, None] + torch.arange(K)).reshape(-1)], y[:, None]], 1)
    other = torch.tensor([next(v for v in range(V) if v not in named[r].tolist()) for r in range(T)])
    token = torch.where(far, other, y)
    Wy = W[token].float()
    H = (H.float() + Wy * (70.0 * torch.rand(T, generator=torch.Generator().manual_seed(4)) / (Wy * Wy).sum(1)).unsqueeze(1)).to(BF)
    x = (H, W, y, valid, ids, tl, start)
    for renorm in (True, False):
        eng = CatLoss(T, d, V, K)
        conf = torch.full((T,), 0.9)
        check(eng, run(eng, *x, beta=0.2, renormalize=renorm, conf_ext=conf), x, K, beta=0.2, renormalize=renorm, conf_ext=conf)


def test_no_row_takes_part_and_padding_may_hold_anything():
    T, K, d, V, k = 72, 8, 64, 500, 4
    for dtype in (BF, F32):
        H, W, y, valid, ids, tl, start = make(T, K, d, V, k, dtype)
        clean, dirty = H.clone(), H.clone()
        clean[valid == 0], dirty[valid == 0] = 0, float("nan")
        a, b = CatLoss(T, d, V, K, dtype=dtype), CatLoss(T, d, V, K, dtype=dtype)
        p, q = run(a, clean, W, y, valid, ids, tl, start), run(b, dirty, W, y, valid, ids, tl, start)
        for s, t in zip(p, q):
            assert torch.equal(s, t) and bool(torch.isfinite(t).all())
        none = torch.zeros_like(valid)
        loss3, dH, dW = run(a, dirty, W, y, none, ids, tl, start)
        assert not loss3.any() and not dH.any() and not dW.any()


def test_pitched_lists_and_refusals():
    T, K, d, V, k = 32, 8, 64, 300, 4
    H, W, y, valid, ids, tl, start = make(T, K, d, V, k, BF)
    eng = CatLoss(T, d, V, K)
    a = [t.clone() for t in run(eng, H, W, y, valid, ids, tl, start)]
    L = ids.shape[0]
    wi, wt = torch.full((L, k + 3), 9, device=DEV), torch.full((L, k + 3), 50.0, device=DEV)
    wi[:, :k], wt[:, :k] = ids.to(DEV), tl.to(DEV)
    b = eng.topk_kd_forward_backward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV).bool(), wi[:, :k], wt[:, :k], start.to(DEV))
    for s, t in zip(a, b):
        assert torch.equal(s, t)
    g = [t.to(DEV) for t in (H, W, y, valid, ids, tl, start)]
    for i, bad in ((4, g[4].int()), (5, g[5].double()), (2, g[2].float()), (0, g[0].float())):
        with pytest.raises(TypeError):
            eng.topk_kd_forward_backward(*(bad if j == i else t for j, t in enumerate(g)))
    for i, bad in ((4, wi[:, :k]), (5, g[5][:, :3]), (6, g[6][:2]), (6, start), (0, g[0][:8])):
        with pytest.raises(ValueError):
            eng.topk_kd_forward_backward(*(bad if j == i else t for j, t in enumerate(g)))
    with pytest.raises(ValueError):
        eng.topk_kd_forward_backward(*g, beta=-1.0)


def test_pitched_rows_leave_the_gaps_alone():
    T, K, d, V, k = 264, 8, 72, 900, 5
    for dtype, wdt in ((BF, BF), (BF, F32), (F32, F32)):
        H, W, y, valid, ids, tl, start = (t.to(DEV) for t in make(T, K, d, V, k, dtype))
        eng = CatLoss(T, d, V, K, dtype=dtype, dW_dtype=wdt)
        loss3, dH, dW = eng.topk_kd_forward_backward(H, W, y, valid, ids, tl, start)
        code = {BF: B.CAT_BF16, F32: B.CAT_F32}
        ldH, ldW = d + 24, d + 8
        shape = B.make_shape(T, d, V, K, code[dtype], code[wdt], ldH=ldH, ldW=ldW)
        desc = B.make_topk_kd_desc(ids.shape[0], k, 0.1)
        wH, wW = torch.full((T, ldH), float("nan"), dtype=dtype, device=DEV), torch.full((V, ldW), float("nan"), dtype=dtype, device=DEV)
        wH[:, :d], wW[:, :d] = H, W
        pH, pW = torch.full((T, ldH), 7.0, dtype=dtype, device=DEV), torch.full((V, ldW), 7.0, dtype=wdt, device=DEV)
        n = B.cat_topk_kd_workspace_bytes(shape, desc)
        ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
        out = [torch.empty(3, device=DEV)] + [torch.empty(T, device=DEV) for _ in range(3)]
        B.cat_topk_kd_loss_fwd_bwd(shape, desc, wH, wW, y, valid, ids, tl, start, None, None, *out, None, pH, pW, False, ws[:n])
        assert torch.equal(out[0], loss3) and torch.equal(pH[:, :d], dH) and torch.equal(pW[:, :d], dW)
        assert bool((pH[:, d:] == 7.0).all()) and bool((pW[:, d:] == 7.0).all()) and bool((ws[n:] == 0xA5).all())


def test_offsets_past_31_bits():
    """A slab of more than 2^31 logits: the blocks at its end against the oracle."""
    T, K, d, V, k = 13504, 8, 64, 160001, 3
    H, W, y, valid, ids, tl, start = make(T, K, d, V, k, BF)
    eng = CatLoss(T, d, V, K, slab_mib=8192)
    loss3, dH, _ = run(eng, H, W, y, valid, ids, tl, start, beta=0.3)
    rows = slice(T - 40, T)
    ref = O.topk_kd(H[rows], W, y[rows], valid[rows], K, ids, tl, start[-5:], beta=0.3)
    n = eng.fwd_stats().n_valid
    want = ref["dH"] * ref["n_valid"] / n
    # roundings of dz and of the result (2^-8 each), of z - ref (2^-10)
    assert np.linalg.norm(np64(dH[rows]) - want) <= (2 * 2.0 ** -8 + 2.0 ** -10) * np.linalg.norm(want)
    assert np.abs(np64(eng.lse[rows]) - ref["lse"])[ref["ok"]].max() <= 1e-4


def test_repeatable_captured_and_on_another_stream():
    T, K, d, V, k = 256, 8, 128, 4000, 16
    x = [t.to(DEV) for t in make(T, K, d, V, k, BF)]
    eng = CatLoss(T, d, V, K)
    a = [t.clone() for t in eng.topk_kd_forward_backward(*x)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = [t.clone() for t in eng.topk_kd_forward_backward(*x)]
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = eng.topk_kd_forward_backward(*x)
    eng.dH.zero_(), eng.dW.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for p, q, r in zip(a, b, c):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_lists_written_by_one_operator_train_the_other():
    """The whole path: a teacher head scores a sequence and writes its lists, its confidences weigh the draft's rows, and the step
    distils from the lists; a list of the whole vocabulary gives what distilling from the teacher's head gives."""
    T, K, d, V = 64, 8, 64, 256
    H, W, y, valid, _, _, start = make(T, K, d, V, 4, BF, masked=0.0)
    L = T // K + K - 1
    g = torch.Generator().manual_seed(8)
    Ht, Wt = (3 * torch.randn(L, d, generator=g)).to(BF), (0.05 * torch.randn(V, d, generator=g)).to(BF)
    seq = torch.randint(0, V, (L,), generator=g)
    teacher = TokenLogProb(L, d, V, top_k=V)
    r = teacher.forward(Ht.to(DEV), Wt.to(DEV), seq.to(DEV))
    conf = torch.empty(T, device=DEV)
    B.cat_conf_window(r.logp.exp(), L, start.to(DEV), T // K, K, conf)
    eng = CatLoss(T, d, V, K)
    loss3, dH, dW = (t.clone() for t in eng.topk_kd_forward_backward(H.to(DEV), W.to(DEV), y.to(DEV), None, r.top_ids, r.top_logp,
                                                                    start.to(DEV), beta=0.2, renormalize=False, conf_ext=conf))
    ref, oH, oW = C.cat_kd_forward_backward(H, W, y, None, K, Ht, Wt, start, 0.2, conf_ext=conf.cpu().numpy())
    assert abs(float(loss3[0]) - ref["loss"]) <= 1e-4 * ref["loss"]
    # dz and the result are rounded to bf16 (2^-8 each), z - ref to steps of 2^-9
    assert np.linalg.norm(np64(dH) - oH) <= 2 ** -6 * np.linalg.norm(oH) and np.linalg.norm(np64(dW) - oW) <= 2 ** -6 * np.linalg.norm(oW)
    other = CatLoss(T, d, V, K)
    full3, fH, fW = other.kd_forward_backward(H.to(DEV), W.to(DEV), y.to(DEV), None, Ht.to(DEV), Wt.to(DEV), start, 0.2, conf_ext=conf)
    assert abs(float(full3[0]) - float(loss3[0])) <= 2e-3 * float(loss3[0])
    # a top-16 list keeps most of the teacher's mass: the step points the same way
    few = TokenLogProb(L, d, V, top_k=16).forward(Ht.to(DEV), Wt.to(DEV))
    assert torch.equal(few.top_ids, r.top_ids[:, :16])


def test_without_cta_pairs():
    """The one-CTA kernels (128-row tiles) in a process of their own: the choice is made once per process."""
    here = os.path.dirname(os.path.abspath(__file__))
    pick = "matches_oracle or slabs or guarded or pitched or padding"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.join(here, "test_logprob_gpu.py"),
                        os.path.join(here, "test_topk_kd_gpu.py"), "-k", pick], env=dict(os.environ, CAT_LOSS_CTA_PAIR="0"),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]
