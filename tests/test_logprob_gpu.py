"""cat_logprob_fwd / cat_logprob_bwd against the fp64 oracle, through the public classes; bounds in head_ops_util."""
import math

import numpy as np
import pytest
import torch

from head_ops_util import U, check_grads, tolerances
from oracle import head_ops_oracle as O
from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import LogProbModule, TokenLogProb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make(T, d, V, dtype, seed=0, masked=0.2, sure=0.5):
    g = torch.Generator().manual_seed(seed)
    W = (0.02 * torch.randn(V, d, generator=g)).to(dtype)
    H = torch.randn(T, d, generator=g)
    y = torch.randint(0, V, (T,), generator=g)
    amount = 12.0 * torch.rand(T, generator=g) * (torch.rand(T, generator=g) < sure)
    Wy = W[y].float()
    H = (H + Wy * (amount / (Wy * Wy).sum(1).clamp(min=1e-6)).unsqueeze(1)).to(dtype)
    valid = (torch.rand(T, generator=g) >= masked).to(torch.uint8)
    y = torch.where(torch.rand(T, generator=g) < 0.05, torch.full_like(y, V + 3), y)
    return H, W, y, valid


def np64(t):
    return t.detach().cpu().double().numpy()


def check_forward(r, H, W, y, valid, k, bf16):
    ref = O.logprob_forward(H, W, y, valid, k)
    on = ref["on"]
    tol_z, tol_l = tolerances(np64(H), np64(W), on, ref["z"], bf16)
    lse = np64(r.lse)
    tol = tol_z + tol_l + 8 * U * np.abs(ref["lse"])
    assert np.all(np.abs(lse - ref["lse"]) <= tol)
    V = W.shape[0]
    assert np.all(np.abs(np64(r.entropy) - ref["entropy"]) <= 4 * (1 + math.log(V)) * (tol_z + tol_l))
    if y is not None:
        assert np.all(np.abs(np64(r.logp) - ref["logp"]) <= tol + 2 * U * np.abs(ref["logp"]))
        assert not np64(r.logp)[~ref["known"]].any()
    if k:
        ids, tl = r.top_ids.cpu().numpy(), np64(r.top_logp)
        assert np.array_equal(ids, ref["top_ids"])
        there = ref["top_ids"] >= 0
        assert np.all(np.isneginf(tl[~there]))
        want = np.where(there, ref["top_logp"], 0.0)
        assert np.all(np.abs(tl - want)[there] <= (tol[:, None] + 2 * U * np.abs(want))[there])
    assert not lse[~on].any() and not np64(r.entropy)[~on].any()
    return ref


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,d,V,k,dtype", [
    (1, 64, 1, 1, BF), (1, 64, 3, 8, BF), (1, 512, 5003, 20, BF), (2, 8, 33, 33, BF), (3, 72, 256, 256, BF), (5, 128, 257, 1, BF),
    (37, 256, 8191, 64, BF), (130, 136, 20011, 5, BF), (257, 256, 12000, 20, BF), (600, 128, 3000, 0, BF),
    (32, 64, 30000, 20, BF), (33, 200, 20001, 8, BF), (64, 1024, 9473, 64, BF), (65, 64, 14209, 20, BF), (127, 72, 40000, 3, BF),
    (128, 2048, 19000, 20, BF), (129, 64, 14209, 20, BF), (128, 64, 700, 0, BF), (16, 64, 18945, 0, BF),
    (1, 3, 1, 2, F32), (7, 5, 63, 64, F32), (65, 33, 129, 7, F32), (130, 100, 4097, 20, F32), (70, 64, 2500, 0, F32),
])
def test_forward_matches_oracle(T, d, V, k, dtype):
    H, W, y, valid = make(T, d, V, dtype, seed=T + V)
    e = TokenLogProb(T, d, V, top_k=k, dtype=dtype)
    r = e.forward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV))
    check_forward(r, H, W, y, valid, k, dtype == BF)
    assert e.status() == 0
    # no mask, no labels: the other outputs alone
    r = e.forward(H.to(DEV), W.to(DEV))
    assert r.logp is None
    check_forward(r, H, W, None, None, k, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_row_slabs_give_the_same(dtype):
    T, d, V, k = 1100, 64, 5000, 12
    H, W, y, valid = (t.to(DEV) for t in make(T, d, V, dtype))
    whole = TokenLogProb(T, d, V, k, dtype=dtype).forward(H, W, y, valid)
    e = TokenLogProb(T, d, V, k, dtype=dtype, slab_mib=3)
    cut = e.forward(H, W, y, valid)
    assert e.ws.numel() < TokenLogProb(T, d, V, k, dtype=dtype).ws.numel()
    assert torch.equal(whole.top_ids, cut.top_ids)
    check_forward(cut, H.cpu(), W.cpu(), y.cpu(), valid.cpu(), k, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_equal_logits_and_rows_of_zeros(dtype):
    """Equal rows of W tie exactly; a zero row of H ties everything; a common offset crowds the stored logits' rounding."""
    T, d, V, k = 6, 64, 6000, 40
    H, W, y, _ = make(T, d, V, dtype, sure=0.0)
    W[1000:3000] = W[7]                     # 2001 equal rows, more than are held at a time
    H[0] = 0
    H[1] = (W[7].float() * 30).to(dtype)    # ... and they are this row's largest
    H[2] = -(W[7].float() * 30).to(dtype)
    W[:, 0] = 1.0
    H[3, 0] = 500.0                         # logits of 500 +- 1: the fp16 copies step by 0.25 to 0.5
    H[4] = 0
    H[4, 0] = 3.0                           # all equal, and not zero
    r = TokenLogProb(T, d, V, k, dtype=dtype).forward(H.to(DEV), W.to(DEV), y.to(DEV))
    ref = check_forward(r, H, W, y, None, k, dtype == BF)
    assert ref["top_ids"][0].tolist() == list(range(k)) == ref["top_ids"][4].tolist()
    assert ref["top_ids"][1].tolist() == [7] + list(range(1000, 1000 + k - 1))


def test_padding_may_hold_anything_and_other_rows_are_untouched():
    T, d, V, k = 70, 64, 1000, 9
    for dtype in (BF, F32):
        H, W, y, valid = make(T, d, V, dtype)
        clean = H.clone()
        clean[valid == 0] = 0
        H[valid == 0] = float("nan")
        H[int(np.nonzero(valid.numpy() == 0)[0][0])] = float("inf")
        gl, ge = torch.randn(T), torch.randn(T)
        e, f = (TokenLogProb(T, d, V, k, dtype=dtype) for _ in range(2))
        a, b = e.forward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV)), f.forward(clean.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV))
        for x, z in zip(a, b):
            assert torch.equal(x, z)
        ga = e.backward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV), gl.to(DEV), ge.to(DEV))
        gb = f.backward(clean.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV), gl.to(DEV), ge.to(DEV))
        assert torch.equal(ga[0], gb[0]) and torch.equal(ga[1], gb[1]) and bool(torch.isfinite(ga[1]).all())
        assert not ga[0][valid.to(DEV) == 0].any()


def test_rows_that_are_not_finite_say_so():
    T, d, V, k = 5, 64, 700, 6
    H, W, y, _ = make(T, d, V, BF)
    H[1, 3] = float("nan")
    H[3, 0] = float("inf")
    r = TokenLogProb(T, d, V, k).forward(H.to(DEV), W.to(DEV), y.clamp(max=V - 1).to(DEV))
    for i in range(T):
        bad = i in (1, 3)
        assert bool(torch.isnan(r.entropy[i])) == bad and bool(torch.isfinite(r.lse[i])) != bad
        assert bool((r.top_ids[i] == -1).all()) == bad and bool(torch.isnan(r.top_logp[i]).all()) == bad


@pytest.mark.parametrize("T,d,V,dtype,dW_dtype,slab_mib", [
    (1, 64, 1, BF, F32, 0), (3, 64, 300, BF, BF, 0), (130, 136, 5003, BF, F32, 0), (300, 256, 3000, BF, BF, 1), (520, 64, 1111, BF, F32, 1),
    (1, 3, 2, F32, F32, 0), (70, 33, 1025, F32, F32, 0), (200, 64, 2000, F32, F32, 1),
])
@pytest.mark.parametrize("which", ["logp", "entropy", "both"])
def test_backward_matches_oracle(T, d, V, dtype, dW_dtype, slab_mib, which):
    H, W, y, valid = make(T, d, V, dtype, seed=V)
    g = torch.Generator().manual_seed(5)
    gl = torch.randn(T, generator=g) if which != "entropy" else None
    ge = 0.3 * torch.randn(T, generator=g) if which != "logp" else None
    e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=dW_dtype, slab_mib=slab_mib)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    e.forward(dev(H), dev(W), dev(y), dev(valid))
    dH, dW = e.backward(dev(H), dev(W), dev(y) if gl is not None else None, dev(valid), dev(gl), dev(ge))
    assert e.bwd_status() == 0
    on = O.logprob_forward(H, W, y, valid)["on"]
    z = O.logprob_forward(H, W, y, valid)["z"]
    tol_z, tol_l = tolerances(np64(H), np64(W), on, z, dtype == BF)
    ref = O.logprob_backward(H, W, y if gl is not None else None, valid, gl, ge)
    # p is off by the error of z - lse; the entropy's coefficient by that of log p + entropy, held against |log p| + entropy
    tol = 2 * tol_z + tol_l + 16 * U * (1 + np.abs(z).max()) + 4 * (1 + math.log(V)) * (tol_z + tol_l)
    Hc = np.where(on[:, None], np64(H), 0.0)
    check_grads(np64(dH), np64(dW), ref, np64(W), Hc, tol, dtype == BF, dW_bf16=dW_dtype == BF)
    # added to what dW holds
    again = dW.clone()
    dH2, dW2 = e.backward(dev(H), dev(W), dev(y) if gl is not None else None, dev(valid), dev(gl), dev(ge), accumulate_dW=True)
    assert torch.allclose(dW2.float(), 2 * again.float(), rtol=2 ** -7 if dW_dtype == BF else 2 ** -22, atol=1e-30)


def test_backward_against_differences():
    """f(H + h D, W + h E) - f(H - h D, W - h E) over 2 h, f from the fp32 forward pass.  h = 2^-6: the third derivative's part is below
    h^2, and the forward's error (a few 1e-6 a row, T rows) over 2 h below 3e-3."""
    T, d, V = 40, 32, 500
    H, W, y, _ = make(T, d, V, F32, sure=0.0)
    y = y.clamp(max=V - 1)
    g = torch.Generator().manual_seed(2)
    gl, ge = torch.randn(T, generator=g), torch.randn(T, generator=g)
    D, E = torch.randn(T, d, generator=g) / math.sqrt(T * d), torch.randn(V, d, generator=g) / math.sqrt(V * d)
    e = TokenLogProb(T, d, V, dtype=F32)

    def f(H, W):
        r = e.forward(H.to(DEV), W.to(DEV), y.to(DEV))
        return float((gl.double() * r.logp.cpu().double() + ge.double() * r.entropy.cpu().double()).sum())

    h = 2.0 ** -6
    slope = (f(H + h * D, W + h * E) - f(H - h * D, W - h * E)) / (2 * h)
    e.forward(H.to(DEV), W.to(DEV), y.to(DEV))
    dH, dW = e.backward(H.to(DEV), W.to(DEV), y.to(DEV), None, gl.to(DEV), ge.to(DEV))
    got = float((dH.cpu().double() * D).sum() + (dW.cpu().double() * E).sum())
    assert abs(got - slope) <= 3e-3 + h * h


def test_strided_inputs_and_guarded_outputs():
    T, d, V, k = 33, 64, 777, 5
    H, W, y, valid = make(T, d, V, BF)
    wide_H, wide_W = torch.full((T, d + 24), float("nan"), dtype=BF, device=DEV), torch.full((V, d + 8), float("nan"), dtype=BF, device=DEV)
    wide_H[:, :d] = H.to(DEV)
    wide_W[:, :d] = W.to(DEV)
    e = TokenLogProb(T, d, V, k)
    a = [t.clone() for t in e.forward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV))]
    b = e.forward(wide_H[:, :d], wide_W[:, :d], y.to(DEV), valid.to(DEV).bool())
    for x, z in zip(a, b):
        assert torch.equal(x, z)
    with pytest.raises(ValueError):
        e.backward(wide_H[:, :d], wide_W[:, :d], y.to(DEV), None, e.logp)
    with pytest.raises(B.CatError) as err:      # a pitch that TMA cannot take
        e.forward(torch.zeros(T, d + 4, dtype=BF, device=DEV)[:, :d], W.to(DEV))
    assert err.value.code == -4
    # nothing is written past the outputs
    shape = B.make_shape(T, d, V, 1, B.CAT_BF16)
    n = B.cat_logprob_workspace_bytes(shape, k, 0)
    big = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    out = [torch.full((T + 8,), 7.0, device=DEV) for _ in range(3)]
    ids, tl = torch.full((T + 8, k), 77, dtype=torch.int64, device=DEV), torch.full((T + 8, k), 7.0, device=DEV)
    B.cat_logprob_fwd(shape, H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV), k, out[0], out[1], out[2], ids, tl, big[:n])
    torch.cuda.synchronize()
    assert bool((big[n:] == 0xA5).all()) and all(bool((o[T:] == 7.0).all()) for o in out)
    assert bool((ids[T:] == 77).all()) and bool((tl[T:] == 7.0).all())
    assert torch.equal(out[0][:T], a[0]) and torch.equal(ids[:T], a[3])


def test_refusals_of_the_python_layer():
    e = TokenLogProb(8, 64, 100, 4)
    H, W, y = torch.zeros(8, 64, dtype=BF, device=DEV), torch.zeros(100, 64, dtype=BF, device=DEV), torch.zeros(8, dtype=torch.int64, device=DEV)
    for bad in (lambda: e.forward(H.float(), W, y), lambda: e.forward(H, W, y.int())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: e.forward(H[:4], W, y), lambda: e.forward(H, W, y.cpu()), lambda: e.forward(H.cpu(), W, y),
                lambda: e.backward(H, W, None, None, e.logp), lambda: e.backward(H, W, y, None, e.logp, accumulate_dW=True),
                lambda: TokenLogProb(8, 60, 100), lambda: TokenLogProb(8, 64, 100, top_k=B.CAT_TOPK_MAX + 1)):
        with pytest.raises(ValueError):
            bad()


def test_streams_graphs_and_repeatability():
    T, d, V, k = 96, 128, 4000, 16
    H, W, y, valid = (t.to(DEV) for t in make(T, d, V, BF))
    gl, ge = torch.randn(T, device=DEV), torch.randn(T, device=DEV)
    e = TokenLogProb(T, d, V, k)
    first = [t.clone() for t in e.forward(H, W, y, valid)] + [t.clone() for t in e.backward(H, W, y, valid, gl, ge)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = [t.clone() for t in e.forward(H, W, y, valid)] + [t.clone() for t in e.backward(H, W, y, valid, gl, ge)]
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = e.forward(H, W, y, valid)
        dH, dW = e.backward(H, W, y, valid, gl, ge)
    for _ in range(2):
        e.dH.zero_(), e.dW.zero_(), e.lse.zero_(), e.top_ids.zero_()
        graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, list(r) + [dH, dW]):
        assert torch.equal(a, b) and torch.equal(a, c)
    # new inputs in the captured buffers
    H2 = make(T, d, V, BF, seed=9)[0]
    H.copy_(H2)
    graph.replay()
    check_forward(r, H2, W.cpu(), y.cpu(), valid.cpu(), k, True)


def test_nothing_to_do_and_no_gradient():
    T, d, V, k = 40, 64, 500, 4
    for dtype in (BF, F32):
        H, W, y, valid = (t.to(DEV) for t in make(T, d, V, dtype))
        e = TokenLogProb(T, d, V, k, dtype=dtype)
        r = e.forward(H, W, y, torch.zeros_like(valid))
        assert not r.logp.any() and not r.lse.any() and not r.entropy.any()
        assert bool((r.top_ids == -1).all()) and bool(torch.isneginf(r.top_logp).all())
        g = torch.ones(T, device=DEV)
        dH, dW = e.backward(H, W, y, torch.zeros_like(valid), g, g)
        assert not dH.any() and not dW.any()
        e.forward(H, W, y, valid)
        dH, dW = e.backward(H, W, None, valid)
        assert not dH.any() and not dW.any()


def test_offsets_past_31_bits():
    """A slab of more than 2^31 logits: the rows at its end against the oracle."""
    T, d, V, k = 13500, 64, 160001, 3
    H, W, y, _ = make(T, d, V, BF, sure=0.0)
    y = y.clamp(max=V - 1)
    e = TokenLogProb(T, d, V, k, slab_mib=8192)
    r = e.forward(H.to(DEV), W.to(DEV), y.to(DEV))
    rows = slice(T - 40, T)
    part = type(r)(r.logp[rows], r.lse[rows], r.entropy[rows], r.top_ids[rows], r.top_logp[rows])
    check_forward(part, H[rows], W, y[rows], None, k, True)
    g = torch.zeros(T)
    g[rows] = 1.0
    dH, _ = e.backward(H.to(DEV), W.to(DEV), y.to(DEV), None, g.to(DEV))
    ref = O.logprob_backward(H[rows], W, y[rows], None, np.ones(40))
    assert not dH[: T - 40].any()
    assert np.linalg.norm(np64(dH[rows]) - ref[0]) <= 2 * 2.0 ** -8 * np.linalg.norm(ref[0])


def test_pitched_gradients_leave_the_gaps_alone():
    T, d, V = 300, 72, 1000
    for dtype, wdt in ((BF, BF), (BF, F32), (F32, F32)):
        H, W, y, valid = make(T, d, V, dtype)
        code = {BF: B.CAT_BF16, F32: B.CAT_F32}
        ldH, ldW = d + 24, d + 8
        shape = B.make_shape(T, d, V, 1, code[dtype], code[wdt], ldH=ldH, ldW=ldW)
        wH, wW = torch.full((T, ldH), float("nan"), dtype=dtype, device=DEV), torch.full((V, ldW), float("nan"), dtype=dtype, device=DEV)
        wH[:, :d], wW[:, :d] = H.to(DEV), W.to(DEV)
        gl = torch.randn(T, device=DEV)
        e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=wdt)
        r = e.forward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV))
        dH, dW = e.backward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV), gl, gl)
        pH, pW = torch.full((T, ldH), 7.0, dtype=dtype, device=DEV), torch.full((V, ldW), 7.0, dtype=wdt, device=DEV)
        ws = torch.empty(B.cat_logprob_workspace_bytes(shape, 0, 1), dtype=torch.uint8, device=DEV)
        B.cat_logprob_bwd(shape, wH, wW, y.to(DEV), valid.to(DEV), r.lse, r.entropy, gl, gl, pH, pW, False, ws)
        assert torch.equal(pH[:, :d], dH) and torch.equal(pW[:, :d], dW)
        assert bool((pH[:, d:] == 7.0).all()) and bool((pW[:, d:] == 7.0).all())


def test_two_engines_on_two_streams():
    T, d, V, k = 64, 256, 20000, 8
    a, b = make(T, d, V, BF, seed=1), make(T, d, V, BF, seed=2)
    x, z = [t.to(DEV) for t in a], [t.to(DEV) for t in b]
    e, f = TokenLogProb(T, d, V, k), TokenLogProb(T, d, V, k)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s1):
            r = e.forward(*x)
        with torch.cuda.stream(s2):
            q = f.forward(*z)
    torch.cuda.synchronize()
    check_forward(r, *a, k, True)
    check_forward(q, *b, k, True)


def test_module_gradients():
    T, d, V = 50, 64, 900
    H, W, y, valid = make(T, d, V, F32, sure=0.0)
    head = LogProbModule(W.to(DEV), top_k=3)
    h = H.to(DEV).requires_grad_()
    logp, entropy, ids, tl = head(h, y.to(DEV), valid.to(DEV))
    head(torch.zeros_like(h), y.to(DEV), valid.to(DEV))          # another call through the same engine before backward
    gl, ge = torch.randn(T), torch.randn(T)
    (logp * gl.to(DEV) + entropy * ge.to(DEV)).sum().backward()
    dH, dW, *_ = O.logprob_backward(H, W, y, valid, gl, ge)
    assert np.linalg.norm(np64(h.grad) - dH) <= 1e-5 * np.linalg.norm(dH)
    assert np.linalg.norm(np64(head.weight.grad) - dW) <= 1e-5 * np.linalg.norm(dW)
    assert not ids.requires_grad and not tl.requires_grad
    on_dev = y.to(DEV), valid.to(DEV)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="captured"):
        with torch.cuda.graph(graph):
            head(h, *on_dev)
    h.grad = None
    head(h, None, valid.to(DEV))[1].sum().backward()             # without labels: the entropy alone
    dH, *_ = O.logprob_backward(H, W, None, valid, None, np.ones(T))
    assert np.linalg.norm(np64(h.grad) - dH) <= 1e-5 * np.linalg.norm(dH)


def sure_rows(T, d, V, dtype, seed, rest):
    """Rows whose label has all but about `rest` of the probability."""
    g = torch.Generator().manual_seed(seed)
    W = (0.02 * torch.randn(V, d, generator=g)).to(dtype)
    y = torch.randint(0, V, (T,), generator=g)
    Wy = W[y].float()
    H = 0.3 * torch.randn(T, d, generator=g)
    up = math.log(V / rest) - (H * Wy).sum(1)
    H = (H + Wy * (up / (Wy * Wy).sum(1)).unsqueeze(1)).to(dtype)
    return H, W, y


@pytest.mark.parametrize("d,V,dtype,rest", [(96, 700, F32, 1e-5), (320, 3001, F32, 1e-4), (128, 2500, BF, 1e-2), (512, 1111, BF, 1e-2)])
def test_gradient_of_rows_that_are_sure_of_their_label(d, V, dtype, rest):
    """1 - p of such a row is small against p: the label's entry may not be the difference of a rounded p from 1.

    Every entry v != y of dz is p_v gl with p_v off by a factor exp(e), |e| <= tol_z (its logit) + tol_l (lse), and the label's entry, gl (1 - p), is
    off by no more than they are (fp32: their sum) or, from its exact logit (bf16), by the error of lse against 1 - p: lse = m + log l
    rounds to U |lse| and log l to 2 U, and l is off by tol_z of its part outside the largest logit, 1 - p of it.  dH is one row of products
    of dz with W: sum |dz| |W| times that, V + 16 roundings of its sum, and for bf16 the rounding of the result.
    """
    T = 6
    H, W, y = sure_rows(T, d, V, dtype, 3, rest)
    e = TokenLogProb(T, d, V, dtype=dtype, dW_dtype=dtype)
    f = e.forward(H.to(DEV), W.to(DEV), y.to(DEV))
    gl = torch.linspace(0.5, 2.0, T)
    dH, _ = e.backward(H.to(DEV), W.to(DEV), y.to(DEV), None, gl.to(DEV))
    bf16 = dtype == BF
    z = np64(H) @ np64(W).T
    m = z.max(1, keepdims=True)
    lse = m[:, 0] + np.log(np.exp(z - m).sum(1))
    p = np.exp(z - lse[:, None])
    at = np.arange(T), y.numpy()
    q = p.copy()
    q[at] = 0.0
    left = q.sum(1)                      # 1 - p, without the difference
    # the others' logits are normal with s = |label's logit| / sqrt(d), and exp of them averages e^(s^2 / 2): at most 5.5 for these sizes
    assert (left < 50 * rest).all() and (left > 0).all()
    dz = -np.asarray(gl)[:, None] * q
    dz[at] = np64(gl) * left
    tol_z, tol_l = tolerances(np64(H), np64(W), np.ones(T, bool), z, bf16)
    rel = tol_z + tol_l + 8 * U * np.abs(lse)
    label = rel + (((U * np.abs(lse) + 4 * U) / left + tol_z) if bf16 else 0.0)
    err = (np.abs(dz) * rel[:, None])
    err[at] = np64(gl) * left * label
    want = dz @ np64(W)
    tol = err @ np.abs(np64(W)) + (V + 16) * U * (np.abs(dz) @ np.abs(np64(W)))
    if bf16:                             # dz in two terms (2^-16 of it), the result rounded once
        tol = tol * 1.01 + 2.0 ** -16 * (np.abs(dz) @ np.abs(np64(W))) + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(np64(dH) - want) <= tol)
    # and its log probability, the logarithm of 1 - (1 - p): off by rel of 1 - p, and by the roundings of l near 1 and of log l
    assert np.all(np.abs(np64(f.logp) - np.log1p(-left)) <= rel * left + 6 * U)


@pytest.mark.parametrize("T,dtype", [(5, BF), (400, BF), (70, F32)])
def test_a_label_among_the_alternatives_has_one_log_probability(T, dtype):
    """The two outputs take the label's logit from the same sum, whichever way the other alternatives' are taken."""
    H, W, y, valid = make(T, 768, 3000, dtype, seed=9, sure=0.9)
    e = TokenLogProb(T, 768, 3000, top_k=12, dtype=dtype)
    r = e.forward(H.to(DEV), W.to(DEV), y.to(DEV), valid.to(DEV))
    there = r.top_ids == y.to(DEV).unsqueeze(1)
    rows = there.any(1)
    assert rows.sum() > T // 4
    same = r.top_logp[there] == r.logp[rows]
    assert bool(same.all())


def test_alternatives_are_as_exact_as_the_label():
    """Few rows: alternatives are fp32 sums of d products (four chains of d / 128 a lane, and the lanes' five steps), lse is off by at most the
    tensor cores' truncation of what lies outside the largest logit, a tenth of it after the correction, and by its rounding."""
    T, d, V, k = 3, 3928, 2048, 20
    H, W, y, _ = make(T, d, V, BF, seed=4, masked=0.0, sure=1.0)
    r = TokenLogProb(T, d, V, top_k=k, dtype=BF).forward(H.to(DEV), W.to(DEV), None)
    z = np64(H) @ np64(W).T
    lse = z.max(1) + np.log(np.exp(z - z.max(1, keepdims=True)).sum(1))
    ids = np.argsort(-z, axis=1, kind="stable")[:, :k]
    assert np.array_equal(r.top_ids.cpu().numpy(), ids)
    size = np.abs(np64(H)) @ np.abs(np64(W)).T
    sums = (d / 128 + 8) * U * np.take_along_axis(size, ids, 1)
    cut = (d / 16) * 2 * U * np.abs(z).max(1)           # d / 16 truncations of a sum that stays within the largest logit: up to 2 U each
    tol = sums + 0.2 * cut[:, None] + 4 * U * np.abs(lse)[:, None]
    assert np.all(np.abs(np64(r.top_logp) - (np.take_along_axis(z, ids, 1) - lse[:, None])) <= tol)


@pytest.mark.parametrize("T,dW_dtype,accumulate,masked", [(129, BF, False, 0.3), (300, F32, False, 0.0), (300, BF, True, 0.2), (1024, F32, True, 0.1)])
def test_labels_entries_of_dz_are_not_rounded(T, dW_dtype, accumulate, masked):
    """Batches of 129 to 1024 bf16 rows: the label's entry of dz, nearly all of its row here, reaches both gradients unrounded, several rows of one
    label among them.  What stays rounded (2^-8) is the rest of dz, p_v of about 1 / V each; fp32 sums add (T + 16) U; bf16
    results are rounded once, 2^-8.  Were the labels' entries rounded, results would be off by up to 2^-8 more."""
    d, V = 96, 2000
    g = torch.Generator().manual_seed(T)
    W = 0.01 * torch.randn(V, d, generator=g)
    names = torch.tensor([3, 700, 701, 1280, V - 1])
    W[names] *= 100.0
    W = W.to(BF)
    H = (0.01 * torch.randn(T, d, generator=g)).to(BF)
    y = names[torch.randint(0, 5, (T,), generator=g)]
    y[::17] = V + 1                                   # no token
    valid = (torch.rand(T, generator=g) >= masked).to(torch.uint8)
    gl = torch.randn(T, generator=g)
    e = TokenLogProb(T, d, V, dtype=BF, dW_dtype=dW_dtype)
    e.dW = torch.randn(V, d, generator=g).to(dW_dtype).to(DEV) if accumulate else None
    before = np64(e.dW) if accumulate else 0.0
    Hd = H.to(DEV)
    Hd[(valid == 0).to(DEV)] = float("nan")
    e.forward(Hd, W.to(DEV), y.to(DEV), valid.to(DEV))
    dH, dW = e.backward(Hd, W.to(DEV), y.to(DEV), valid.to(DEV), gl.to(DEV), accumulate_dW=accumulate)
    known = (valid.numpy() != 0) & (y.numpy() < V)
    z = np64(H) @ np64(W).T
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    c = np.where(known, np64(gl), 0.0)
    rest = -c[:, None] * p
    label = np.zeros_like(rest)
    at = np.arange(T)[known], y.numpy()[known]
    label[at] = c[known] * (1.0 - p[at])
    rest[at] = 0.0
    tol_z, tol_l = tolerances(np64(H), np64(W), known, z, True)
    e_rest, e_label = 2.0 ** -8 + 2 * (tol_z + tol_l), 4 * (tol_z + tol_l) + (T + 16) * U
    for got, want, size_rest, size_label, bf16 in (
            (np64(dH), (rest + label) @ np64(W), np.abs(rest) @ np.abs(np64(W)), np.abs(label) @ np.abs(np64(W)), True),
            (np64(dW), before + (rest + label).T @ np64(H), np.abs(rest).T @ np.abs(np64(H)), np.abs(label).T @ np.abs(np64(H)), dW_dtype == BF)):
        tol = e_rest * size_rest + e_label * size_label + 4 * U * np.abs(want)
        if bf16:
            tol = tol * 1.01 + 2.0 ** -8 * np.abs(want)
        assert np.all(np.abs(got - want) <= tol)
    again = np64(dW)
    if not accumulate:                                # in the order of the rows, whoever is first
        assert np.array_equal(np64(e.backward(Hd, W.to(DEV), y.to(DEV), valid.to(DEV), gl.to(DEV))[1]), again)


def test_gradient_buffers_of_the_user_are_checked():
    T, d, V = 9, 64, 500
    H, W, y, _ = make(T, d, V, BF, masked=0.0)
    H, W, y = H.to(DEV), W.to(DEV), y.to(DEV)
    e = TokenLogProb(T, d, V, dtype=BF, dW_dtype=BF)
    e.forward(H, W, y)
    g = torch.ones(T, device=DEV)
    for bad in (torch.zeros(V, d, device=DEV), torch.zeros(V - 1, d, dtype=BF, device=DEV), torch.zeros(V, d, dtype=BF),
                torch.zeros(d, V, dtype=BF, device=DEV).t()):
        e.dW = bad
        with pytest.raises((TypeError, ValueError), match="dW"):
            e.backward(H, W, y, grad_logp=g)
    e.dW, e.dH = None, torch.zeros(T + 1, d, dtype=BF, device=DEV)
    with pytest.raises(ValueError, match="dH"):
        e.backward(H, W, y, grad_logp=g)


@pytest.mark.parametrize("T", [1, 128, 129, 297, 1024, 1025])
def test_captured_forward_and_backward_follow_new_inputs(T):
    """Sizes on both sides of every rule on the number of rows: a replay gives what a plain call gives, bit for bit."""
    d, V = 64, 1500

    def inputs(seed):
        H, W, y, valid = make(T, d, V, BF, seed=seed)
        g = torch.Generator().manual_seed(seed)
        return [t.to(DEV) for t in (H, W, y, valid, torch.randn(T, generator=g), 0.1 * torch.randn(T, generator=g))]

    def both(e, H, W, y, valid, gl, ge):
        return tuple(e.forward(H, W, y, valid)) + tuple(e.backward(H, W, y, valid, gl, ge))

    e = TokenLogProb(T, d, V, top_k=6, dtype=BF, dW_dtype=BF)
    held = inputs(1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(e, *held)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = both(e, *held)
    torch.cuda.synchronize()
    new = inputs(2)
    for a, b in zip(held, new):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    want = both(TokenLogProb(T, d, V, top_k=6, dtype=BF, dW_dtype=BF), *new)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
