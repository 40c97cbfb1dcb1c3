"""LogProbModule: calls that share nothing with one another, whatever their lengths, streams and threads; layouts; bfloat16."""
import threading

import numpy as np
import pytest
import torch

from oracle import head_ops_oracle as O
from paper_2605_08632_b200.api import LogProbModule, TokenLogProb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().cpu().double().numpy()


def inputs(T, d, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    H, W = torch.randn(T, d, generator=g).to(dtype), (0.05 * torch.randn(V, d, generator=g)).to(dtype)
    return H.to(DEV), W.to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV), (torch.rand(T, generator=g) < 0.8).to(DEV)


def step(head, H, y, valid, gl, ge):
    h = H.detach().requires_grad_()
    head.weight.grad = None
    logp, entropy, ids, tl = head(h, y, valid)
    (logp * gl + entropy * ge).sum().backward()
    return [logp.detach(), entropy.detach(), ids, tl, h.grad, head.weight.grad]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_lengths_leave_nothing_behind(dtype):
    """Batches of ever new lengths: what a call needed goes back to the allocator."""
    d, V = 64, 3000
    _, W, _, _ = inputs(1, d, V, dtype, 0)
    head = LogProbModule(W, top_k=8)
    held = []
    for T in range(200, 240):
        H, _, y, valid = inputs(T, d, V, dtype, T)
        g = torch.ones(T, device=DEV)
        step(head, H, y, valid, g, g)
        head.weight.grad = None
        del H, y, valid, g
        torch.cuda.synchronize()
        held.append(torch.cuda.memory_allocated())
    assert max(held[1:]) - held[0] <= 1 << 20, held
    head.top_k = 3                              # looked at by every call
    H, _, y, valid = inputs(200, d, V, dtype, 200)
    assert head(H, y, valid)[2].shape == (200, 3)


def test_two_threads_on_streams_of_their_own():
    """Two threads, one module, the same length: each gets its own results, over and over."""
    T, d, V, n = 64, 128, 8000, 30
    cases = [inputs(T, d, V, BF, s) for s in (1, 2)]
    head = LogProbModule(cases[0][1], top_k=6)
    head.weight.requires_grad_(False)
    g = torch.randn(T, generator=torch.Generator().manual_seed(4)).to(DEV)

    def one(H, y, valid):
        h = H.detach().requires_grad_()
        logp, entropy, ids, tl = head(h, y, valid)
        (logp * g + entropy * g).sum().backward()
        return [logp.detach(), entropy.detach(), ids, tl, h.grad]

    want = [one(c[0], c[2], c[3]) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        H, _, y, valid = cases[i]
        with torch.cuda.stream(stream):
            got = [one(H, y, valid) for _ in range(n)]
        stream.synchronize()
        wrong.extend(i for r in got if not all(torch.equal(a, b) for a, b in zip(r, want[i])))

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_several_calls_before_one_backward():
    """The same module three times in one graph, as a loss over three batches of one length has it; saved results may be written to."""
    T, d, V = 40, 64, 700
    H, W, y, valid = inputs(T, d, V, F32, 5)
    head = LogProbModule(W.clone())
    hs = [(H * s).detach().requires_grad_() for s in (1.0, 0.5, -1.0)]
    total = 0.0
    for h in hs:
        logp, entropy, _, _ = head(h, y, valid)
        total = total + logp.sum() + 0.1 * entropy.sum()
        logp.detach().zero_(), entropy.detach().zero_()         # the results are the caller's
    total.backward()
    dW = 0.0
    for h in hs:
        a, b, *_ = O.logprob_backward(h.detach().cpu(), W.cpu(), y.cpu(), valid.cpu(), np.ones(T), 0.1 * np.ones(T))
        assert np.linalg.norm(np64(h.grad) - a) <= 1e-5 * np.linalg.norm(a)
        dW = dW + b
    assert np.linalg.norm(np64(head.weight.grad) - dW) <= 1e-5 * np.linalg.norm(dW)


def test_bfloat16_against_the_oracle():
    """Results rounded to bf16 once (2^-8 at most, 2^-9 on average), dz in two terms below 129 rows."""
    T, d, V = 100, 64, 900
    H, W, y, valid = inputs(T, d, V, BF, 6)
    g = torch.Generator().manual_seed(7)
    gl, ge = torch.randn(T, generator=g), 0.3 * torch.randn(T, generator=g)
    got = step(LogProbModule(W.clone(), top_k=4), H, y, valid, gl.to(DEV), ge.to(DEV))
    f = O.logprob_forward(H.cpu(), W.cpu(), y.cpu(), valid.cpu(), 4)
    a, b, *_ = O.logprob_backward(H.cpu(), W.cpu(), y.cpu(), valid.cpu(), gl, ge)
    assert np.abs(np64(got[0]) - f["logp"]).max() <= 1e-5 and np.array_equal(got[2].cpu().numpy(), f["top_ids"])
    assert got[4].dtype == BF and got[5].dtype == BF
    assert np.linalg.norm(np64(got[4]) - a) <= 2 ** -8 * np.linalg.norm(a)
    assert np.linalg.norm(np64(got[5]) - b) <= 2 ** -8 * np.linalg.norm(b)


def test_captured_without_gradients_beside_eager_calls():
    """A captured scoring call owns what it uses: eager calls of the same and of other lengths leave its replays alone."""
    T, d, V = 70, 64, 2000
    H, W, y, valid = inputs(T, d, V, BF, 8)
    head = LogProbModule(W, top_k=5)
    with torch.no_grad():
        head(H, y, valid)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = head(H, y, valid)
        new = inputs(T, d, V, BF, 9)
        H.copy_(new[0])
        for n in (T, 300, T):
            head(*(inputs(n, d, V, BF, 10)[i] for i in (0, 2, 3)))
        graph.replay()
        torch.cuda.synchronize()
        e = TokenLogProb(T, d, V, 5)
        r = e.forward(new[0], W, y, valid)
        assert torch.equal(out[0], r.logp) and torch.equal(out[1], r.entropy) and torch.equal(out[2], r.top_ids) and torch.equal(out[3], r.top_logp)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_pitched_hidden_states_get_their_gradient(dtype):
    T, d, V = 50, 64, 900
    H, W, y, valid = inputs(T, d, V, dtype, 1)
    g = torch.randn(T, generator=torch.Generator().manual_seed(3)).to(DEV)
    want = step(LogProbModule(W.clone()), H, y, valid, g, g)
    wide = torch.zeros(T, d + 16, dtype=dtype, device=DEV)
    wide[:, :d] = H
    wide.requires_grad_()
    head = LogProbModule(W.clone())
    logp, entropy, _, _ = head(wide[:, :d], y, valid)
    (logp * g + entropy * g).sum().backward()
    assert torch.equal(wide.grad[:, :d], want[4]) and not wide.grad[:, d:].any()
    assert torch.equal(head.weight.grad, want[5])
    pitched = torch.zeros(V, d + 16, dtype=dtype, device=DEV)[:, :d]
    with pytest.raises(ValueError, match="weight"):        # at once, not after the forward pass
        LogProbModule(torch.nn.Parameter(pitched))(H, y, valid)
