"""A wait that ran out on the device reaches whoever asks an 8-bit head, whose calls keep no workspace.  The wait is the library's self-test, which ends by itself."""
import pytest
import torch

from i8_util import head, tokens
from paper_2605_08632_b200 import binding as B
from paper_2605_08632_b200.api import Int8Head

DEV = "cuda"


def test_arguments_are_checked_on_the_host():
    assert B.lib().cat_device_status(None, 0, None) == -1


def test_a_head_reports_the_status_of_its_device(monkeypatch):
    asked, entered = [], []

    class Device:
        def __init__(self, device): self.device = device
        def __enter__(self): entered.append(self.device)
        def __exit__(self, *_): entered.append(None)

    h = Int8Head.__new__(Int8Head)
    torch.nn.Module.__init__(h)
    h.register_buffer("q", torch.zeros(3, 16, dtype=torch.int8))
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(B, "cat_device_status", lambda clear: asked.append((clear, entered[-1])) or -8)
    assert h.status() == -8 and h.status(clear=True) == -8
    assert asked == [(False, torch.device("cpu")), (True, torch.device("cpu"))] and entered[-1] is None


def run_out():
    B.cat_selftest_wait_timeout(0, 5_000_000, 2_000_000_000, torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(12, dtype=torch.int64, device=DEV))


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported_until_it_is_cleared():
    h = Int8Head.from_quantized(*(t.to(DEV) for t in head(3000, 64)))
    X = {T: tokens(T, 64, torch.bfloat16).to(DEV) for T in (5, 300)}
    y = torch.zeros(300, dtype=torch.int64, device=DEV)

    def calls():
        for T, x in X.items():
            nll, lse = h.loss_forward(x, y[:T])
            h.logits(x), h.loss_backward(x, y[:T], None, nll, nll, lse)

    h.status(clear=True)                    # other tests run out of waits too
    calls()
    assert h.status() == 0
    run_out()
    calls()                                 # which clear the status words of their own workspaces
    assert h.status() == -8 and h.status() == -8 and "wait" in B.cat_status_string(h.status())
    assert h.status(clear=True) == -8 and h.status() == 0
    calls()
    assert h.status() == 0


@pytest.mark.gpu
def test_other_streams_and_captures():
    h = Int8Head.from_quantized(*(t.to(DEV) for t in head(300, 64)))
    x = tokens(5, 64, torch.bfloat16).to(DEV)
    h.status(clear=True)
    want = h.logits(x)
    with torch.cuda.stream(torch.cuda.Stream()):
        run_out()
        assert h.status(clear=True) == -8 and h.status() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = h.logits(x)
        with pytest.raises(B.CatError):
            h.status()
    graph.replay()
    assert torch.equal(got, want) and h.status() == 0
