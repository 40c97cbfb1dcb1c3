"""LogProbModule's refusals that need no GPU."""
import types

import pytest
import torch

from paper_2605_08632_b200 import api


def test_backward_refuses_a_capture(monkeypatch):
    """A forward pass outside, its backward inside a capture: refused before anything is launched or allocated."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    ctx = types.SimpleNamespace(saved_tensors=(None,) * 6, engine=None)
    backward = getattr(api._LogProbFn.backward, "__wrapped__", api._LogProbFn.backward)
    with pytest.raises(RuntimeError, match="captured"):
        backward(ctx, None, None, None, None)
