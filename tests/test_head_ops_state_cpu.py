"""Sizes and rules behind what the LM-head operators' engines keep, without a GPU."""
import types

import pytest
import torch

from paper_2605_08632_b200 import binding as B


@pytest.mark.parametrize("T,d,V,K,code,slab", [(96, 64, 700, 8, B.CAT_BF16, 0), (16384, 2048, 128256, 8, B.CAT_BF16, 0), (1040, 64, 3000, 8, B.CAT_F32, 2),
                                               (6000, 1024, 151936, 16, B.CAT_BF16, 256), (3, 64, 2, 3, B.CAT_BF16, 0)])
def test_the_longest_lists_workspace_serves_every_length(T, d, V, K, code, slab):
    """An engine sizes its workspace once, for lists of CAT_TOPK_MAX; it costs little beside the slab."""
    s = B.make_shape(T, d, V, K, code, slab_mib=slab)
    most = B.cat_topk_kd_workspace_bytes(s, B.make_topk_kd_desc(1, B.CAT_TOPK_MAX, 0.0))
    for k in (1, 2, 8, 63, 64, 255, B.CAT_TOPK_MAX):
        for L in (1, T, 5 * T):
            assert B.cat_topk_kd_workspace_bytes(s, B.make_topk_kd_desc(L, k, 0.1)) <= most
    least = B.cat_topk_kd_workspace_bytes(s, B.make_topk_kd_desc(T, 1, 0.1))
    assert most - least <= (T + 255) // 256 * 256 * 4 * B.CAT_TOPK_MAX + 256       # a slab is whole tiles of 256 rows


def test_stream_handle_without_the_undocumented_way(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: types.SimpleNamespace(cuda_stream=1000 + dev))
    monkeypatch.setattr(B, "_raw_stream", None)
    assert B._stream() == 1003
    monkeypatch.setattr(B, "_raw_stream", lambda dev: 2000 + dev)
    assert B._stream() == 2003
