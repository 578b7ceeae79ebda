"""Heads without a value are refused like every other wrong shape, with the library's own error (no GPU is touched)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding


@pytest.fixture(autouse=True)
def on_gpu(monkeypatch):
    """tensors of the host pass for those of GPU 0; the library refuses before it would read any"""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)


def test_heads_without_values():
    q, k, cu = torch.zeros((4, 4, 0)), torch.zeros((4, 2, 0)), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(oz.Oz2Error, match="oz2_attention"):
        oz.attention(q, k, k, cu)
    with pytest.raises(oz.Oz2Error, match="oz2_attention"):
        oz.attention(q, k, k, cu, scale=1.0)
    with pytest.raises(oz.Oz2Error):  # a cache cannot have such heads
        oz.KV4Cache.empty(3, 2, 16, 0, device="cpu")
