"""Tensors without elements have whatever strides they come with (NumPy's have zeros), and are accepted: there is nothing to do (no GPU is touched)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding
from test_attention_arguments import F16, P, _Kept, attention, cache, calls, ref, rows, sequences


@pytest.fixture
def on_gpu(monkeypatch):
    """tensors of the host pass for those of GPU 0; the library has nothing to launch"""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)


def empty(*shape, dtype=np.float32):
    t = torch.from_numpy(np.zeros(shape, dtype=dtype))
    assert t.numel() == 0 and not any(t.stride())
    return t


def test_rows_of_no_tokens_in_the_library():
    flat = rows(P, 0, 0)
    assert attention(tokens=0, q=flat, k=flat, v=flat, out=flat) == 0
    L, c, on = oz.lib(), cache(), sequences(tokens=0)
    assert L.oz2_kv4_append(ref(c), ref(on), None, ref(flat), ref(flat), ref(flat), ref(flat), None) == 0
    assert L.oz2_kv4_attention(ref(c), ref(on), 8, 0.1, ref(flat), ref(flat), None) == 0
    # their types are looked at all the same
    assert attention(tokens=0, q=rows(P, 0, 0, 3)) == -9 and attention(tokens=0, k=rows(P, 0, 0, F16)) == -10
    none = dict(sequences=0, table=None, lengths=None, positions=None, weights=None)
    kept = _Kept(None, None, 0, 0, None, 0, 0)
    assert L.oz2_kv4_evict(ref(c), ref(sequences(**none)), 4, 0, ref(kept), None) == 0


def test_attention_of_no_tokens(on_gpu):
    q, k, cu = empty(0, 4, 64), empty(0, 2, 64), torch.zeros(3, dtype=torch.int32)
    assert oz.attention(q, k, k, cu).shape == (0, 4, 64)
    out = empty(0, 4, 64)
    assert oz.attention(q, k, k, cu, out=out) is out


def test_caches_without_new_tokens_or_sequences(on_gpu):
    c = oz.KV4Cache.empty(3, 2, 16, 64, device="cpu")
    c.index = 0
    q, k, table, lengths, cu = empty(0, 4, 64), empty(0, 2, 64), torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    places, positions = torch.zeros((1, 2, 32)), torch.zeros((1, 2, 32), dtype=torch.int32)
    oz.kv4_append(c, k, k, cu, table, lengths, at=empty(0, dtype=np.int32), positions=positions, weights=places, held=(empty(0, 2, 64), empty(0, 2, 64)))
    assert oz.kv4_attention(c, q, cu, table, lengths).shape == q.shape
    # no sequences at all
    table, lengths, cu = empty(0, 2, dtype=np.int32), empty(0, dtype=np.int32), torch.zeros(1, dtype=torch.int32)
    places, positions = empty(0, 2, 32), empty(0, 2, 32, dtype=np.int32)
    oz.kv4_append(c, k, k, cu, table, lengths, at=empty(0, dtype=np.int32), positions=positions, weights=places)
    assert oz.kv4_attention(c, q, cu, table, lengths, weights=places).shape == q.shape
    for out in (None, (empty(0, dtype=np.int32), empty(0, 2, 32, dtype=np.int32), empty(0, 2, 32))):
        assert oz.kv4_evict(c, table, lengths, positions, places, 2, out=out)[0].shape == (0,)


def test_products_of_no_vectors(on_gpu):
    W = oz.W4Matrix(torch.zeros((8, 32), dtype=torch.uint8), torch.ones((8, 1)), group=64)
    assert oz.w4_matvec(W, empty(0, 64)).shape == (0, 8)
