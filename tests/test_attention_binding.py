"""What the Python binding of attention and of caches held in 4 bits refuses before the library is asked (no GPU is touched)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding


def cache(pages=3, heads=2, page_size=16, dim=64):
    return oz.KV4Cache.empty(pages, heads, page_size, dim, device="cpu")


def test_a_cache_knows_its_tensors():
    c = cache()
    assert (c.pages, c.heads, c.page_size, c.dim) == (3, 2, 16, 64)
    assert (c.struct.codes_page, c.struct.codes_head, c.struct.scales_page, c.struct.scales_head) == (1024, 512, 32, 16)
    # every second layer of one tensor
    codes, scales = torch.zeros((3, 4, 2, 16, 32), dtype=torch.uint8), torch.zeros((3, 4, 2, 16, 2), dtype=torch.float16)
    c = oz.KV4Cache(codes[:, 0], scales[:, 0], codes[:, 1], scales[:, 1])
    assert (c.struct.codes_page, c.struct.codes_head, c.struct.scales_page, c.struct.scales_head) == (4096, 512, 128, 16)


def test_caches_are_refused():
    codes, scales = torch.zeros((3, 2, 16, 32), dtype=torch.uint8), torch.zeros((3, 2, 16, 2), dtype=torch.float16)
    for bad in ((codes[0], scales, codes, scales), (codes.int(), scales, codes, scales), (codes, scales.float(), codes, scales), (codes, scales, codes[:2], scales),
                (codes, scales[..., :1], codes, scales), (codes, scales, codes[..., :16], scales), (codes[..., ::2], scales, codes[..., ::2], scales),
                (codes, scales, torch.zeros((2, 3, 16, 32), dtype=torch.uint8).transpose(0, 1), scales), (codes[:, :, :8], scales, codes, scales)):
        with pytest.raises(oz.Oz2Error):
            oz.KV4Cache(*bad)


def test_tensors_off_the_gpu_are_refused():
    q, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32)
    c, places = cache(), torch.zeros((1, 2, 32))
    calls = [lambda: oz.attention(q, k, k, cu), lambda: oz.kv4_append(c, k, k, cu, table, lengths), lambda: oz.kv4_attention(c, q, cu, table, lengths),
             lambda: oz.kv4_evict(c, table, lengths, places.int(), places, 2)]
    for call in calls:
        with pytest.raises(oz.Oz2Error, match="GPU"):
            call()


def test_tensors_that_require_a_gradient_are_refused():
    q, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32)
    c, places = cache(), torch.zeros((1, 2, 32))
    calls = [(q, lambda: oz.attention(q, k, k, cu)), (k, lambda: oz.attention(q, k, k, cu)), (k, lambda: oz.kv4_append(c, k, k, cu, table, lengths)),
             (q, lambda: oz.kv4_attention(c, q, cu, table, lengths)), (places, lambda: oz.kv4_attention(c, q, cu, table, lengths, weights=places)),
             (places, lambda: oz.kv4_evict(c, table, lengths, places.detach().int(), places, 2))]
    for v, call in calls:
        v.requires_grad_(True)
        with pytest.raises(oz.Oz2Error, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(oz.Oz2Error, match="GPU"):
            call()
        v.requires_grad_(False)


@pytest.fixture
def on_gpu(monkeypatch):
    """tensors of the host pass for those of GPU 0, so that the checks behind that one are reached; the library is not"""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)

    class Library:
        def __getattr__(self, name):
            return lambda *a: 0

    monkeypatch.setattr(binding, "lib", lambda: Library())


def test_shapes_and_types_are_refused(on_gpu):
    q, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32)
    assert oz.attention(q, k, k, cu).shape == q.shape
    for bad in ((q[0], k, k, cu), (q, k[:3], k, cu), (q, k, k[..., :32], cu), (q, k, k[:, :1], cu), (q.double(), k, k, cu), (q, k, k, cu.long()), (q, k, k, cu[:0]),
                (q, k, k, cu[None]), (q.transpose(1, 2).contiguous().transpose(1, 2), k, k, cu)):
        with pytest.raises(oz.Oz2Error):
            oz.attention(*bad)
    with pytest.raises(oz.Oz2Error):
        oz.attention(q, k, k, cu, out=q[:, :2])
    c = cache()
    c.index = 0
    places, positions = torch.zeros((1, 2, 32)), torch.zeros((1, 2, 32), dtype=torch.int32)
    at = torch.zeros(4, dtype=torch.int32)
    oz.kv4_append(c, k, k, cu, table, lengths, at=at, positions=positions, weights=places)
    for bad in (dict(at=at), dict(positions=positions), dict(at=at.long(), positions=positions), dict(at=at[:3], positions=positions), dict(weights=places[..., :31]),
                dict(weights=places.double()), dict(weights=places[:, :1]), dict(held=(k, q)), dict(at=at, positions=places)):
        with pytest.raises(oz.Oz2Error):
            oz.kv4_append(c, k, k, cu, table, lengths, **bad)
    for bad in ((c, q[..., :32], cu, table, lengths), (c, q, cu[:1], table, lengths), (c, q, cu, table[0], lengths), (c, q, cu, table, lengths.long()),
                (c, q, cu, table.long(), lengths), (c, q, cu, table, torch.cat((lengths, lengths)))):
        with pytest.raises(oz.Oz2Error):
            oz.kv4_attention(*bad)
    for bad in ((None, places), (positions, None), (positions.long(), places), (positions, places.half())):
        with pytest.raises(oz.Oz2Error):
            oz.kv4_evict(c, table, lengths, *bad, 2)
    with pytest.raises(oz.Oz2Error):
        oz.kv4_evict(c, table, lengths, positions, places, 2, out=(lengths, positions, places[..., :10]))


def test_tensors_on_another_device_than_the_cache_are_refused(on_gpu, monkeypatch):
    q, cu = torch.zeros((4, 4, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths, c = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32), cache()
    c.index = 1
    with pytest.raises(oz.Oz2Error, match="one GPU"):
        oz.kv4_attention(c, q, cu, table, lengths)
    c.index = 0
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    for call in (lambda: oz.kv4_attention(c, q, cu, table, lengths), lambda: oz.attention(q, q, q, cu)):
        with pytest.raises(oz.Oz2Error, match="cuda:0.*cuda:1"):
            call()
