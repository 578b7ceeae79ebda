"""What the Python binding of the products with weights in 4 bits tells the library about the tensors it is given, and what it refuses (no GPU is touched)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding


def stack(count, n, k, group=32):
    return oz.W4Matrix(torch.zeros((count, n, k // 2), dtype=torch.uint8), torch.ones((count, n, -(-k // group))), group=group)


def test_rows_that_overlap_are_refused():
    row = torch.arange(8.0)
    for bad in (row.expand(4, 8), row.view(1, 8).expand(4, 8), torch.zeros(16).as_strided((3, 8), (4, 1)), torch.zeros(30).as_strided((2, 8), (7, 1))):
        with pytest.raises(oz.Oz2Error):
            binding._rows("x", bad, 8)
    assert binding._rows("x", torch.zeros(16).as_strided((2, 8), (8, 1)), 8) == 8
    assert binding._rows("x", torch.zeros((5, 11))[:, 2:10], 8) == 11
    # one row has no next one: its stride says nothing
    assert binding._rows("x", row.expand(1, 8), 8) == 8
    assert binding._rows("x", torch.zeros((9, 8))[4:5], 8) == 8
    assert binding._rows("x", torch.zeros((0, 8)), 8) == 8
    assert binding._rows("x", torch.zeros((3, 0)), 0) >= 0


def test_a_router_whose_rows_overlap_is_refused():
    gate, up, down = stack(4, 60, 100), stack(4, 60, 100), stack(4, 100, 60)
    assert oz.MoeLayer(torch.zeros((4, 104))[:, :100], gate, up, down, 2).struct.ld_router == 104
    with pytest.raises(oz.Oz2Error):
        oz.MoeLayer(torch.zeros(100).expand(4, 100), gate, up, down, 2)
    one = stack(1, 60, 100)
    assert oz.MoeLayer(torch.zeros(100).expand(1, 100), one, one, stack(1, 100, 60), 1).struct.ld_router == 100


def test_expanded_weights_are_refused():
    """codes, scales or zero points that rows share have a pitch of 0, which the library names as a bad matrix"""
    import ctypes
    codes, scales = torch.zeros((8, 50), dtype=torch.uint8), torch.ones((8, 4))
    for w in (oz.W4Matrix(codes[:1].expand(8, 50), scales, group=32), oz.W4Matrix(codes, scales[:1].expand(8, 4), group=32),
              oz.W4Matrix(codes, scales, torch.zeros((1, 4), dtype=torch.uint8).expand(8, 4), group=32)):
        assert oz.lib().oz2_w4_matvec(ctypes.addressof(w.struct), 1, 1.0, 0, 4096, 100, 0.0, None, 0, 0, 4096, 8, None) == -1


def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: 1, raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 4096 + index)
    assert binding._stream_on(None, 1) == 4097 and binding._stream_on(77, 1) == 77
    for stream in (None, 77):
        with pytest.raises(oz.Oz2Error, match="cuda:0.*cuda:1"):
            binding._stream_on(stream, 0)


def test_tensors_that_require_a_gradient_are_refused():
    """in grad mode, where a graph would be recorded; otherwise the call goes on to its next check, which here is that of the device"""
    w, x, c = stack(1, 60, 100), torch.zeros((2, 100)), torch.zeros((2, 60))
    layer = oz.MoeLayer(torch.zeros((4, 100)), stack(4, 60, 100), stack(4, 60, 100), stack(4, 100, 60), 2, bias=torch.zeros(4))
    calls = [(x, lambda: oz.w4_matvec(w, x)), (c, lambda: oz.w4_matvec(w, x, beta=1.0, c=c)), (c, lambda: oz.w4_matvec(w, x, out=c)),
             (w.scales, lambda: oz.w4_matvec(w, x))]
    calls += [(v, lambda: oz.w4_moe(layer, x)) for v in (x, layer.router, layer.bias, layer.gate.scales, layer.up.scales, layer.down.scales)]
    for v, call in calls:
        with pytest.raises(oz.Oz2Error, match="on the GPU"):
            call()
        v.requires_grad_(True)
        with pytest.raises(oz.Oz2Error, match="gradient"):
            call()
        for mode in (torch.no_grad, torch.inference_mode):
            with mode(), pytest.raises(oz.Oz2Error, match="on the GPU"):
                call()
        v.requires_grad_(False)
