"""Refusals of the products with weights held in 4 bits: every bad argument is named by its position before anything is launched."""
import copy
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding

INVALID = 1 << 12   # an address that nothing may be read from: these calls return before they would


def _matrix(n=64, k=100, group=32, count=1, **more):
    groups = -(-k // group) if group > 0 else 1
    fields = dict(n=n, k=k, group=group, codes=INVALID, ld_codes=(k + 1) // 2, scales=INVALID, ld_scales=groups, zeros=None, ld_zeros=0, count=count,
                  stride_codes=n * ((k + 1) // 2), stride_scales=n * groups, stride_zeros=0, scale_type=oz.OZ2_F32)
    fields.update(more)
    return binding._W4(**fields)


def _matvec(w, t=2, alpha=1.0, x_type=0, x=INVALID, ldx=100, beta=0.0, c=None, ldc=0, y_type=0, y=INVALID, ldy=64):
    return oz.lib().oz2_w4_matvec(None if w is None else ctypes.addressof(w), t, alpha, x_type, x, ldx, beta, c, ldc, y_type, y, ldy, None)


@pytest.mark.parametrize("fields", [dict(n=-1), dict(k=-1), dict(n=1 << 31), dict(k=1 << 31), dict(group=0), dict(group=-32), dict(group=16),
                                    dict(group=96), dict(group=160), dict(scale_type=3), dict(scale_type=-1), dict(codes=None), dict(scales=None),
                                    dict(ld_codes=49), dict(ld_scales=3), dict(zeros=INVALID, ld_zeros=3)])
def test_matvec_refuses_a_matrix_it_cannot_read(fields):
    assert _matvec(_matrix(**fields)) == -1


def test_matvec_names_the_bad_argument():
    w = _matrix()
    assert _matvec(None) == -1
    assert _matvec(w, t=-1) == -2 and _matvec(w, t=65536) == -2
    assert _matvec(w, x_type=3) == -4 and _matvec(w, x_type=-1) == -4
    assert _matvec(w, x=None) == -5
    assert _matvec(w, ldx=99) == -6
    assert _matvec(w, beta=1.0, c=None, ldc=64) == -8
    assert _matvec(w, beta=1.0, c=INVALID, ldc=63) == -9
    assert _matvec(w, y_type=7) == -10
    assert _matvec(w, y=None) == -11
    assert _matvec(w, ldy=63) == -12


def test_matvec_with_nothing_to_write_is_done():
    assert _matvec(_matrix(n=0, codes=None, scales=None), y=None, x=None) == 0
    assert _matvec(_matrix(), t=0, y=None, x=None) == 0


def _layer(**more):
    d, f, count = 100, 60, 4
    fields = dict(gate=_matrix(f, d, count=count), up=_matrix(f, d, count=count), down=_matrix(d, f, count=count), router=INVALID, ld_router=d, bias=None,
                  router_type=0, top_k=2, score=0, renormalize=1, activation=0, factor=1.0)
    fields.update(more)
    return binding._Moe(**fields)


def _moe(layer, t=2, x_type=0, x=INVALID, ldx=100, y_type=0, y=INVALID, ldy=100):
    return oz.lib().oz2_w4_moe(None if layer is None else ctypes.addressof(layer), t, x_type, x, ldx, None, y_type, y, ldy, None, None, None)


@pytest.mark.parametrize("fields", [dict(router=None), dict(ld_router=99), dict(router_type=3), dict(top_k=0), dict(top_k=5), dict(score=2), dict(activation=2),
                                    dict(up=_matrix(61, 100, count=4)), dict(up=_matrix(60, 99, count=4)), dict(up=_matrix(60, 100, count=3)),
                                    dict(down=_matrix(100, 61, count=4)), dict(down=_matrix(99, 60, count=4)), dict(down=_matrix(100, 60, count=5)),
                                    dict(gate=_matrix(60, 100, count=4, group=48)), dict(gate=_matrix(60, 100, count=0)),
                                    dict(gate=_matrix(60, 100, count=4, stride_codes=59 * 50)),
                                    dict(up=_matrix(60, 100, count=4, stride_scales=239)), dict(down=_matrix(100, 60, count=4, codes=None))])
def test_moe_refuses_a_layer_it_cannot_read(fields):
    layer = _layer(**fields)
    assert _moe(layer) == -1
    assert oz.lib().oz2_w4_moe_workspace_bytes(ctypes.addressof(layer), 2) == 0


def test_moe_refuses_too_many_experts():
    stack = dict(count=1025)
    layer = _layer(gate=_matrix(60, 100, **stack), up=_matrix(60, 100, **stack), down=_matrix(100, 60, **stack))
    assert _moe(layer) == -1
    stack = dict(count=64)
    layer = _layer(gate=_matrix(60, 100, **stack), up=_matrix(60, 100, **stack), down=_matrix(100, 60, **stack), top_k=33)
    assert _moe(layer) == -1


def test_moe_names_the_bad_argument():
    layer = _layer()
    assert _moe(None) == -1
    assert _moe(layer, t=-1) == -2 and _moe(layer, t=4097) == -2
    assert _moe(layer, x_type=3) == -3
    assert _moe(layer, x=None) == -4
    assert _moe(layer, ldx=99) == -5
    assert _moe(layer, y_type=3) == -7
    assert _moe(layer, y=None) == -8
    assert _moe(layer, ldy=99) == -9
    assert _moe(layer, t=0, x=None, y=None) == 0


def test_moe_without_a_workspace_says_so_and_a_context_counts_itself():
    layer = _layer()
    at = ctypes.addressof(layer)
    need = oz.lib().oz2_w4_moe_workspace_bytes(at, 2)
    assert need > 0 and oz.lib().oz2_w4_moe_workspace_bytes(at, 4097) == 0
    ctx = oz.Context()
    args = (at, 2, 0, INVALID, 100, None, 0, INVALID, 100, None, None, None)
    assert oz.lib().oz2_context_w4_moe(ctx.handle, *args) == 1
    assert oz.lib().oz2_context_set_workspace(ctx.handle, 256 * 16, need - 1) == 0
    assert oz.lib().oz2_context_w4_moe(ctx.handle, *args) == 1
    assert oz.lib().oz2_context_w4_moe(ctx.handle, None, *args[1:]) == -2
    assert oz.lib().oz2_context_w4_moe(ctx.handle, at, 2, 3, *args[3:]) == -4
    ctx.close()


def test_python_objects_refuse_what_does_not_fit():
    codes, scales = torch.zeros((8, 50), dtype=torch.uint8), torch.ones((8, 4))
    w = oz.W4Matrix(codes, scales, k=100, group=32)
    assert (w.n, w.k, w.count, w.struct.ld_codes, w.struct.ld_scales) == (8, 100, 1, 50, 4)
    for bad in [lambda: oz.W4Matrix(codes.int(), scales, group=32), lambda: oz.W4Matrix(codes, scales, k=101, group=32),
                lambda: oz.W4Matrix(codes, scales[:, :3], k=100, group=32), lambda: oz.W4Matrix(codes, scales.double(), k=100, group=32),
                lambda: oz.W4Matrix(codes, scales[:7], k=100, group=32), lambda: oz.W4Matrix(codes, scales, zeros=scales, k=100, group=32),
                lambda: oz.W4Matrix(codes.t().contiguous().t(), scales, k=100, group=32), lambda: oz.W4Matrix(codes[0], scales[0], k=100, group=32),
                lambda: oz.w4_matvec(w, torch.zeros((2, 99))), lambda: oz.w4_matvec(w, torch.zeros((100, 2)).t()),
                lambda: oz.w4_matvec(w, torch.zeros((2, 100)), out=torch.zeros((2, 9))), lambda: oz.w4_matvec(w, torch.zeros((2, 100)), out=torch.zeros((1, 8))),
                lambda: oz.w4_matvec(w, torch.zeros((2, 100), dtype=torch.float64)),
                lambda: oz.w4_matvec(w, torch.zeros((2, 100)), beta=1.0, c=torch.zeros((2, 8), dtype=torch.bfloat16))]:
        with pytest.raises(oz.Oz2Error):
            bad()

    def stack(n, k):
        return oz.W4Matrix(torch.zeros((4, n, k // 2), dtype=torch.uint8), torch.ones((4, n, -(-k // 32))), group=32)

    gate, up, down, router = stack(60, 100), stack(60, 100), stack(100, 60), torch.zeros((4, 100))
    layer = oz.MoeLayer(router, gate, up, down, 2)
    assert oz.w4_moe_workspace_bytes(layer, 3) > 0 and oz.w4_moe_workspace_bytes(oz.MoeLayer(router, gate, up, down, 5), 3) == 0
    for bad in [lambda: oz.MoeLayer(router[:3], gate, up, down, 2), lambda: oz.MoeLayer(router, gate, down, up, 2),
                lambda: oz.MoeLayer(router, gate, up, down, 2, bias=torch.zeros(3)), lambda: oz.w4_moe(layer, torch.zeros((2, 99))),
                lambda: oz.w4_matvec(gate, torch.zeros((2, 100))), lambda: oz.w4_moe(layer, torch.zeros((2, 100)), active=torch.zeros(3, dtype=torch.bool)),
                lambda: oz.w4_moe(layer, torch.zeros((2, 100)), ids=torch.zeros((2, 2), dtype=torch.int64))]:
        with pytest.raises(oz.Oz2Error):
            bad()
    with pytest.raises(ValueError):
        oz.MoeLayer(router, gate, up, down, 2, activation="relu")
