"""Results that would be written over what a product with weights in 4 bits still reads are refused before anything is launched.  The addresses here belong to
nobody; every call returns ahead of its launch."""
import ctypes

import pytest

pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_w4_arguments import _layer, _matrix

AT = 1 << 20


def _matvec(t, x, ldx, y, ldy, beta=0.0, c=None, ldc=0, x_type=0, y_type=0):
    w = _matrix(n=64, k=100)
    return oz.lib().oz2_w4_matvec(ctypes.addressof(w), t, 1.0, x_type, x, ldx, beta, c, ldc, y_type, y, ldy, None)


@pytest.mark.parametrize("t,ldx,ldy,away", [(1, 0, 0, 0), (1, 100, 64, 99 * 4), (1, 100, 64, -63 * 4), (3, 100, 64, 0), (3, 100, 100, 299 * 4), (3, 100, 64, -191 * 4),
                                            (4, 200, 200, 99 * 4), (4, 200, 200, 199 * 4 + 1), (4, 200, 300, 100 * 4), (1000, 164, 164, 101 * 4),
                                            (1000, 165, 164, 100 * 4), (65535, 1000, 999, 100 * 4)])
def test_matvec_over_its_vectors(t, ldx, ldy, away):
    assert _matvec(t, AT, ldx, AT + away, ldy) == -11


@pytest.mark.parametrize("t,ldc,ldy,away", [(2, 64, 65, 0), (2, 65, 64, 0), (1, 64, 64, 4), (2, 64, 64, 64 * 4), (5, 100, 100, -63 * 4), (5, 100, 100, 360 * 4)])
def test_matvec_over_a_residual_that_is_not_its_result(t, ldc, ldy, away):
    assert _matvec(t, 1 << 40, 100, AT + away, ldy, beta=1.0, c=AT, ldc=ldc) == -8


def test_sizes_of_types_count():
    assert _matvec(2, AT, 100, AT + 399, 64, x_type=1) == -11     # 200 elements of 2 bytes
    assert _matvec(2, AT + 127 + 128, 100, AT, 64, y_type=2) == -11


@pytest.mark.parametrize("t,ldx,ldy,away,y_type", [(1, 100, 100, 4, 0), (3, 100, 101, 0, 0), (3, 200, 200, 99 * 4, 0), (2, 100, 100, 0, 1), (40, 150, 150, -149 * 4, 0)])
def test_moe_over_its_tokens(t, ldx, ldy, away, y_type):
    layer = _layer()
    assert oz.lib().oz2_w4_moe(ctypes.addressof(layer), t, 0, AT, ldx, None, y_type, AT + away, ldy, None, None, None) == -8


def test_moe_takes_a_result_in_the_place_of_its_tokens_and_between_them():
    """no workspace: that is what is missing when all else is well"""
    layer = _layer()
    at = ctypes.addressof(layer)
    ctx = oz.Context()
    for t, ldx, ldy, away in ((1, 100, 100, 0), (1, 100, 999, 0), (40, 150, 150, 0), (3, 250, 250, 100 * 4), (3, 250, 250, -150 * 4), (3, 100, 100, 300 * 4),
                              (3, 100, 100, -300 * 4), (1, 100, 100, 400), (1, 100, 100, -400)):
        assert oz.lib().oz2_context_w4_moe(ctx.handle, at, t, 0, AT, ldx, None, 0, AT + away, ldy, None, None, None) == 1
    ctx.close()
