"""Calls of the products with weights in 4 bits that are refused through the public entry points, on tensors on the GPU; nothing is launched for them."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz


def matrix(n, k, count=0):
    lead = (count,) if count else ()
    codes = torch.randint(0, 256, (*lead, n, k // 2), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    return oz.W4Matrix(codes, torch.full((*lead, n, k // 32), 0.01, device="cuda"), group=32)


def layer():
    return oz.MoeLayer(torch.randn((5, 256), device="cuda"), matrix(128, 256, 5), matrix(128, 256, 5), matrix(256, 128, 5), 3)


def test_expanded_tensors():
    w, x, c = matrix(96, 256), torch.randn((4, 256), device="cuda"), torch.randn((4, 96), device="cuda")
    for bad in (lambda: oz.w4_matvec(w, x[:1].expand(4, 256)), lambda: oz.w4_matvec(w, x, beta=1.0, c=c[0].expand(4, 96)),
                lambda: oz.w4_matvec(w, x, out=c[:1].expand(4, 96)), lambda: oz.w4_matvec(w, torch.randn(300, device="cuda").as_strided((4, 256), (8, 1)))):
        with pytest.raises(oz.Oz2Error, match="overlap"):
            bad()
    moe, ctx = layer(), oz.Context()
    ctx.allocate_moe_workspace(moe, 4)
    for bad in (lambda: ctx.w4_moe(moe, x[:1].expand(4, 256)), lambda: ctx.w4_moe(moe, x, out=torch.empty((1, 256), device="cuda").expand(4, 256))):
        with pytest.raises(oz.Oz2Error, match="overlap"):
            bad()
    # one row is a row, however it came about
    assert torch.equal(oz.w4_matvec(w, x[0].expand(1, 256), beta=1.0, c=c[0].expand(1, 96)), oz.w4_matvec(w, x[:1], beta=1.0, c=c[:1]))


def test_results_over_what_is_read():
    """refused where they would be; in the place of a residual and of a layer's tokens they are what they are elsewhere"""
    w, x = matrix(256, 256), torch.randn((5, 256), device="cuda")
    want, before = oz.w4_matvec(w, x), x.clone()
    for bad in (lambda: oz.w4_matvec(w, x, out=x), lambda: oz.w4_matvec(w, x[:4], out=x[1:]), lambda: oz.w4_matvec(w, x[:2], beta=1.0, c=x[2:4], out=x[3:])):
        with pytest.raises(oz.Oz2Error):
            bad()
    assert torch.equal(x, before)
    both = torch.zeros((5, 600), device="cuda")
    both[:, :256] = x
    assert torch.equal(oz.w4_matvec(w, both[:, :256], out=both[:, 256:512]), want)
    assert torch.equal(oz.w4_matvec(w, both[:, :256], beta=1.0, c=both[:, 256:512], out=both[:, 256:512]), oz.w4_matvec(w, x, beta=1.0, c=want))
    moe, ctx = layer(), oz.Context()
    ctx.allocate_moe_workspace(moe, 70)
    x = torch.randn((70, 256), device="cuda")
    want = ctx.w4_moe(moe, x)[0].clone()
    with pytest.raises(oz.Oz2Error):
        ctx.w4_moe(moe, x[:60], out=x[10:])
    ctx.w4_moe(moe, x, out=x)
    assert torch.equal(x, want)
