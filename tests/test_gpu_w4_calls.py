"""How the products with weights in 4 bits are called: many rows of few codes."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz


@pytest.mark.parametrize("n", [(1 << 26) - 3, (1 << 26) + 70, (1 << 27) + 1])
def test_matvec_with_more_rows_than_a_grid_has_waves(n):
    print(n, flush=True)
    c = torch.arange(n, device="cuda").remainder_(251).to(torch.bfloat16).view(1, n)
    none = oz.W4Matrix(torch.zeros((n, 0), dtype=torch.uint8, device="cuda"), torch.zeros((n, 0), device="cuda"), k=0, group=32)
    y = oz.w4_matvec(none, torch.zeros((1, 0), dtype=torch.bfloat16, device="cuda"), beta=2.0, c=c)
    assert torch.equal(y, c * 2)
    codes = torch.arange(n, device="cuda").remainder_(253).to(torch.uint8).view(n, 1)
    w = oz.W4Matrix(codes, torch.full((n, 1), 0.5, dtype=torch.bfloat16, device="cuda"), k=2, group=32)
    y = oz.w4_matvec(w, torch.tensor([[2.0, 64.0]], dtype=torch.bfloat16, device="cuda"), out=torch.empty((1, n), device="cuda"))
    want = (codes & 15).float().sub_(8).add_((codes >> 4).float().sub_(8).mul_(32)).view(1, n)  # (exact)
    assert torch.equal(y, want)
