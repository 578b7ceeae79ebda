"""How the products with weights in 4 bits are called: many rows of few codes; results made on another stream."""
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


def matrix(n, k, count=0):
    lead = (count,) if count else ()
    gen = torch.Generator("cuda").manual_seed(3)
    codes = torch.randint(0, 256, (*lead, n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
    return oz.W4Matrix(codes, torch.full((*lead, n, k // 32), 0.01, device="cuda"), group=32)


def after_pending_writes(shapes, launch):
    """What `launch` returns, made while the current stream has still to write into memory that it has given back: results belong to the stream
    that forms them, and those writes must not come after it."""
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for shape, dtype in shapes:
        torch.empty(shape, dtype=dtype, device="cuda").fill_(7)
    side = torch.cuda.Stream()
    got = launch(side)
    side.synchronize()
    torch.cuda.synchronize()
    return got


def test_matvec_makes_its_result_on_the_stream_it_is_given():
    w, x = matrix(1000, 1024), torch.randn((3, 1024), device="cuda")
    want = oz.w4_matvec(w, x).clone()
    for pointer in (False, True):
        got = after_pending_writes([((3, 1000), torch.float32)], lambda s: oz.w4_matvec(w, x, stream=s.cuda_stream if pointer else s))
        assert torch.equal(got, want)


def test_moe_makes_its_results_on_the_stream_it_is_given():
    layer = oz.MoeLayer(torch.randn((5, 256), device="cuda"), matrix(128, 256, 5), matrix(128, 256, 5), matrix(256, 128, 5), 3)
    ctx = oz.Context()
    ctx.allocate_moe_workspace(layer, 700)
    x = torch.randn((700, 256), device="cuda")
    want = [v.clone() for v in ctx.w4_moe(layer, x)]
    shapes = [((700, 256), torch.float32), ((700, 3), torch.int32), ((700, 3), torch.float32)]
    got = after_pending_writes(shapes, lambda s: ctx.w4_moe(layer, x, stream=s))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
