"""examples/decode_w4.py: both operators in a decoder's step, eager, captured, and against products with the weights in 64 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decode_w4", os.path.join(ROOT, "examples", "decode_w4.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(w):
    q = torch.stack((w.codes & 15, w.codes >> 4), dim=-1).flatten(-2).double() - 8
    return q * w.scales.double().repeat_interleave(64, dim=-1)  # (groups of 64)


@pytest.mark.parametrize("tokens", [1, 3, 6])
def test_a_captured_step_repeats_the_eager_one(tokens):
    d = example().Decoder(tokens, 2, 256, 192, 6, 2, 500)
    first, eager = d.token.clone(), []
    for _ in range(5):
        d.step()
        eager.append((d.token.clone(), d.logits.clone()))
    d.token.copy_(first)
    d.capture()
    for token, logits in eager:
        d.graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d.token, token) and torch.equal(d.logits, logits)


@pytest.mark.parametrize("tokens", [1, 5])
def test_a_step_against_64_bits(tokens):
    """One layer, every tensor from the ones that the step left: a result in bf16 is within 2^-8 of it, and what FP32 sums of at most 512 products
    add is far below that of the sizes."""
    d = example().Decoder(tokens, 1, 256, 512, 6, 2, 500)
    d.step()
    up, down, moe = d.layers[0]
    x = d.embedding[torch.arange(tokens, device="cuda")].double()
    inner = (x @ plain(up).t()).relu()
    assert bool(((d.inner.double() - inner).abs() <= 2.0 ** -8 * inner.abs() + 1e-4).all())
    mixed = d.inner.double() @ plain(down).t() + x
    assert bool(((d.mixed.double() - mixed).abs() <= 2.0 ** -8 * mixed.abs() + 1e-4).all())
    m = d.mixed.double()
    p, ids = (m @ moe.router.double().t()).softmax(1).topk(2)
    want = torch.zeros_like(m)
    gate, upper, lower = plain(moe.gate), plain(moe.up), plain(moe.down)
    for t in range(tokens):
        for j in range(2):
            e = int(ids[t, j])
            g = gate[e] @ m[t]
            want[t] += p[t, j] / p[t].sum() * (lower[e] @ (g * g.sigmoid() * (upper[e] @ m[t])))
    assert bool(((d.expert.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
