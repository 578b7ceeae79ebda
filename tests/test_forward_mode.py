"""Tensors with a tangent (forward-mode differentiation) are refused, as are those that require a gradient: the library forms neither (no GPU is touched)."""
import pytest

torch = pytest.importorskip("torch")
forward_ad = pytest.importorskip("torch.autograd.forward_ad")

import paper_2504_08009_amd as oz


def calls():
    """(names, call of tensors by name)"""
    q, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths, places = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.zeros((1, 2, 32))
    cache = oz.KV4Cache.empty(3, 2, 16, 64, device="cpu")
    t = dict(q=q, k=k, v=k.clone(), out=q.clone(), weights=places)
    yield ("q", "k", "v", "out"), t, lambda q, k, v, out, **_: oz.attention(q, k, v, cu, out=out)
    yield ("k", "v", "weights"), t, lambda k, v, weights, **_: oz.kv4_append(cache, k, v, cu, table, lengths, weights=weights)
    yield ("k", "v"), t, lambda k, v, **_: oz.kv4_append(cache, t["k"], t["v"], cu, table, lengths, held=(k, v))
    yield ("q", "out", "weights"), t, lambda q, out, weights, **_: oz.kv4_attention(cache, q, cu, table, lengths, weights=weights, out=out)
    yield ("q",), t, lambda q, **_: oz.Context().kv4_attention(cache, q, cu, table, lengths)
    yield ("weights",), t, lambda weights, **_: oz.kv4_evict(cache, table, lengths, places.int(), weights, 2)
    W = oz.W4Matrix(torch.zeros((8, 32), dtype=torch.uint8), torch.ones((8, 1)), group=64)
    w = dict(x=torch.zeros((3, 64)), c=torch.zeros((3, 8)), out=torch.zeros((3, 8)))
    yield ("x", "c", "out"), w, lambda x, c, out: oz.w4_matvec(W, x, beta=1.0, c=c, out=out)
    stack = lambda n: oz.W4Matrix(torch.zeros((4, n, 32), dtype=torch.uint8), torch.ones((4, n, 1)), group=64)
    layer = oz.MoeLayer(torch.zeros((4, 64)), stack(64), stack(64), stack(64), top_k=2)
    yield ("x",), w, lambda x, **_: oz.w4_moe(layer, x)


def test_tangents_are_refused():
    for names, tensors, call in calls():
        for name in names:
            with forward_ad.dual_level():
                dual = dict(tensors, **{name: forward_ad.make_dual(tensors[name], torch.ones_like(tensors[name]))})
                with pytest.raises(oz.Oz2Error, match="tangent"):
                    call(**dual)
                with torch.no_grad(), pytest.raises(oz.Oz2Error, match="tangent"):
                    call(**dual)
                with pytest.raises(oz.Oz2Error, match="GPU"):  # without one, also while others have some
                    call(**tensors)


def test_tangents_of_weights_are_refused():
    with forward_ad.dual_level():
        W = oz.W4Matrix(torch.zeros((8, 32), dtype=torch.uint8), forward_ad.make_dual(torch.ones((8, 1)), torch.ones((8, 1))), group=64)
        with pytest.raises(oz.Oz2Error, match="tangent"):
            oz.w4_matvec(W, torch.zeros((3, 64)))


def test_transforms_of_functions_are_refused():
    x, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(oz.Oz2Error, match="tangent"):
        torch.func.jvp(lambda x: oz.attention(x, k, k, cu), (x,), (x,))
    with pytest.raises(oz.Oz2Error, match="gradient"):
        torch.func.grad(lambda x: oz.attention(x, k, k, cu).sum())(x)
