"""Caches whose scales require a gradient, or have a tangent, are refused like other tensors that do (no GPU is touched)."""
import pytest

torch = pytest.importorskip("torch")
forward_ad = pytest.importorskip("torch.autograd.forward_ad")

import paper_2504_08009_amd as oz


def calls(cache):
    q, k, cu = torch.zeros((4, 4, 64)), torch.zeros((4, 2, 64)), torch.tensor([0, 4], dtype=torch.int32)
    table, lengths, places = torch.zeros((1, 2), dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.zeros((1, 2, 32))
    ctx = oz.Context()
    yield lambda: oz.kv4_append(cache, k, k, cu, table, lengths)
    yield lambda: oz.kv4_attention(cache, q, cu, table, lengths)
    yield lambda: ctx.kv4_attention(cache, q, cu, table, lengths)
    yield lambda: oz.kv4_evict(cache, table, lengths, places.int(), places, 2)
    yield lambda: ctx.kv4_evict(cache, table, lengths, places.int(), places, 2)


def parts():
    codes, scales = torch.zeros((3, 2, 16, 32), dtype=torch.uint8), torch.zeros((3, 2, 16, 2), dtype=torch.float16)
    return [codes, scales, codes.clone(), scales.clone()]


@pytest.mark.parametrize("which", [1, 3], ids=["keys", "values"])
def test_scales_that_require_a_gradient(which):
    made = parts()
    cache = oz.KV4Cache(*made)
    for call in calls(cache):
        with pytest.raises(oz.Oz2Error, match="GPU"):
            call()
        made[which].requires_grad_(True)
        with pytest.raises(oz.Oz2Error, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(oz.Oz2Error, match="GPU"):
            call()
        made[which].requires_grad_(False)


@pytest.mark.parametrize("which", [1, 3], ids=["keys", "values"])
def test_scales_with_a_tangent(which):
    with forward_ad.dual_level():
        made = parts()
        made[which] = forward_ad.make_dual(made[which], torch.ones_like(made[which]))
        for call in calls(oz.KV4Cache(*made)):
            with pytest.raises(oz.Oz2Error, match="tangent"):
                call()
