"""Attention over packed prompts where keys hold infinities and their scores are -infinity: such keys weigh nothing, whatever the dim, and a row that sees no other is 0.

Formula and tolerances: test_gpu_attention; the largest sum |q k| is that of the keys whose scores are finite."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_attention import TYPES, close, made, offsets


def infinite(rng, q, k, at):
    """keys at `at` get an infinity in the first dim or the last that meets values of q of one sign there: scores of -infinity"""
    dim = q.shape[2]
    q[..., 0] = q[..., 0].abs() + 0.25
    q[..., dim - 1] = -q[..., dim - 1].abs() - 0.25
    for t in at:
        if dim == 1 or rng.random() < 0.6:
            k[t, :, 0] = math.inf if dim == 1 else -math.inf  # (of a single dim q is below 0)
        else:
            k[t, :, dim - 1] = math.inf


def check(q, k, v, lengths, at, name, causal, place=lambda t: t):
    cu = offsets(lengths)
    kd = k.double().numpy().copy()
    kd[~np.isfinite(kd)] = 0.0
    qd, vd, dim = q.double().numpy(), v.double().numpy(), q.shape[2]
    group, odd = q.shape[1] // k.shape[1], np.zeros(len(qd), bool)
    odd[list(at)] = True
    out, size, most, keys = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2] + (1,)), np.ones((len(qd), 1, 1))
    for a, b in zip(cu[:-1], cu[1:]):
        for i in range(a, b):
            seen = np.arange(a, i + 1 if causal else b)
            seen = seen[~odd[seen]]
            keys[i] = b - a
            for h in range(q.shape[1] if len(seen) else 0):
                x = dim ** -0.5 * (kd[seen, h // group] @ qd[i, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                out[i, h], size[i, h] = p @ vd[seen, h // group], p @ np.abs(vd[seen, h // group])
                most[i, h] = dim ** -0.5 * (np.abs(kd[seen, h // group]) @ np.abs(qd[i, h])).max()
    got = oz.attention(*(place(t.cuda()) for t in (q, k, v)), torch.from_numpy(cu).int().cuda(), causal=causal)
    assert torch.isfinite(got).all()
    close(got, (out, size, most, keys), name, dim)
    return got


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dim", [1, 3, 8, 33, 40, 64, 72, 80, 96, 100, 112, 128, 136, 200, 255, 256])
def test_infinite_keys_of_no_weight(dim, causal, name):
    rng = np.random.default_rng(dim)
    lengths = [70, 5, 130]
    q, k, v = made(rng, sum(lengths), 4, 2, dim, name)
    at = set(range(70, 75)) | {0, 3, 69, 75, 80, 140, 204} | set(rng.integers(0, 205, 10).tolist())  # (all of the second sequence's, and the first of each)
    infinite(rng, q, k, at)
    got = check(q, k, v, lengths, at, name, causal)
    assert not got[70:75].any()


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [40, 80, 112, 128])
def test_infinite_keys_in_rows_that_start_anywhere(dim, name):
    def anywhere(t):
        buf = torch.full((t.shape[0], t.shape[1] * dim + 1), math.nan, dtype=t.dtype, device="cuda")
        view = buf[:, 1:].unflatten(1, t.shape[1:])
        view.copy_(t)
        return view

    rng = np.random.default_rng(dim)
    q, k, v = made(rng, 90, 4, 2, dim, name)
    infinite(rng, q, k, {0, 7, 50, 89})
    check(q, k, v, [60, 30], {0, 7, 50, 89}, name, True, anywhere)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("dim,heads,lengths", [(80, 16, [1500]), (40, 2, [1200]), (112, 2, [900]), (104, 8, [3200])])
def test_infinite_keys_of_long_prompts(dim, heads, lengths, name):
    """tiles of all sizes, with keys in one part and in two; a few rows against the formula, and no NaN in the others"""
    rng = np.random.default_rng(dim)
    n = lengths[0]
    q, k, v = made(rng, n, heads, 1, dim, name)
    at = sorted(set(rng.integers(0, n, n // 10).tolist()))
    infinite(rng, q, k, at)
    got = oz.attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, n], dtype=torch.int32, device="cuda"), causal=False)
    assert torch.isfinite(got).all()
    keep = [t for t in range(n) if t not in set(at)]
    kd, vd, qd = k[keep, 0].double().numpy(), v[keep, 0].double().numpy(), q[::97].double().numpy()
    x = np.einsum("ihd,jd->ihj", qd, kd) * dim ** -0.5
    p = np.exp(x - x.max(2, keepdims=True))
    p /= p.sum(2, keepdims=True)
    most = np.einsum("ihd,jd->ihj", np.abs(qd), np.abs(kd)).max(2)[..., None] * dim ** -0.5
    close(got[::97], (p @ vd, p @ np.abs(vd), most, np.full((len(qd), 1, 1), n)), name, dim)
