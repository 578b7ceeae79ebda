"""Attention with scores of any size, over packed prompts and over a cache held in 4 bits: from 2^24 on neighbouring FP32 numbers are more than one apart, and what is left of
a product when its rounded value is taken off is no longer small.

The keys differ by a 128th or more, so one of them has all the weight.  Tolerance: p is off by a few u = 2^-24, and by half a step h of the type of q once (p before it meets
v), the result by h for its rounding: (2 h + 16 u) |v|; over a cache p s by 2^-16 of it.  Rows of ordinary scores beside them: as in test_gpu_attention and test_gpu_kv4."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_attention import HALF, TYPES, U, close, formula, offsets
from test_gpu_kv4 import Held, ints

LOG2E = 1.4426950408889634
SIZES = [20, 24, 25, 26, 28, 31, 33, 36, 60, 100, 125]  # powers of two of the scores to base 2


def parts(power, name):
    """a, b, scale: scale a b log2(e) is just below 2^power, a and b within the type"""
    if name == "f16":
        a, b = 2.0 ** min(power / 2 // 1, 14), 2.0 ** min(power / 2 // 1, 14)
    else:
        a, b = 2.0 ** (power // 2), 2.0 ** (power // 4)
    scale = 2.0 ** power / (a * b * LOG2E) * 0.49  # (keys are up to 2 b)
    return (a, b, scale) if scale < 2.0 ** 126 else None


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 40, 256])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_large_scores_of_prompts(order, dim, name):
    rng = np.random.default_rng(dim)
    n = 150
    for power in SIZES:
        a, b, scale = parts(power, name)
        for sign in (1.0, -1.0):
            j = {"rising": np.arange(n) % 128, "falling": 127 - np.arange(n) % 128, "mixed": rng.permutation(n) % 128}[order]
            q, k = torch.zeros((n, 2, dim), dtype=torch.float64), torch.zeros((n, 1, dim), dtype=torch.float64)
            q[:, 0, 0], k[:, 0, 0] = sign * a, torch.from_numpy(b * (1 + j / 128))
            # the other head of the same keys: scores of -4 to 4
            k[:, 0, 1] = torch.from_numpy(rng.integers(-64, 65, n) / 16.0)
            q[:, 1, 1] = 1.0 / scale if 2.0 ** -14 < scale < 2.0 ** 14 else 0.0
            q, k = q.to(TYPES[name]), k.to(TYPES[name])
            v = torch.from_numpy(rng.standard_normal((n, 1, dim))).to(TYPES[name])
            got = oz.attention(q.cuda(), k.cuda(), v.cuda(), ints([0, n]), scale=scale)
            big = got[:, 0].double().cpu().numpy()
            vd = v[:, 0].double().numpy()
            for i in range(n):
                best = j[: i + 1].max() if sign > 0 else j[: i + 1].min()
                same = np.flatnonzero(j[: i + 1] == best)
                want, size = vd[same].mean(0), np.abs(vd[same]).mean(0)
                off = np.abs(big[i] - want)
                assert (off <= (2 * HALF[name] + 16 * U) * size + 2.0 ** -24).all(), (power, sign, i)
            qd, kd = q.double().numpy(), k.double().numpy()
            out, size, most, keys = formula(qd, kd, v.double().numpy(), offsets([n]), True, scale)
            close(got[:, 1:], (out[:, 1:], size[:, 1:], most[:, 1:], keys), name, dim)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [64, 80])
def test_ordinary_scores_behind_large_ones(dim, name):
    """first keys far below 0, then ordinary ones, whose softmax counts; and the other way round"""
    rng = np.random.default_rng(dim)
    n = 200
    for power in SIZES:
        a, b, scale = parts(power, name)
        for first in (True, False):
            far = np.arange(n) < 100 if first else np.arange(n) >= 100
            q, k = torch.zeros((n, 1, dim), dtype=torch.float64), torch.zeros((n, 1, dim), dtype=torch.float64)
            q[:, 0, 0], q[:, 0, 1] = a, 1.0 / scale if 2.0 ** -14 < scale < 2.0 ** 14 else 0.0
            k[far, 0, 0] = torch.from_numpy(-b * (1 + rng.integers(0, 128, 100) / 128))
            k[~far, 0, 1] = torch.from_numpy(rng.integers(-64, 65, 100) / 16.0)
            q, k = q.to(TYPES[name]), k.to(TYPES[name])
            v = torch.from_numpy(rng.standard_normal((n, 1, dim))).to(TYPES[name])
            got = oz.attention(q.cuda(), k.cuda(), v.cuda(), ints([0, n]), scale=scale, causal=False)
            near = np.flatnonzero(~far)
            qd, kd, vd = (t.double().numpy() for t in (q, k[near], v[near]))
            kd[..., 0] = 0.0
            x = scale * (kd[:, 0] @ qd[0, 0])
            p = np.exp(x - x.max())
            p /= p.sum()
            want = [np.broadcast_to(t, (n, 1, t.shape[-1])) for t in (p @ vd[:, 0], p @ np.abs(vd[:, 0]), np.full(1, 4.1))] + [np.full((1, 1, 1), n)]
            close(got, want, name, dim)


def test_large_scores_of_long_prompts():
    """keys in two parts, and tiles that all rows see"""
    for name, power in (("bf16", 33), ("f16", 33), ("bf16", 125), ("f32", 60), ("f16", 26)):
        for n, heads in ((1500, 2), (1500, 16), (700, 1)):
            a, b, scale = parts(power, name)
            j = np.random.default_rng(n).permutation(n)
            top = 63 + (j == n - 1)  # one is the largest
            q, k = torch.zeros((n, heads, 128)), torch.zeros((n, 1, 128))
            q[..., 0], k[:, 0, 0] = a, torch.from_numpy(b * (1 + np.where(j == n - 1, top, j % 63) / 128)).float()
            v = torch.from_numpy(np.random.default_rng(1).standard_normal((n, 1, 128))).to(TYPES[name])
            got = oz.attention(q.to(TYPES[name]).cuda(), k.to(TYPES[name]).cuda(), v.cuda(), ints([0, n]), scale=scale, causal=False).double().cpu().numpy()
            want = v[int(np.flatnonzero(j == n - 1)[0]), 0].double().numpy()
            assert (np.abs(got - want) <= (2 * HALF[name] + 16 * U) * np.abs(want) + 2.0 ** -24).all()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("n", [100, 700])
def test_large_scores_over_a_cache(n, dim, name):
    """one chunk of places, and several that come together; and what places receive"""
    rng = np.random.default_rng(n)
    for power in SIZES:
        for sign in (1.0, -1.0):
            held = Held(rng, [n, n], 1, dim, 16)
            j = rng.permutation(n) % 128
            a = 2.0 ** min(power // 2, 14 if name == "f16" else 60)
            scale = 2.0 ** power / (a * 4 * LOG2E) * 0.49
            if scale > 2.0 ** 55:
                continue
            t = np.arange(n)
            for s in (0, 1):  # keys of one value: its offset, 4 to 8
                held.scales["k"][held.table[s, t // 16], 0, t % 16, 0] = 0.0
                held.scales["k"][held.table[s, t // 16], 0, t % 16, 1] = torch.from_numpy(4 + j / 32).half()
            held.cache.k_scales.copy_(held.scales["k"])
            q = torch.zeros((2, 2, dim))
            q[:, :, 0] = sign * a
            ctx = oz.Context()
            ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=2, heads=2, weights=True)
            received = torch.zeros(held.weights.shape, device="cuda")
            out = ctx.kv4_attention(held.cache, q.to(TYPES[name]).cuda(), ints([0, 1, 2]), held.gpu_table, held.gpu_lengths, scale=scale, weights=received)
            best = np.flatnonzero(j == (j.max() if sign > 0 else j.min()))
            for s in (0, 1):
                v, vs, vo, _ = held.row("v", s, 0)
                size = (15 * vs + np.abs(vo))[best].mean()
                off = np.abs(out[s].double().cpu().numpy() - v[best].mean(0))
                assert (off <= (2.0 ** -16 + 64 * U) * size + HALF[name] * np.abs(v[best]).max()).all(), (power, sign)
                got = received[s, 0].double().cpu().numpy()
                assert (np.abs(got[best] - 2 / len(best)) <= 64 * U).all() and not np.delete(got, best).any(), (power, sign)


@pytest.mark.parametrize("name", TYPES)
def test_scores_of_zero_at_the_largest_scales(name):
    """a query of zeros weighs all keys alike"""
    rng = np.random.default_rng(5)
    held = Held(rng, [300], 1, 64, 16)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=1, heads=2, weights=True)
    q, received = torch.zeros((1, 2, 64), dtype=TYPES[name], device="cuda"), torch.zeros(held.weights.shape, device="cuda")
    out = ctx.kv4_attention(held.cache, q, ints([0, 1]), held.gpu_table, held.gpu_lengths, scale=2.0 ** 55, weights=received)
    v, vs, vo, _ = held.row("v", 0, 0)
    size = np.mean(15 * vs + np.abs(vo))
    assert (np.abs(out[0].double().cpu().numpy() - v.mean(0)) <= (2.0 ** -16 + 400 * U) * size + HALF[name] * np.abs(v.mean(0))).all()
    assert (np.abs(received[0, 0, :300].double().cpu().numpy() - 2 / 300) <= 400 * U * 2 / 300).all()
    x = torch.from_numpy(rng.standard_normal((50, 1, 64))).to(TYPES[name])
    got = oz.attention(torch.zeros_like(x).cuda(), x.cuda(), x.cuda(), ints([0, 50]), scale=2.0 ** 126, causal=False)
    mean = x.double().numpy().mean(0)
    size = np.abs(x.double().numpy()).mean(0)
    assert (np.abs(got.double().cpu().numpy() - mean) <= 400 * U * size + HALF[name] * np.abs(mean)).all()


@pytest.mark.parametrize("dim", [64, 100, 255])
def test_scores_near_the_lowest_number(dim):
    """in FP32, to base 2 -3.2e38 and 2 % below: the larger ones have all weight"""
    n = 90
    rng = np.random.default_rng(dim)
    large = rng.random(n) < 0.3
    large[0] = True
    q, k = torch.zeros((n, 1, dim)), torch.zeros((n, 1, dim))
    q[:, 0, 0] = -(2.0 ** 70)
    k[:, 0, 0] = torch.from_numpy(np.where(large, 1.0, 1.02) * 3.2e38 / LOG2E / 2.0 ** 70).float()
    v = torch.from_numpy(rng.standard_normal((n, 1, dim))).float()
    got = oz.attention(q.cuda(), k.cuda(), v.cuda(), ints([0, n]), scale=1.0, causal=False).double().cpu().numpy()
    want, size = v.double().numpy()[large].mean(0), v.abs().double().numpy()[large].mean(0)
    assert (np.abs(got - want) <= (n + 16) * U * size).all()
