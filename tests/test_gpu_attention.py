"""Attention over packed prompts, against its formula in 64 bits.

Tolerances (u = 2^-24).  A score is a sum of dim exact or FP32 products in FP32, then scaled and taken to base 2: off by at most e = (dim + 16) u scale max_j sum_d |q k_j|,
so p is off by a factor within 1 +- (2 e + 8 u); sums of n terms add n u.  16-bit types round p once more, by half a step h (2^-8, 2^-11), before it meets v:
with A = sum p |v| the result is off by at most (2 e + h + (n + 72) u) (A + |out|), times 2 for what is of second order, before the
one rounding to the type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step, relative
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def formula(q, k, v, cu, causal, scale):
    """(out, A, max sum |q k|, keys) in 64 bits; q (tokens, heads, dim) ..., what a row does not see is not touched"""
    tokens, heads, dim = q.shape
    group = heads // k.shape[1]
    out, size, most, keys = np.zeros(q.shape), np.zeros(q.shape), np.zeros((tokens, heads, 1)), np.ones((tokens, 1, 1))
    with np.errstate(all="ignore"):
        for a, b in zip(cu[:-1], cu[1:]):
            for h in range(heads):
                for i in range(a, b):
                    e = i + 1 if causal else b
                    s = scale * (k[a:e, h // group] @ q[i, h])
                    if not (s > -np.inf).any() and not np.isnan(s).any():
                        continue
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[i, h], size[i, h] = p @ v[a:e, h // group], p @ np.abs(v[a:e, h // group])
                    most[i, h], keys[i] = scale * (np.abs(k[a:e, h // group]) @ np.abs(q[i, h])).max(), e - a
    return out, size, most, keys


def close(got, want, name, dim, rows=slice(None)):
    out, size, most, keys = (w[rows] for w in want)
    got = got.double().cpu().numpy()[rows]
    h = 0.0 if name == "f32" else HALF[name]
    slack = 2 * (2 * (dim + 16) * U * most + h + (keys + 72) * U) * (size + np.abs(out))
    tol = slack + HALF[name] * (np.abs(out) + slack) + LEAST[name]
    bad = ~(np.abs(got - out) <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g times the tolerance" % (bad.sum(), bad.size, np.nanmax(np.abs(got - out) / tol))


def made(rng, tokens, heads, kv_heads, dim, name, size=1.0):
    q, k, v = (torch.from_numpy(rng.standard_normal((tokens, n, dim)) * s).to(TYPES[name]) for n, s in ((heads, size), (kv_heads, 1.0), (kv_heads, 1.0)))
    return q, k, v


def check(lengths, heads, kv_heads, dim, name, causal=True, behind=0, seed=0, size=1.0, scale=None):
    rng = np.random.default_rng(seed)
    cu = offsets(lengths)
    tokens = int(cu[-1]) + behind
    q, k, v = made(rng, tokens, heads, kv_heads, dim, name, size)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    back = oz.attention(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cu).int().cuda(), causal=causal, scale=scale, out=out)
    assert back is out
    want = formula(*(t.double().numpy() for t in (q, k, v)), cu, causal, dim ** -0.5 if scale is None else scale)
    close(out, want, name, dim, slice(0, int(cu[-1])))
    assert (out[cu[-1]:] == 7.0).all()


SHAPES = [  # lengths, heads, kv heads, dim
    ([1], 1, 1, 64), ([1], 8, 2, 128), ([2], 4, 1, 64), ([17], 2, 2, 128), ([31, 1, 33], 4, 2, 64), ([0, 5, 0, 64, 1, 0], 6, 2, 128), ([63, 65], 3, 1, 128),
    ([64, 128], 8, 8, 64), ([127, 129], 8, 1, 128), ([257], 4, 2, 128), ([300, 7, 100], 8, 2, 128), ([513], 2, 1, 64), ([40] * 9, 4, 4, 96), ([130, 70], 4, 2, 80),
    ([129], 2, 1, 256), ([75, 3], 4, 2, 200), ([66], 16, 1, 128), ([33], 5, 1, 72), ([90], 7, 7, 40), ([50, 20], 2, 1, 8),
]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape, causal, name):
    check(*shape, name, causal, behind=3, seed=len(str(shape)))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 17, 33, 63, 65, 100, 127, 129, 255])
def test_odd_dims(dim, name):
    check([35, 4], 2, 1, dim, name, seed=dim)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
def test_peaked_scores(dim, name):
    """one key takes nearly everything, and the maximum rises along the row"""
    check([200, 90], 4, 2, dim, name, size=8.0, seed=5)
    check([100], 2, 1, dim, name, scale=3.0, seed=6)
    check([100], 2, 1, dim, name, scale=1e-6, seed=7)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_maximum_that_rises_at_every_key(name):
    """scores that climb by more than the kernel lets pass before it takes a new maximum"""
    n, dim = 300, 64
    q, k = torch.zeros((n, 1, dim)), torch.zeros((n, 1, dim))
    q[:, 0, 0], k[:, 0, 0] = 16.0, torch.arange(n)
    q, k = q.to(TYPES[name]), k.to(TYPES[name])
    v = torch.from_numpy(np.random.default_rng(0).standard_normal((n, 1, dim))).to(TYPES[name])
    cu = np.array([0, n])
    for order in (torch.arange(n), torch.arange(n - 1, -1, -1)):
        out = oz.attention(q.cuda(), k[order].cuda(), v.cuda(), torch.tensor(cu, dtype=torch.int32, device="cuda"), causal=False)
        close(out, formula(q.double().numpy(), k[order].double().numpy(), v.double().numpy(), cu, False, dim ** -0.5), name, dim)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 128), (3, 1, 64), (2, 2, 40)])
def test_strides(heads, kv_heads, dim, name):
    """parts of one packed tensor, rows that start anywhere, heads before tokens"""
    rng = np.random.default_rng(1)
    lengths = [70, 30]
    cu = offsets(lengths)
    n = int(cu[-1])
    q, k, v = made(rng, n, heads, kv_heads, dim, name)
    want = formula(*(t.double().numpy() for t in (q, k, v)), cu, True, dim ** -0.5)
    cu_gpu = torch.from_numpy(cu).int().cuda()
    for shift in (0, 1, 3):
        packed = torch.full((n, (2 * heads + 2 * kv_heads) * dim + shift), math.nan, dtype=TYPES[name], device="cuda")
        parts, at = [], shift
        for t in (q, k, v, q):
            parts.append(packed[:, at: at + t.shape[1] * dim].unflatten(1, (t.shape[1], dim)))
            at += t.shape[1] * dim
        for to, t in zip(parts[:3], (q, k, v)):
            to.copy_(t)
        before = packed.clone()
        oz.attention(*parts[:3], cu_gpu, out=parts[3])
        close(parts[3], want, name, dim)
        end = (heads + 2 * kv_heads) * dim + shift
        assert torch.equal(packed[:, shift:end], before[:, shift:end])
    turned = [t.cuda().transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    out = torch.empty((heads, n, dim), dtype=TYPES[name], device="cuda").transpose(0, 1)
    close(oz.attention(*turned, cu_gpu, out=out), want, name, dim)
    wide = torch.empty((n, heads, dim), device="cuda")
    close(oz.attention(*turned, cu_gpu, out=wide), want, "f32" if name == "f32" else name, dim)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(what, dim, name):
    """keys and values of later tokens and of the neighbouring sequences that are not finite; the rows that see them are as the formula says"""
    rng = np.random.default_rng(2)
    lengths = [37, 70, 20]
    cu = offsets(lengths)
    q, k, v = made(rng, int(cu[-1]) + 2, 4, 2, dim, name)
    cases = [(v, cu[1] + 33, slice(None), slice(3, 6)), (k, cu[1] + 50, 0, slice(None)), (v, cu[0], 1, slice(1)), (v, cu[3], slice(None), slice(None)),
             (k, cu[3] + 1, slice(None), slice(None)), (v, cu[3] - 1, 0, slice(dim - 1, dim))]
    for t, at, head, dims in cases:
        t[int(at), head, dims] = what
    want = formula(*(t.double().numpy() for t in (q, k, v)), cu, True, dim ** -0.5)
    out = oz.attention(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cu).int().cuda())
    got, n = out.double().cpu().numpy()[: cu[-1]], int(cu[-1])
    fine = np.isfinite(want[0][:n])
    assert fine.any() and not fine.all()
    # (a score of +-infinity times finite values, and what is not finite in 64 bits: the same kind of number, or NaN where infinities meet)
    assert np.isfinite(got[fine]).all() and not np.isfinite(got[~fine]).any()
    safe = np.where(fine, want[0][:n], 0.0)
    finite = [np.nan_to_num(w[:n], nan=0.0, posinf=0.0, neginf=0.0) for w in (want[1], np.broadcast_to(want[2], want[0].shape))]
    close(torch.from_numpy(np.where(fine, got, 0.0)), (safe, finite[0], finite[1], want[3][:n]), name, dim)


def test_offsets_that_lie_are_cut_off():
    """nothing outside the tensors is read or written: ends behind them, begins before them, offsets that descend"""
    q, k, v = (t.cuda() for t in made(np.random.default_rng(3), 50, 4, 2, 128, "bf16"))
    for cu in ([0, 60], [-5, 50], [0, 30, 20, 50], [50, 50, 90], [0, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1], [0, 25, 25, 25, 50]):
        out = torch.full_like(q, 7.0)
        oz.attention(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out=out)
        if cu[-1] >= 50 and sorted(cu) == cu and len(cu) == 2:
            assert torch.equal(out, oz.attention(q, k, v, torch.tensor([0, 50], dtype=torch.int32, device="cuda")))


def test_long_prompts():
    """a sequence of 4097 tokens beside short ones: rows spread over it, against the formula"""
    rng = np.random.default_rng(4)
    lengths, heads, kv_heads, dim = [5, 4097, 600], 2, 1, 128
    cu = offsets(lengths)
    q, k, v = made(rng, int(cu[-1]), heads, kv_heads, dim, "bf16")
    out = oz.attention(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cu).int().cuda()).cpu()
    for i in [0, 4, 5, 6, 100, 2048, 4095, 4101, 4102, 4701]:
        a = cu[np.searchsorted(cu, i, side="right") - 1]
        kd, vd, qd = k[a : i + 1, 0].double().numpy(), v[a : i + 1, 0].double().numpy(), q[i].double().numpy()
        s = qd @ kd.T * dim ** -0.5
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want = ((p @ vd)[None], (p @ np.abs(vd))[None], (np.abs(qd) @ np.abs(kd).T).max(1)[None, :, None] * dim ** -0.5, np.full((1, 1, 1), len(kd)))
        close(out[i : i + 1], want, "bf16", dim)


def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs():
    q, k, v = (t.cuda() for t in made(np.random.default_rng(5), 700, 8, 2, 128, "bf16"))
    cu = torch.tensor([0, 400, 700], dtype=torch.int32, device="cuda")
    want = oz.attention(q, k, v, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = oz.attention(q, k, v, cu, stream=side)
    side.synchronize()
    assert torch.equal(there, want)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oz.attention(q, k, v, cu, out=out)
    for i in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        q.mul_(0.5)
        want = oz.attention(q, k, v, cu)
