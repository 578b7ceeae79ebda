"""Attention over packed prompts where a call is of another size than a test by the formula in Python can be: many rows, many sequences, strides beyond 2^32 bytes.

The formula is evaluated in 64 bits on the GPU; tolerances as in test_gpu_attention (there derived): with u = 2^-24, h half a step of the type of p,
A = sum p |v| and S = scale max sum |q k|: 2 (2 (dim + 16) u S + h + (n + 72) u) (A + |out|) and one rounding to the type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def check(out, q, k, v, cu, causal=True, skip=()):
    """every row of `out` against the formula; rows of `skip` are not looked at"""
    tokens, heads, dim = q.shape
    kv_heads = k.shape[1]
    scale, h = dim ** -0.5, 0.0 if q.dtype == torch.float32 else HALF[q.dtype]
    for a, b in zip(cu[:-1], cu[1:]):
        for g in range(kv_heads if b > a else 0):
            kd, vd = k[a:b, g].double(), v[a:b, g].double()
            mask = torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").triu(1) if causal else None
            for i in range(g * heads // kv_heads, (g + 1) * heads // kv_heads):
                qd = q[a:b, i].double()
                s, most = scale * (qd @ kd.T), scale * (qd.abs() @ kd.abs().T)
                if causal:
                    s, most = s.masked_fill(mask, -math.inf), most.masked_fill(mask, 0.0)
                p = torch.softmax(s, dim=1)
                want, size = p @ vd, p @ vd.abs()
                slack = 2 * (2 * (dim + 16) * U * most.amax(1, keepdim=True) + h + (b - a + 72) * U) * (size + want.abs())
                tol = slack + HALF[out.dtype] * (want.abs() + slack) + LEAST[out.dtype]
                bad = ~((out[a:b, i].double() - want).abs() <= tol).all(1)
                for r in skip:
                    if a <= r < b:
                        bad[r - a] = False
                assert not bad.any(), "sequence at %d, head %d: rows %s" % (a, i, bad.nonzero().flatten()[:8].tolist())


def made(seed, tokens, heads, kv_heads, dim, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randn((tokens, n, dim), generator=g, device="cuda").to(dtype) for n in (heads, kv_heads, kv_heads))


def offsets(lengths):
    cu = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    return cu, torch.tensor(cu, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dim", [40, 64, 96, 128])
def test_tiles_of_all_sizes(dim, causal, name):
    """128 rows to a workgroup, 256, and 128 and 64 with keys in two parts: at ends of tiles, with shared heads that do not divide a tile"""
    for lengths, heads, kv_heads in (([1500, 0, 1, 257, 256, 64, 700], 30, 2), ([1500, 0, 1, 257, 256, 64, 700], 29, 29), ([4100, 1900], 14, 2), ([3000], 27, 27),
                                     ([3111], 6, 2), ([1100, 930], 5, 5), ([1000, 35], 14, 2), ([513, 511, 640], 3, 3), ([2900], 5, 1), ([1111, 1, 900], 2, 1)):
        cu, on = offsets(lengths)
        q, k, v = made(dim, cu[-1] + 5, heads, kv_heads, dim, TYPES[name])
        out = torch.full_like(q, 7.0)
        oz.attention(q, k, v, on, causal=causal, out=out)
        check(out, q, k, v, cu, causal)
        assert (out[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,kv_heads,more", [(32, 8, 0), (8, 8, 0), (32, 8, 3000), (4, 2, 0)], ids=["128", "128_parts", "256", "64_parts"])
def test_values_that_some_rows_do_not_see(heads, kv_heads, more, what, name):
    cu, on = offsets([1300, 1700 + more])
    q, k, v = made(3, cu[-1], heads, kv_heads, 128, TYPES[name])
    clean = v.clone()
    at = [700, 1299, 1300 + 64, 1300 + 1695]
    for t in at:
        v[t, :, 5] = what
    out = oz.attention(q, k, v, on)
    odd = [t for t in range(cu[-1]) if any(t >= a and (t < 1300) == (a < 1300) for a in at)]
    check(out, q, k, clean, cu, skip=odd)
    rest = [d for d in range(128) if d != 5]
    assert torch.isfinite(out[:, :, rest]).all() and not torch.isfinite(out[odd][:, :, 5]).any()


@pytest.mark.parametrize("name,dim,heads", [("bf16", 64, 2), ("f16", 128, 4), ("f32", 40, 2), ("bf16", 256, 2), ("bf16", 33, 2), ("bf16", 128, 40)])
def test_many_sequences(name, dim, heads):
    """more than 64, and more than 4096, some of them empty"""
    rng = np.random.default_rng(dim)
    for lengths in (rng.integers(0, 90, 65), rng.integers(0, 4, 4500), [0] * 100 + [70, 130] + [0] * 30, [1] * 300):
        cu, on = offsets(lengths)
        q, k, v = made(1, cu[-1] + 3, heads, 2, dim, TYPES[name])
        out = torch.full_like(q, 7.0)
        oz.attention(q, k, v, on, out=out)
        some = sorted(rng.choice(len(lengths), 40, replace=False)) if len(lengths) > 1000 else range(len(lengths))
        for s in some:
            check(out, q, k, v, cu[s : s + 2])
        assert (out[cu[-1]:] == 7.0).all() and torch.isfinite(out).all()
        if len(lengths) > 1000:  # the others: as if alone
            single = [i for i in range(len(lengths)) if lengths[i] == 1]
            rows = torch.tensor([cu[i] for i in single], device="cuda")
            assert torch.equal(out[rows].float(), v[rows].repeat_interleave(heads // 2, dim=1).float())


@pytest.mark.parametrize("name,dim", [("bf16", 128), ("f32", 64), ("f16", 256), ("bf16", 20)])
def test_strides_beyond_32_bits(name, dim):
    """tokens and heads that are further apart than 2^32 bytes"""
    n, step = 600, (1 << 22) + 64  # (600 2^22 elements)
    buf = torch.empty(n * step, dtype=TYPES[name], device="cuda")
    cu, on = offsets([400, 200])
    q, k, v = made(2, n, 4, 2, dim, TYPES[name])
    views = [torch.as_strided(buf, (n, h, dim), (step, dim, 1), at) for h, at in ((4, 0), (2, 4096), (2, 8192), (4, 12288))]
    for to, t in zip(views, (q, k, v)):
        to.copy_(t)
    oz.attention(*views[:3], on, out=views[3])
    check(views[3], q, k, v, cu)
    if name != "f32":  # heads before tokens
        q, k, v = made(2, 100, 600, 600, dim, TYPES[name])
        cu, on = offsets([60, 40])
        views = [torch.as_strided(buf, (100, 600, dim), (dim, step, 1), at) for at in (0, 100000, 200000, 300000)]
        for to, t in zip(views, (q, k, v)):
            to.copy_(t)
        oz.attention(*views[:3], on, out=views[3])
        check(views[3], q, k, v, cu)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("to", TYPES)
@pytest.mark.parametrize("dim", [64, 50])
def test_results_in_another_type(dim, name, to):
    cu, on = offsets([130, 20])
    q, k, v = made(4, cu[-1], 4, 2, dim, TYPES[name])
    out = torch.empty(q.shape, dtype=TYPES[to], device="cuda")
    oz.attention(q, k, v, on, out=out)
    check(out, q, k, v, cu)


def test_large_groups():
    for heads, dim, name in ((257, 128, "bf16"), (700, 64, "f16"), (100, 80, "f32")):
        cu, on = offsets([37, 3])
        q, k, v = made(5, cu[-1], heads, 1, dim, TYPES[name])
        check(oz.attention(q, k, v, on), q, k, v, cu)


def test_two_calls_at_once_and_graphs_beside_them():
    """no workspace is shared: calls of two streams and a captured one, under way together, each as if alone"""
    sets = [made(i, 2000, 16, 2, 128, torch.bfloat16) for i in range(3)]
    cu, on = offsets([1500, 500])
    want = [oz.attention(*s, on) for s in sets]
    outs = [torch.empty_like(s[0]) for s in sets]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oz.attention(*sets[2], on, out=outs[2])
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            oz.attention(*sets[i], on, out=outs[i], stream=streams[i])
        with torch.cuda.stream(streams[2]):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_no_sequences_and_no_tokens():
    q, k, v = made(6, 10, 4, 2, 64, torch.bfloat16)
    out = torch.full_like(q, 7.0)
    oz.attention(q, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"), out=out)
    oz.attention(q, k, v, torch.zeros(70, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 7.0).all()
    assert oz.attention(q[:0], k[:0], v[:0], torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
