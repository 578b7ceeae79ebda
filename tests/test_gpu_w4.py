"""Products with weights held in 4 bits and layers of experts on them, against their formulas in 64 bits.

Tolerances.  All sums are in FP32 (u = 2^-24).  A kernel may add (c + q) x with a constant c <= 16 in the place of q x and take c sum x off
again, so a group's sum is off by at most (terms of its longest chain of additions) u sum (16 + q + z) |x|; with S = sum |s| (32 + z) |x| >= all
of that, and chains of at most min(group, k) terms inside a group and ceil(k / group) + 16 outside, a product is off by at most
  depth u S,   depth = 2 min(group, k, 1024) + ceil(k / 32) + 32,
(a kernel may cut long groups into pieces of 32 or more), before the one rounding to the result's type.  What depends on a product through act() is
followed by its derivative: |act'| < 1.13 for silu and gelu."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": (2.0 ** -24, 2.0 ** -149), "bf16": (2.0 ** -8, 2.0 ** -133), "f16": (2.0 ** -11, 2.0 ** -24)}  # (an ulp, to be safe)


def rounded(x, name):
    """numpy float64 holding values of the type, and the tensor of them on the GPU"""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(TYPES[name])
    return t.double().numpy(), t.cuda()


class Weights:
    def __init__(self, rng, stack, n, k, group, zeros, scales="f32", pad=0):
        self.k, self.group, groups, width = k, group, -(-k // group), (k + 1) // 2
        self.codes = rng.integers(0, 256, (*stack, n, width + pad), dtype=np.uint8)
        q = np.stack((self.codes[..., :width] & 15, self.codes[..., :width] >> 4), axis=-1).reshape(*stack, n, 2 * width)[..., :k]
        self.s, s = rounded(rng.uniform(0.5, 1.5, (*stack, n, groups)) * np.where(rng.random((*stack, n, groups)) < 0.1, -1, 1) / math.sqrt(max(k, 1)), scales)
        self.z = rng.integers(0, 16, (*stack, n, groups)).astype(np.uint8) if zeros else None
        if pad:
            s = torch.nn.functional.pad(s, (0, pad), value=float("nan"))
        z = None if self.z is None else torch.from_numpy(np.pad(self.z, [(0, 0)] * (self.z.ndim - 1) + [(0, pad)], constant_values=255)).cuda()
        self.gpu = oz.W4Matrix(torch.from_numpy(self.codes).cuda(), s, z, k=k, group=group)
        at = np.arange(k) // group
        self.q = q.astype(np.float64) - (8.0 if self.z is None else self.z[..., at])
        self.w = self.s[..., at] * self.q
        zeros_at = 8.0 if self.z is None else self.z[..., at].astype(np.float64)
        self.size = np.abs(self.s[..., at]) * (32.0 + zeros_at)
        self.depth = 2 * min(group, k, 1024) + -(-k // 32) + 32

    def one(self, e):
        other = object.__new__(Weights)
        other.w, other.size, other.depth = self.w[e], self.size[e], self.depth
        return other


def close(got, want, slack, name):
    """got: tensor; want, slack: float64 arrays"""
    g = got.double().cpu().numpy()
    rel, least = HALF_ULP[name]
    tol = slack + rel * (np.abs(want) + slack) + least
    assert g.shape == want.shape
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g times the tolerance" % (bad.sum(), bad.size, np.nanmax(np.abs(g - want) / tol))


MATVEC = [  # n, k, t, group, zeros, x, scales, result
    (1, 1, 1, 32, False, "f32", "f32", "f32"),
    (1, 2, 1, 32, True, "bf16", "bf16", "bf16"),
    (3, 31, 1, 32, True, "f16", "f16", "f16"),
    (16, 32, 2, 32, False, "bf16", "f32", "f32"),
    (17, 33, 2, 32, True, "f32", "bf16", "f32"),
    (15, 64, 3, 64, True, "f32", "f32", "f32"),
    (64, 127, 4, 64, False, "f16", "f32", "f32"),
    (64, 128, 4, 128, True, "bf16", "bf16", "f32"),
    (100, 129, 5, 128, True, "bf16", "f16", "bf16"),
    (65, 255, 8, 128, False, "f32", "f32", "f32"),
    (257, 1000, 16, 128, True, "bf16", "bf16", "bf16"),
    (33, 4160, 17, 64, True, "f16", "f16", "f16"),
    (250, 777, 33, 32, True, "f32", "f32", "f32"),
    (48, 9001, 1, 32, False, "f32", "f32", "f32"),
    (40, 700, 6, 1024, True, "bf16", "f32", "f32"),
    (40, 700, 1, 384, True, "f16", "f32", "f32"),
    (31, 2500, 9, 256, False, "f32", "bf16", "f32"),
    (1, 16384, 1, 128, False, "bf16", "bf16", "f32"),
    (2000, 96, 1, 32, False, "bf16", "bf16", "f32"),
    (70, 3200, 64, 128, True, "bf16", "bf16", "f32"),
    (5, 20011, 4, 64, True, "f32", "f32", "f32"),
    (129, 2048, 13, 128, False, "f16", "f16", "f32"),
    (4100, 512, 2, 128, False, "bf16", "bf16", "bf16"),
]


@pytest.mark.parametrize("case", MATVEC, ids=lambda c: "-".join(map(str, c)))
def test_matvec(case):
    n, k, t, group, zeros, x_type, s_type, y_type = case
    rng = np.random.default_rng(n * 1000 + k + t)
    print(case, flush=True)
    w = Weights(rng, (), n, k, group, zeros, s_type)
    x, gx = rounded(rng.standard_normal((t, k)) * np.where(rng.random(k) < 0.05, 30, 1), x_type)
    y = oz.w4_matvec(w.gpu, gx, out=torch.full((t, n), float("nan"), dtype=TYPES[y_type], device="cuda"))
    close(y, x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), y_type)


@pytest.mark.parametrize("x_type,t,k", [("bf16", 3, 300), ("f32", 1, 301), ("f16", 18, 1027), ("bf16", 1, 2049), ("f32", 7, 96)])
@pytest.mark.parametrize("start", [0, 1, 3])
def test_matvec_with_gaps_and_odd_starts_in_place(x_type, t, k, start):
    """alpha W x + beta C in place, codes at odd addresses, pitches with gaps that hold NaN or garbage, nothing written between"""
    rng = np.random.default_rng(k + start)
    n, group = 75, 64
    print(x_type, t, k, start, flush=True)
    w = Weights(rng, (), n, k, group, True, "f32", pad=5)
    codes = torch.zeros(n * w.codes.shape[1] + 16, dtype=torch.uint8, device="cuda")
    view = codes[start:start + n * w.codes.shape[1]].view(n, w.codes.shape[1])
    view.copy_(torch.from_numpy(w.codes))
    gpu = oz.W4Matrix(view, w.gpu.scales, w.gpu.zeros, k=k, group=group)
    x, gx = rounded(rng.standard_normal((t, k)), x_type)
    wide = torch.full((t, k + 7), float("nan"), dtype=gx.dtype, device="cuda")
    wide[:, start:start + k] = gx
    c, gc = rounded(rng.standard_normal((t, n)), x_type)
    y = torch.full((t, n + 3), 5.0, dtype=gx.dtype, device="cuda")
    y[:, :n] = gc
    oz.w4_matvec(gpu, wide[:, start:start + k], alpha=-0.75, beta=1.5, c=y[:, :n], out=y[:, :n])
    want = -0.75 * (x @ w.w.T) + 1.5 * c
    close(y[:, :n], want, (w.depth + 4) * U * (np.abs(x) @ w.size.T + 2 * np.abs(c)), x_type)
    assert bool((y[:, n:] == 5.0).all())


def test_matvec_reads_no_more_than_its_rows():
    """the last row ends where the codes, scales, zeros and x end; what a pitch leaves between rows is never used"""
    rng = np.random.default_rng(3)
    for n, k, group in [(19, 999, 32), (16, 130, 128), (1, 5, 32), (33, 257, 64)]:
        print(n, k, group, flush=True)
        w = Weights(rng, (), n, k, group, True)
        x, gx = rounded(rng.standard_normal((2, k)), "bf16")
        y = oz.w4_matvec(w.gpu, gx, out=torch.empty((2, n), device="cuda"))
        again = Weights.__new__(Weights)
        poisoned = w.codes.copy()
        if k % 2:
            poisoned[:, -1] ^= 0xF0     # the half byte behind an odd row
        again = oz.W4Matrix(torch.from_numpy(poisoned).cuda(), w.gpu.scales, w.gpu.zeros, k=k, group=group)
        assert torch.equal(y, oz.w4_matvec(again, gx, out=torch.empty((2, n), device="cuda")))
        close(y, x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")


def test_matvec_of_nothing_and_scalars():
    rng = np.random.default_rng(4)
    w = Weights(rng, (), 40, 100, 32, False)
    x, gx = rounded(rng.standard_normal((3, 100)), "f32")
    c, gc = rounded(rng.standard_normal((3, 40)), "f32")
    nan = torch.full((3, 100), float("nan"), device="cuda")
    assert np.array_equal(oz.w4_matvec(w.gpu, nan, alpha=0.0, beta=2.0, c=gc).cpu().numpy(), (2 * c).astype(np.float32))
    assert bool((oz.w4_matvec(w.gpu, nan, alpha=0.0) == 0).all())
    out = torch.full((3, 40), float("nan"), device="cuda")
    oz.w4_matvec(w.gpu, gx, beta=0.0, c=out, out=out)
    close(out, x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")
    none = oz.W4Matrix(torch.zeros((40, 0), dtype=torch.uint8, device="cuda"), torch.zeros((40, 0), device="cuda"), k=0, group=32)
    assert np.array_equal(oz.w4_matvec(none, torch.zeros((3, 0), device="cuda"), beta=-1.0, c=gc).cpu().numpy(), -c.astype(np.float32))
    assert bool((oz.w4_matvec(none, torch.zeros((3, 0), device="cuda"), out=torch.ones((3, 40), device="cuda")) == 0).all())
    assert oz.w4_matvec(w.gpu, gx[:0]).shape == (0, 40)
    assert bool((oz.w4_matvec(w.gpu, torch.zeros_like(gx)) == 0).all())


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("t", [1, 5])
def test_matvec_with_infinities_and_nans_follows_the_formula(x_type, t):
    """by groups: s sum (q - z) x; an infinity where q is z makes a NaN, elsewhere an infinity of its sign or, beside its opposite, a NaN"""
    rng = np.random.default_rng(5 + t)
    n, k, group = 90, 500, 64
    print(x_type, t, flush=True)
    w = Weights(rng, (), n, k, group, True)
    x = rng.standard_normal((t, k))
    x[0, 70] = np.inf
    if t > 1:
        x[1, 499] = -np.inf
        x[2, [3, 4]] = np.inf
        x[3, 250] = np.nan
    x, gx = rounded(x, x_type)
    got = oz.w4_matvec(w.gpu, gx, out=torch.empty((t, n), device="cuda")).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        groups = np.arange(0, k, group)
        sums = np.add.reduceat(w.q[None] * x[:, None, :], groups, axis=2)
        want = (sums * w.s[None]).sum(axis=2)
    assert np.isinf(want).any() and (t == 1 or np.isnan(want).any())
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    fine = np.isfinite(want)
    slack = w.depth * U * (np.abs(np.where(np.isfinite(x), x, 0)) @ w.size.T)
    assert np.all(np.abs(got - want)[fine] <= (slack + U * np.abs(want) + 1e-30)[fine])


def test_matvec_with_values_at_the_ends_of_the_range():
    """FP32 inputs near the largest and the smallest values: nothing overflows or is lost that the formula keeps"""
    rng = np.random.default_rng(6)
    w = Weights(rng, (), 64, 256, 32, True)
    for scale in (2.0 ** 120, 2.0 ** -100):
        x, gx = rounded(rng.standard_normal((2, 256)) * scale, "f32")
        close(oz.w4_matvec(w.gpu, gx), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")
    x = np.zeros((1, 256))
    x[0, 7] = 3.4e38
    x, gx = rounded(x, "f32")
    small = oz.W4Matrix(w.gpu.codes, w.gpu.scales * 2.0 ** -20, w.gpu.zeros, group=32)
    close(oz.w4_matvec(small, gx), x @ w.w.T * 2.0 ** -20, w.depth * U * (np.abs(x) @ w.size.T) * 2.0 ** -20, "f32")


@pytest.mark.parametrize("t,n,k", [(1, 40, 1500), (2, 40, 1500), (3, 40, 700), (9, 40, 700), (1, 40, 40)])
def test_matvec_keeps_the_smallest_half_precision_values(t, n, k):
    """subnormal f16 values of x are values"""
    rng = np.random.default_rng(31 + t)
    w = Weights(rng, (), n, k, 32, True)
    x, gx = rounded(rng.standard_normal((t, k)) * 2.0 ** -20, "f16")
    assert np.abs(x).max() < 2.0 ** -14
    close(oz.w4_matvec(w.gpu, gx, out=torch.empty((t, n), device="cuda")), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,group", [(1024, 64), (1100, 32), (2048, 128), (2050, 128), (5000, 64), (16384, 1024), (16390, 128)])
@pytest.mark.parametrize("t", [1, 2, 3, 6])
def test_matvec_at_the_ends_of_its_kernels_ranges(x_type, k, group, t):
    rng = np.random.default_rng(k + t)
    n = 37
    w = Weights(rng, (), n, k, group, k % 4 == 0, x_type)
    x, gx = rounded(rng.standard_normal((t, k)), x_type)
    close(oz.w4_matvec(w.gpu, gx, out=torch.empty((t, n), device="cuda")), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")


@pytest.mark.parametrize("t", [1, 2, 4, 16])
def test_matvec_of_many_rows(t):
    """more rows than one round of the workgroups takes, and a last batch that is not whole"""
    rng = np.random.default_rng(32 + t)
    n, k = 60001, 1056
    codes = torch.from_numpy(rng.integers(0, 256, (n, k // 2), dtype=np.uint8)).cuda()
    scales = torch.rand((n, k // 32), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) + 0.5
    x, gx = rounded(rng.standard_normal((t, k)), "bf16")
    y = oz.w4_matvec(oz.W4Matrix(codes, scales, group=32), gx, out=torch.empty((t, n), device="cuda"))
    q = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(1).double() - 8
    w = q * scales.double().repeat_interleave(32, dim=1)
    tol = (2 * 32 + 33 + 32) * U * (gx.double().abs() @ (scales.double() * 40).repeat_interleave(32, dim=1).t()) + 1e-30
    assert bool(((y.double() - gx.double() @ w.t()).abs() <= tol * (1 + U)).all())


def test_matvec_vectors_do_not_touch_each_other():
    """what one vector holds changes no bit of another's result"""
    rng = np.random.default_rng(33)
    for t, n, k in [(2, 50, 1500), (4, 50, 700), (11, 50, 900), (20, 50, 300)]:
        w = Weights(rng, (), n, k, 64, True)
        x, gx = rounded(rng.standard_normal((t, k)), "f32")
        clean = oz.w4_matvec(w.gpu, gx)
        gx[1, [0, k - 1]] = torch.tensor([float("inf"), float("nan")], device="cuda")
        got = oz.w4_matvec(w.gpu, gx)
        keep = [i for i in range(t) if i != 1]
        assert torch.equal(got[keep], clean[keep]) and bool(got[1].isnan().all())


def test_matvec_with_a_scale_that_is_not_finite():
    rng = np.random.default_rng(34)
    for t, k in [(1, 1300), (3, 650), (1, 30)]:
        w = Weights(rng, (), 40, k, 32, False)
        w.gpu.scales[7, 0] = float("inf")
        w.gpu.scales[11, -1] = float("nan")
        x, gx = rounded(rng.standard_normal((t, k)) + 3, "bf16")
        y = oz.w4_matvec(w.gpu, gx, out=torch.empty((t, 40), device="cuda"))
        bad = torch.zeros(40, dtype=torch.bool, device="cuda")
        bad[[7, 11]] = True
        assert not bool(y[:, bad].isfinite().any()) and bool(y[:, ~bad].isfinite().all())


def test_matvec_beyond_32_bits_of_offset():
    """rows, and vectors, more than 2^32 bytes apart"""
    rng = np.random.default_rng(7)
    n, k, pitch = 4, 70, (1 << 31) - 1
    w = Weights(rng, (), n, k, 32, False)
    big = torch.zeros(3 * pitch + 64, dtype=torch.uint8, device="cuda")
    codes = big.as_strided((n, 35), (pitch, 1))
    codes.copy_(torch.from_numpy(w.codes))
    x, gx = rounded(rng.standard_normal((3, k)), "bf16")
    room = torch.zeros(2 * (1 << 30) + 128, dtype=torch.bfloat16, device="cuda")
    xs = room.as_strided((3, k), (1 << 30, 1))
    xs.copy_(gx)
    ys = room.as_strided((3, n), (1 << 30, 1), 100)
    oz.w4_matvec(oz.W4Matrix(codes, w.gpu.scales, k=k, group=32), xs, out=ys)
    close(ys.contiguous(), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "bf16")


def test_matvec_repeats_bit_for_bit_on_any_stream_and_in_a_graph():
    rng = np.random.default_rng(8)
    w = Weights(rng, (), 300, 1500, 128, True, "bf16")
    xs = [rounded(rng.standard_normal((3, 1500)), "bf16")[1] for _ in range(4)]
    first = [oz.w4_matvec(w.gpu, x) for x in xs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for x, y in zip(xs, first):
        there = oz.w4_matvec(w.gpu, x, stream=side)
        side.synchronize()
        assert torch.equal(there, y)
    x, y = xs[0].clone(), torch.empty_like(first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oz.w4_matvec(w.gpu, x, out=y)
    for other, want in list(zip(xs, first)) * 2:
        x.copy_(other)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


# ---------------------------------------------------------------------------------------------------------------------------------------------


def act(name, v):
    if name == "silu":
        return v / (1 + np.exp(-v))
    return np.array([0.5 * a * (1 + math.erf(a / math.sqrt(2))) for a in v.ravel()]).reshape(v.shape)


class Layer:
    def __init__(self, rng, experts, top_k, d, f, group=32, zeros=True, scales="f32", router="f32", bias=None, score="softmax", renormalize=True, factor=1.0,
                 activation="silu", pad=0):
        self.gate, self.up = (Weights(rng, (experts,), f, d, group, zeros, scales, pad) for _ in range(2))
        self.down = Weights(rng, (experts,), d, f, group, zeros, scales, pad)
        self.router, r = rounded(rng.standard_normal((experts, d)) / math.sqrt(d), router)
        self.bias = bias
        self.score, self.renormalize, self.factor, self.activation, self.top_k = score, renormalize, factor, activation, top_k
        self.gpu = oz.MoeLayer(r, self.gate.gpu, self.up.gpu, self.down.gpu, top_k, bias=None if bias is None else torch.tensor(bias, dtype=torch.float32).cuda(),
                               score=score, renormalize=renormalize, factor=factor, activation=activation)

    def choose(self, x, active=None):
        """ids, weights, and how far apart the keys of neighbours in the order are (an infinity where only one is finite)"""
        logits = x @ self.router.T
        p = np.exp(logits - logits.max(axis=1, keepdims=True))
        p = p / p.sum(axis=1, keepdims=True) if self.score == "softmax" else 1 / (1 + np.exp(-logits))
        key = p if self.bias is None else p + self.bias
        order = np.argsort(-key, axis=1, kind="stable")
        ranked = np.take_along_axis(key, order, axis=1)[:, :self.top_k + 1]
        with np.errstate(invalid="ignore"):
            gap = np.abs(np.diff(ranked, axis=1)) if ranked.shape[1] > 1 else np.full((len(x), 1), np.inf)
        ids = order[:, :self.top_k]
        there = np.take_along_axis(key, ids, axis=1) > -np.inf
        if active is not None:
            there &= active[:, None].astype(bool)
        weights = np.where(there, np.take_along_axis(p, ids, axis=1), 0)
        if self.renormalize:
            total = weights.sum(axis=1, keepdims=True)
            weights = np.where(total == 0, 0, weights / np.where(total == 0, 1, total))
        return np.where(there, ids, -1), weights * self.factor, np.nanmin(np.where(np.isnan(gap), np.inf, gap))

    def logit_slack(self, x):
        return U * (x.shape[1] / 8 + 16) * (np.abs(x) @ np.abs(self.router).T).max()

    def __call__(self, x, ids, weights):
        """y and how far off it may be before its rounding"""
        y, off = np.zeros((len(x), self.down.w.shape[1])), np.zeros((len(x), self.down.w.shape[1]))
        relative = 4 * self.logit_slack(x) + 40 * U     # of a weight: two logits or their exponentials off, and a few roundings
        for i, j in zip(*np.where(ids >= 0)):
            e, a = ids[i, j], np.abs(x[i])
            g, u = self.gate.w[e] @ x[i], self.up.w[e] @ x[i]
            dg, du = (m.depth * U * (m.size[e] @ a) for m in (self.gate, self.up))
            h = act(self.activation, g) * u
            dh = 1.13 * dg * (np.abs(u) + du) + (np.abs(act(self.activation, g)) + 1.13 * dg) * du + 32 * U * (np.abs(h) + np.abs(u) * np.abs(g))
            one = self.down.w[e] @ h
            done = np.abs(self.down.w[e]) @ dh + self.down.depth * U * (self.down.size[e] @ (np.abs(h) + dh))
            y[i] += weights[i, j] * one
            off[i] += abs(weights[i, j]) * (done + (relative + 40 * U) * (np.abs(one) + done))
        return y, off


def tokens(rng, layer, t, x_type):
    """tokens whose chosen experts no rounding can change"""
    while True:
        x, gx = rounded(rng.standard_normal((t, layer.router.shape[1])), x_type)
        if layer.choose(x)[2] > 4 * layer.logit_slack(x) + 100 * U:
            return x, gx


def call(layer, gx, y_type="f32", active=None, ctx=None):
    ctx = ctx or oz.Context()
    ctx.allocate_moe_workspace(layer.gpu, max(1, gx.shape[0]))
    t, d = gx.shape
    out = (torch.full((t, d), float("nan"), dtype=TYPES[y_type], device="cuda"), torch.full((t, layer.top_k), 7, dtype=torch.int32, device="cuda"),
           torch.full((t, layer.top_k), float("nan"), device="cuda"))
    return ctx.w4_moe(layer.gpu, gx, active=active, out=out[0], ids=out[1], weights=out[2])


def check(layer, x, got, y_type="f32", active=None):
    y, ids, weights = got
    want_ids, want_weights, _ = layer.choose(x, active)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    relative = 4 * layer.logit_slack(x) + 40 * U
    assert np.all(np.abs(weights.double().cpu().numpy() - want_weights) <= relative * np.abs(want_weights))
    want, off = layer(x, want_ids, want_weights)
    close(y, want, off, y_type)


MOE = [  # t, experts, top_k, d, f, group, x, result, more
    (1, 1, 1, 1, 1, 32, "f32", "f32", {}),
    (1, 4, 2, 64, 32, 32, "bf16", "f32", {}),
    (1, 8, 2, 256, 128, 128, "bf16", "bf16", dict(zeros=False, scales="bf16")),
    (2, 8, 8, 100, 60, 32, "f32", "f32", dict(renormalize=False)),
    (3, 9, 3, 130, 77, 64, "f16", "f32", dict(score="sigmoid", factor=2.5)),
    (5, 16, 4, 300, 129, 128, "f32", "f32", dict(activation="gelu")),
    (16, 60, 6, 128, 96, 32, "bf16", "f32", dict(score="sigmoid", renormalize=False)),
    (17, 5, 2, 96, 200, 64, "f16", "f16", {}),
    (40, 3, 2, 260, 130, 128, "f32", "f32", dict(zeros=False)),
    (70, 2, 1, 64, 64, 32, "bf16", "f32", {}),
    (33, 130, 9, 70, 33, 32, "f32", "f32", dict(score="sigmoid")),
    (4, 300, 32, 64, 48, 32, "f32", "f32", dict(score="sigmoid")),
    (2, 6, 2, 1030, 1500, 128, "bf16", "f32", {}),
    (1, 3, 1, 2500, 300, 1024, "f32", "f32", dict(activation="gelu")),
]


MOE += [  # loads from below a half to many tokens an expert, one span and several, chunks of x that LDS holds in pieces
    (8, 64, 2, 1400, 1100, 64, "f16", "f32", dict(scales="f16", zeros=False)),
    (4, 32, 4, 2100, 700, 32, "bf16", "f32", {}),
    (9, 9, 1, 1100, 2200, 128, "f32", "f32", dict(zeros=False)),
    (12, 8, 2, 640, 512, 32, "bf16", "f32", dict(scales="bf16", zeros=False)),
    (31, 4, 3, 1030, 520, 64, "f32", "f32", {}),
    (32, 4, 4, 4200, 300, 128, "bf16", "f32", dict(scales="bf16")),
    (24, 3, 2, 300, 4100, 128, "f16", "f32", {}),
    (35, 2, 2, 3000, 96, 32, "f32", "f32", dict(activation="gelu")),
    (1, 5, 2, 33, 8192, 32, "bf16", "f32", {}),
    (2, 4, 2, 8200, 40, 128, "bf16", "f32", {}),
    (3, 4, 3, 31, 100, 32, "f32", "f32", {}),
    (3, 4, 3, 100, 31, 32, "f32", "f32", {}),
    (3, 13, 2, 5555, 100, 32, "f32", "f32", {}),
    (2, 5, 1, 4101, 1030, 64, "bf16", "f32", dict(scales="bf16", zeros=False)),
    (1, 3, 3, 8192, 1030, 128, "f16", "f32", {}),
]


@pytest.mark.parametrize("case", MOE, ids=lambda c: "-".join(map(str, c[:8])) + "-".join(c[8]))
def test_moe(case):
    t, experts, top_k, d, f, group, x_type, y_type, more = case
    rng = np.random.default_rng(t + experts + d)
    print(case, flush=True)
    layer = Layer(rng, experts, top_k, d, f, group, **more)
    x, gx = tokens(rng, layer, t, x_type)
    check(layer, x, call(layer, gx, y_type), y_type)


def test_moe_with_all_tokens_on_one_expert():
    """more tokens of one expert than a tile of them holds"""
    rng = np.random.default_rng(21)
    layer = Layer(rng, 8, 2, 64, 80, bias=[0, 0, 9.0, 0, 0, 5.0, 0, 0])
    x, gx = tokens(rng, layer, 50, "f32")
    got = call(layer, gx)
    assert bool((got[1] == torch.tensor([2, 5], dtype=torch.int32, device="cuda")).all())
    check(layer, x, got)


@pytest.mark.parametrize("who", ["none", "all", "some", "one"])
def test_moe_leaves_out_tokens_that_are_not_active(who):
    rng = np.random.default_rng(22)
    layer = Layer(rng, 10, 3, 96, 64)
    x, gx = tokens(rng, layer, 9, "f32")
    active = {"none": np.zeros(9), "all": np.ones(9), "some": np.arange(9) % 3 == 0, "one": np.arange(9) == 8}[who].astype(np.uint8)
    dirty = gx.clone()
    dirty[torch.from_numpy(active == 0).cuda()] = float("nan")     # what a padded place holds is nobody's business
    for kind in (torch.uint8, torch.bool):
        got = call(layer, dirty, active=torch.from_numpy(active).to(kind).cuda())
        check(layer, x, got, active=active)
        off = torch.from_numpy(active == 0).cuda()
        assert bool((got[0][off] == 0).all()) and bool((got[1][off] == -1).all()) and bool((got[2][off] == 0).all())


def test_moe_breaks_ties_by_the_lower_index():
    """small whole numbers: logits are exact, and many are equal"""
    rng = np.random.default_rng(23)
    for experts, top_k in [(7, 3), (64, 8), (130, 20), (700, 32)]:
        layer = Layer(rng, experts, top_k, 32, 32, score="sigmoid")
        whole = rng.integers(-1, 2, (experts, 32)).astype(np.float64)
        layer.router = whole
        layer.gpu.router.copy_(torch.from_numpy(whole))
        x, gx = rounded(rng.integers(-1, 2, (6, 32)).astype(np.float64), "f32")
        logits = x @ whole.T
        order = np.argsort(-logits, axis=1, kind="stable")[:, :top_k]
        got = call(layer, gx)
        # scores of different logits may round to the same value far out: only while they are apart
        assert np.abs(np.take_along_axis(logits, order, 1)).max() < 15
        assert np.array_equal(got[1].cpu().numpy(), order)


def test_moe_with_barred_experts():
    """a bias of -infinity bars an expert; a token may find fewer than top_k, or none"""
    rng = np.random.default_rng(24)
    for left in (5, 3, 1, 0):
        bias = [0.0 if e < left else -math.inf for e in range(12)]
        for renormalize in (False, True):
            layer = Layer(rng, 12, 3, 64, 48, bias=bias, renormalize=renormalize)
            x, gx = tokens(rng, layer, 4, "f32")
            got = call(layer, gx)
            check(layer, x, got)
            assert int((got[1] >= 0).sum()) == 4 * min(3, left)


def test_moe_with_scores_of_zero_and_nans():
    """scores that underflow are chosen in order and weigh nothing; a NaN in a token reaches its result and no other's"""
    rng = np.random.default_rng(25)
    layer = Layer(rng, 6, 3, 64, 48, score="softmax")
    r = np.zeros((6, 64))
    r[:, 0] = [0, 1000, 0, 0, 0, 0]
    layer.gpu.router.copy_(torch.from_numpy(r))
    layer.router = r
    x, gx = rounded(np.eye(64)[:2] * 2, "f32")
    got = call(layer, gx)
    assert got[1].cpu().tolist() == [[1, 0, 2], [0, 1, 2]] and got[2][0].cpu().tolist() == [1.0, 0.0, 0.0]
    layer = Layer(rng, 6, 3, 64, 48)
    x, gx = tokens(rng, layer, 5, "f32")
    clean = call(layer, gx)
    gx[3, 10] = float("nan")
    got = call(layer, gx)
    assert bool(got[0][3].isnan().all())
    keep = [0, 1, 2, 4]
    assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[1][keep], clean[1][keep])
    sigmoid = Layer(rng, 4, 2, 64, 48, score="sigmoid")
    r = np.zeros((4, 64))
    r[:, 0] = -1000
    sigmoid.gpu.router.copy_(torch.from_numpy(r))
    got = call(sigmoid, rounded(np.eye(64)[:1], "f32")[1])
    assert got[2].cpu().tolist() == [[0.0, 0.0]] and bool((got[0] == 0).all())


def test_moe_tokens_do_not_touch_each_other():
    """an infinity in one token, however many share its experts, changes no bit of the others' results"""
    rng = np.random.default_rng(35)
    for t, experts, top_k, d, f in [(5, 40, 2, 130, 90), (6, 4, 2, 300, 200), (30, 3, 2, 260, 150)]:
        layer = Layer(rng, experts, top_k, d, f)
        x, gx = tokens(rng, layer, t, "f32")
        clean = [v.clone() for v in call(layer, gx)]
        gx[2, 5] = float("inf")
        got = call(layer, gx)
        keep = [i for i in range(t) if i != 2]
        assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, clean)) and not bool(got[0][2].isfinite().any())


def test_moe_with_gaps_and_another_stream_and_small_pieces():
    rng = np.random.default_rng(26)
    layer = Layer(rng, 7, 2, 101, 45, group=32, pad=3)
    x, gx = tokens(rng, layer, 6, "bf16")
    wide = torch.full((6, 110), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 4:105] = gx
    out = torch.full((6, 120), 3.0, device="cuda")
    ctx = oz.Context()
    ctx.allocate_moe_workspace(layer.gpu, 6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, ids, weights = ctx.w4_moe(layer.gpu, wide[:, 4:105], out=out[:, 2:103], stream=side)
    side.synchronize()
    check(layer, x, (y, ids, weights))
    assert bool((out[:, :2] == 3).all()) and bool((out[:, 103:] == 3).all())
    # the plain call in the process-wide workspace, results that are not asked for left out
    need = oz.w4_moe_workspace_bytes(layer.gpu, 6)
    buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    oz.set_workspace(buf.data_ptr() + -buf.data_ptr() % 256, need)
    try:
        plain = torch.empty((6, 101), device="cuda")
        rc = oz.lib().oz2_w4_moe(layer.gpu.ref, 6, oz.OZ2_BF16, wide.data_ptr() + 8, 110, None, oz.OZ2_F32, plain.data_ptr(), 101, None, None,
                                 torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    finally:
        oz.set_workspace(None, 0)
    assert rc == 0 and torch.equal(plain, y.contiguous())


def test_moe_repeats_bit_for_bit_and_in_a_graph():
    """one context, its workspace full of garbage first: calls of different sizes in turn, and replays between eager work"""
    rng = np.random.default_rng(27)
    layer = Layer(rng, 20, 4, 300, 260, group=128, scales="bf16")
    ctx = oz.Context()
    ctx.allocate_moe_workspace(layer.gpu, 24)
    ctx.buf.fill_(255)
    xs = [rounded(rng.standard_normal((24, 300)), "bf16")[1] for _ in range(3)]
    first = [[v.clone() for v in ctx.w4_moe(layer.gpu, x)] for x in xs]
    small = [v.clone() for v in ctx.w4_moe(layer.gpu, xs[0][:1])]
    for x, want in zip(xs, first):
        assert all(torch.equal(a, b) for a, b in zip(ctx.w4_moe(layer.gpu, x), want))
        assert all(torch.equal(a, b) for a, b in zip(ctx.w4_moe(layer.gpu, xs[0][:1]), small))
    x = xs[0].clone()
    out = [torch.empty_like(v) for v in first[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.w4_moe(layer.gpu, x, out=out[0], ids=out[1], weights=out[2])
    for other, want in list(zip(xs, first)) * 2:
        x.copy_(other)
        for v in out:
            v.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_moe_with_experts_beyond_32_bits_of_offset():
    rng = np.random.default_rng(28)
    layer = Layer(rng, 3, 3, 64, 40)
    x, gx = tokens(rng, layer, 2, "f32")
    stacks = []
    for w in (layer.gate, layer.up, layer.down):
        n, width = w.codes.shape[1:]
        big = torch.empty(2 * ((1 << 32) + 64) + n * width, dtype=torch.uint8, device="cuda")
        codes = big.as_strided((3, n, width), ((1 << 32) + 64, width, 1))
        codes.copy_(torch.from_numpy(w.codes))
        stacks.append(oz.W4Matrix(codes, w.gpu.scales, w.gpu.zeros, k=w.k, group=w.group))
    layer.gpu = oz.MoeLayer(layer.gpu.router, *stacks, 3)
    check(layer, x, call(layer, gx))
