"""Caches of keys and values held in 4 bits: appending, attention, evicting, against their formulas in 64 bits.

Tolerances of attention (u = 2^-24) allow for sums of (16 + c) q with c the codes, of which 16 sum q is taken off again: with B = sum |q| the score's error is at most
e = (dim + 48) u scale max (s 47 B + |o| B), and p is off by a factor within 1 +- (2 e + 8 u).  p s is rounded to two bf16 terms, by 2^-16 of it (three for FP32: 2^-24), and
meets 16 + c likewise: with A = sum p (47 s + |o|) a result is off by at most (2 e + r + (n + 72) u) (A + |out|), r = 2^-16 or 2^-24, times 2
for what is of second order, before the one rounding to its type.  What a place received is a sum of p: off by at most (2 e + (n + 72) u) of it and u of the weight."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


class Held:
    """a cache with random contents, and sequences on it in pages of random order"""

    def __init__(self, rng, lengths, kv_heads, dim, page, spare=0, places=0):
        self.lengths, self.page, self.dim, self.heads = list(lengths), page, dim, kv_heads
        of = [-(-n // page) for n in lengths]
        self.max_pages = max(max(of) + spare, 1)
        self.pages = sum(of) + 2
        order = rng.permutation(self.pages)
        self.table = np.full((len(lengths), self.max_pages), -1, dtype=np.int32)
        begin = 0
        for s, n in enumerate(of):
            self.table[s, :n] = order[begin : begin + n]
            begin += n
        make = lambda last, low, high: rng.uniform(low, high, (self.pages, kv_heads, page, last))
        self.codes = {n: torch.from_numpy(rng.integers(0, 256, (self.pages, kv_heads, page, dim // 2), dtype=np.uint8)) for n in "kv"}
        self.scales = {n: torch.from_numpy(np.concatenate((make(1, 0.1, 0.4), make(1, -3.0, 1.0)), axis=3)).half() for n in "kv"}
        self.capacity = self.max_pages * page
        shape = (len(lengths), kv_heads, self.capacity + places)
        self.weights = torch.from_numpy(rng.exponential(size=shape)).float()
        self.positions = torch.arange(shape[2], dtype=torch.int32).expand(shape).contiguous()
        self.cache = oz.KV4Cache(self.codes["k"].cuda(), self.scales["k"].cuda(), self.codes["v"].cuda(), self.scales["v"].cuda())
        self.gpu_table, self.gpu_lengths = ints(self.table), ints(lengths)

    def row(self, name, s, h):
        """values, scales and offsets of the places of a sequence and head, and which have no page"""
        n = self.lengths[s]
        t = np.arange(n)
        page = self.table[s, t // self.page]
        bad = (page < 0) | (page >= self.pages)
        page = np.where(bad, 0, page)
        codes = self.codes[name].numpy()[page, h, t % self.page]
        scales = self.scales[name].double().numpy()[page, h, t % self.page]
        c = np.stack((codes & 15, codes >> 4), axis=2).reshape(n, self.dim).astype(np.float64)
        return c * scales[:, :1] + scales[:, 1:], scales[:, 0], scales[:, 1], bad


def formula(held, q, cu, scale):
    """out, A, e / ((dim + 48) u), keys, and what places received with its bound"""
    tokens, heads, dim = q.shape
    group = heads // held.heads
    out, size, most, keys = np.zeros(q.shape), np.zeros(q.shape), np.zeros((tokens, heads, 1)), np.ones((tokens, 1, 1))
    received, error = np.zeros(held.weights.shape), np.zeros(held.weights.shape)
    with np.errstate(all="ignore"):
        for s in range(len(held.lengths)):
            a, b = cu[s], cu[s + 1]
            for h in range(held.heads):
                k, ks, ko, bad = held.row("k", s, h)
                v, vs, vo, _ = held.row("v", s, h)
                for i in range(a, b):
                    n = held.lengths[s] - (b - a) + (i - a) + 1
                    seen = np.flatnonzero(~bad[: max(n, 0)])
                    for g in range(h * group, (h + 1) * group):
                        if not len(seen):
                            continue
                        x = scale * (k[seen] @ q[i, g])
                        p = np.exp(x - x.max())
                        p /= p.sum()
                        out[i, g] = p @ v[seen]
                        size[i, g] = p @ (47 * np.abs(vs) + np.abs(vo))[seen]
                        most[i, g] = scale * ((47 * np.abs(ks) + np.abs(ko))[seen]).max() * np.abs(q[i, g]).sum()
                        keys[i] = n
                        received[s, h, seen] += p
                        error[s, h, seen] += p * (2 * (held.dim + 48) * U * most[i, g] + (n + 72) * U)
    return out, size, most, keys, received, error


def close(got, want, name, dim, rows=slice(None)):
    out, size, most, keys = (w[rows] for w in want[:4])
    got = got.double().cpu().numpy()[rows]
    r = U if name == "f32" else 2.0 ** -16
    slack = 2 * (2 * (dim + 48) * U * most + r + (keys + 72) * U) * (size + np.abs(out))
    tol = slack + HALF[name] * (np.abs(out) + slack) + LEAST[name]
    bad = ~(np.abs(got - out) <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g times the tolerance" % (bad.sum(), bad.size, np.nanmax(np.abs(got - out) / tol))


def check(lengths, news, heads, kv_heads, dim, page, name, weights=False, seed=0, size=1.0, behind=2, change=None, spare=1):
    rng = np.random.default_rng(seed)
    held = Held(rng, lengths, kv_heads, dim, page, spare=spare)
    if change:
        change(held)
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]) + behind, heads, dim)) * size).to(TYPES[name])
    want = formula(held, q.double().numpy(), cu, dim ** -0.5)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=q.shape[0], heads=heads, weights=weights)
    out, received = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), held.weights.cuda() if weights else None
    assert ctx.kv4_attention(held.cache, q.cuda(), ints(cu), held.gpu_table, held.gpu_lengths, weights=received, out=out) is out
    close(out, want, name, dim, slice(0, int(cu[-1])))
    assert (out[cu[-1] :] == 7.0).all()
    if weights:
        before = held.weights.double().numpy()
        off = np.abs(received.double().cpu().numpy() - (before + want[4]))
        assert (off <= 2 * want[5] + 2 * U * (before + want[4])).all()


SHAPES = [  # lengths, new tokens, heads, kv heads, dim, page
    ([1], [1], 1, 1, 64, 16), ([1], [1], 8, 1, 128, 32), ([16], [1], 4, 2, 128, 16), ([17, 33], [1, 1], 8, 2, 64, 16), ([31], [1], 2, 2, 256, 64),
    ([100, 1, 250], [1, 1, 1], 8, 2, 128, 48), ([129, 128, 127], [1, 1, 1], 8, 8, 128, 64), ([500], [1], 16, 1, 128, 16), ([300], [5], 6, 3, 96, 16),
    ([64, 90], [3, 8], 12, 3, 80, 32), ([777], [2], 8, 1, 64, 128), ([40], [40], 4, 2, 128, 16), ([50, 20], [17, 3], 9, 3, 128, 16), ([1000, 30], [1, 4], 4, 4, 8, 16),
    ([70], [1], 2, 1, 40, 16), ([200], [2], 4, 1, 136, 32), ([90], [1], 4, 1, 248, 32), ([2, 1], [1, 1], 64, 2, 120, 16), ([1500, 700], [1, 1], 32, 8, 128, 64),
]


@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(shape, name, weights):
    check(*shape, name, weights, seed=len(str(shape)))


@pytest.mark.parametrize("name", TYPES)
def test_sequences_without_places_or_tokens(name):
    """nothing held, no new token, more new tokens than places: rows that see nothing are 0"""
    check([0, 40, 0, 3, 20], [1, 1, 0, 5, 0], 4, 2, 64, 16, name, True)
    check([0], [1], 4, 2, 128, 16, name, True, spare=0)


@pytest.mark.parametrize("name", TYPES)
def test_peaked_scores(name):
    check([400, 90], [1, 2], 8, 2, 128, 16, name, True, size=6.0, seed=3)


def test_pages_that_are_none():
    """numbers outside the cache: nobody sees their places"""
    def change(held):
        held.table[0, 2], held.table[0, 5], held.table[1, 0] = -7, held.pages, 2 ** 31 - 1
        held.gpu_table = ints(held.table)
    check([150, 16], [2, 1], 4, 2, 64, 16, "bf16", True, change=change)


def test_lengths_that_lie_are_cut_off():
    rng = np.random.default_rng(1)
    held = Held(rng, [100, 50], 2, 64, 16, spare=0)
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).bfloat16()
    held.lengths = [held.capacity, 0]
    held.table[0], held.table[1, :] = held.table[0], -1
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=2, heads=4)
    out = ctx.kv4_attention(held.cache, q.cuda(), ints([0, 1, 2]), held.gpu_table, ints([10 ** 9, -5]))
    close(out, formula(held, q.double().numpy(), [0, 1, 2], 64 ** -0.5), "bf16", 64)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_what_a_token_does_not_see_does_not_reach_it(what, name):
    """scales that are not finite: behind the last place, and of a later new token"""
    rng = np.random.default_rng(2)
    held = Held(rng, [60, 45], 2, 128, 16)
    q = torch.from_numpy(rng.standard_normal((5, 4, 128))).to(TYPES[name])
    cu = [0, 3, 5]
    for s, t in ((0, 60), (0, 61), (1, 45), (1, 47), (0, 59), (1, 44)):  # (the last two: seen by the last new token alone)
        for n in "kv":
            held.scales[n][held.table[s, t // 16], :, t % 16, 0] = what
    cache = oz.KV4Cache(held.codes["k"].cuda(), held.scales["k"].cuda(), held.codes["v"].cuda(), held.scales["v"].cuda())
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, held.gpu_table, tokens=5, heads=4)
    out = ctx.kv4_attention(cache, q.cuda(), ints(cu), held.gpu_table, held.gpu_lengths)
    rows = [0, 1, 3]
    close(out, formula(held, q.double().numpy(), cu, 128 ** -0.5), name, 128, rows)
    assert not torch.isfinite(out[[2, 4]]).any()


@pytest.mark.parametrize("dim", [64, 128, 200])
def test_strides(dim):
    """every second layer of one cache, queries from a packed tensor that starts anywhere, a part of a table"""
    rng = np.random.default_rng(3)
    held = Held(rng, [90, 33], 2, dim, 16)
    codes = torch.randint(0, 256, (held.pages, 3, 2, 2, 16, dim // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((held.pages, 3, 2, 2, 16, 2), math.nan, dtype=torch.float16, device="cuda")
    for i, n in enumerate("kv"):
        codes[:, 1, i], scales[:, 1, i] = held.codes[n].cuda(), held.scales[n].cuda()
    cache = oz.KV4Cache(codes[:, 1, 0], scales[:, 1, 0], codes[:, 1, 1], scales[:, 1, 1])
    packed = torch.full((3, 4 * dim + 5), math.nan, dtype=torch.float16, device="cuda")
    q = torch.from_numpy(rng.standard_normal((3, 4, dim))).half()
    view = packed[:, 3 : 3 + 4 * dim].unflatten(1, (4, dim))
    view.copy_(q)
    table = torch.full((2, 40), -1, dtype=torch.int32, device="cuda")
    table[:, : held.max_pages] = held.gpu_table
    part, cu = table[:, : held.max_pages], [0, 2, 3]
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, part, tokens=3, heads=4)
    out = torch.empty((4, 3, dim), device="cuda").transpose(0, 1)
    ctx.kv4_attention(cache, view, ints(cu), part, held.gpu_lengths, out=out)
    close(out, formula(held, q.double().numpy(), cu, dim ** -0.5), "f16", dim)


def test_long_sequences():
    """20000 places of one sequence beside short ones, cut into chunks that come together"""
    rng = np.random.default_rng(4)
    held = Held(rng, [20000, 3, 1200], 1, 64, 64)
    q = torch.from_numpy(rng.standard_normal((4, 4, 64))).bfloat16()
    cu = [0, 2, 3, 4]
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=4, heads=4, weights=True)
    received = held.weights.cuda()
    out = ctx.kv4_attention(held.cache, q.cuda(), ints(cu), held.gpu_table, held.gpu_lengths, weights=received)
    want = formula(held, q.double().numpy(), cu, 0.125)
    close(out, want, "bf16", 64)
    off = np.abs(received.double().cpu().numpy() - (held.weights.double().numpy() + want[4]))
    assert (off <= 2 * want[5] + 2 * U * (held.weights.double().numpy() + want[4])).all()


# appending

def appended(x):
    """codes, scales, offsets of x (tokens, heads, dim) in FP32 arithmetic"""
    x = x.float().numpy()
    low, high = x.min(axis=2), x.max(axis=2)
    with np.errstate(all="ignore"):
        s, o = ((high - low) / np.float32(15)).astype(np.float16), low.astype(np.float16)
        c = np.rint((x - o.astype(np.float32)[..., None]) * (np.float32(1) / s.astype(np.float32))[..., None])
    c = np.where(s[..., None] == 0, 0, np.clip(c, 0, 15)).astype(np.uint8)
    return c, s, o


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("lengths,news,kv_heads,dim,page", [([1], [1], 1, 64, 16), ([30, 17], [1, 1], 2, 128, 16), ([33, 5, 0, 100], [33, 2, 0, 7], 3, 96, 32),
                                                            ([20], [3], 1, 8, 16), ([64, 65], [64, 1], 2, 256, 64), ([3, 9], [5, 2], 2, 40, 16)])
def test_append(lengths, news, kv_heads, dim, page, name):
    rng = np.random.default_rng(dim)
    held = Held(rng, lengths, kv_heads, dim, page)
    cu = np.concatenate([[0], np.cumsum(news)])
    tokens = int(cu[-1]) + 2
    k, v = (torch.from_numpy(rng.standard_normal((tokens, kv_heads, dim)) + 1.0).to(TYPES[name]) for _ in "kv")
    k[0, 0] = 1.5  # (all alike: a scale of 0)
    at = torch.arange(1000, 1000 + tokens, dtype=torch.int32)
    positions, weights = held.positions.cuda(), held.weights.cuda()
    out = tuple(torch.full(k.shape, 7.0, dtype=k.dtype, device="cuda") for _ in "kv")
    oz.kv4_append(held.cache, k.cuda(), v.cuda(), ints(cu), held.gpu_table, held.gpu_lengths, at=at.cuda(), positions=positions, weights=weights, held=out)
    codes, scales = {n: t.clone() for n, t in held.codes.items()}, {n: t.clone() for n, t in held.scales.items()}
    for n, x, back in (("k", k, out[0]), ("v", v, out[1])):
        c, s, o = appended(x)
        for i in range(len(lengths)):
            for j in range(cu[i], cu[i + 1]):
                t = lengths[i] - (cu[i + 1] - j)
                if t < 0:
                    continue
                p = held.table[i, t // page]
                codes[n][p, :, t % page] = torch.from_numpy(c[j, :, 0::2] | c[j, :, 1::2] << 4)
                scales[n][p, :, t % page] = torch.from_numpy(np.stack((s[j], o[j]), axis=1))
                held.positions[i, :, t], held.weights[i, :, t] = at[j], 0.0
        value = c * s.astype(np.float64)[..., None] + o.astype(np.float64)[..., None]
        got = back.double().cpu().numpy()
        assert (np.abs(got - value)[: cu[-1]] <= (HALF[name] * np.abs(value) + 2 * U * np.abs(value) + LEAST[name])[: cu[-1]]).all()
        assert (got[cu[-1] :] == 7.0).all()
    for n, got in (("k", held.cache.k_codes), ("v", held.cache.v_codes)):
        assert torch.equal(got.cpu(), codes[n])
    for n, got in (("k", held.cache.k_scales), ("v", held.cache.v_scales)):
        assert torch.equal(got.cpu().view(torch.int16), scales[n].view(torch.int16))
    assert torch.equal(positions.cpu(), held.positions) and torch.equal(weights.cpu(), held.weights)


@pytest.mark.parametrize("name", TYPES)
def test_append_what_is_not_finite(name):
    """a key with a NaN or an infinity, or values that FP16 does not hold, is held as one that is not finite; its neighbours are not touched"""
    rng = np.random.default_rng(5)
    held = Held(rng, [16], 2, 64, 16)
    k, v = (torch.from_numpy(rng.standard_normal((6, 2, 64))).to(TYPES[name]) for _ in "kv")
    k[0, 0, 5], k[1, 1, 63], v[2, 0, 0] = math.nan, math.inf, -math.inf
    v[3, 1] = torch.linspace(-1, 1, 64).to(v.dtype) * (60000.0 if name == "f16" else 1e30)
    out = torch.empty_like(k, device="cuda"), torch.empty_like(v, device="cuda")
    oz.kv4_append(held.cache, k.cuda(), v.cuda(), ints([0, 6]), held.gpu_table, held.gpu_lengths, held=out)
    finite = [torch.isfinite(t).cpu().numpy() for t in out]
    want = [np.ones((6, 2), bool), np.ones((6, 2), bool)]
    want[0][0, 0] = want[0][1, 1] = want[1][2, 0] = False
    want[1][3, 1] = name == "f16"
    for got, w in zip(finite, want):
        assert (got.all(axis=2) == w).all()


def test_append_in_place_and_from_packed_tensors():
    rng = np.random.default_rng(6)
    held, other = Held(rng, [20], 2, 64, 16), Held(np.random.default_rng(6), [20], 2, 64, 16)
    packed = torch.from_numpy(rng.standard_normal((20, 3 * 2 * 64 + 1))).bfloat16().cuda()
    k, v = (packed[:, 1 + i * 128 : 1 + i * 128 + 128].unflatten(1, (2, 64)) for i in (1, 2))
    rest = packed[:, :129].clone()
    copies = k.contiguous(), v.contiguous()
    out = torch.empty_like(copies[0]), torch.empty_like(copies[1])
    oz.kv4_append(other.cache, *copies, ints([0, 20]), other.gpu_table, other.gpu_lengths, held=out)
    oz.kv4_append(held.cache, k, v, ints([0, 20]), held.gpu_table, held.gpu_lengths, held=(k, v))
    assert torch.equal(k, out[0]) and torch.equal(v, out[1]) and torch.equal(packed[:, :129], rest)
    for n in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert torch.equal(getattr(held.cache, n), getattr(other.cache, n))


def test_append_to_pages_that_are_none():
    rng = np.random.default_rng(7)
    held = Held(rng, [40], 2, 64, 16)
    held.table[0, 1:] = [-1, held.pages, 10 ** 9][: held.max_pages - 1]
    k = torch.ones((40, 2, 64)).cuda()
    oz.kv4_append(held.cache, k, k, ints([0, 40]), ints(held.table), held.gpu_lengths)
    got = held.cache.k_scales.cpu()
    page = held.table[0, 0]
    assert (got[page] == torch.tensor([0.0, 1.0]).half()).all()
    others = [p for p in range(held.pages) if p != page]
    assert torch.equal(got[others], held.scales["k"][others])


# evicting

def evicted(held, keep, recent):
    """lengths, positions, weights, and where each place comes from"""
    lengths, positions, weights = [min(n, keep) for n in held.lengths], held.positions.numpy().copy(), held.weights.numpy().copy()
    moves = {}
    for s, n in enumerate(held.lengths):
        if n <= keep:
            continue
        for h in range(held.heads):
            w, p = held.weights[s, h, :n].numpy().astype(np.float64), held.positions[s, h, :n].numpy().astype(np.int64)
            key = [(2 if p[t] > p.max() - recent else 1 if np.isnan(w[t]) else 0, 0.0 if np.isnan(w[t]) or p[t] > p.max() - recent else w[t], -t) for t in range(n)]
            stay = set(sorted(range(n), key=lambda t: key[t], reverse=True)[:keep])
            holes, movers = [t for t in range(keep) if t not in stay], [t for t in range(keep, n) if t in stay]
            assert len(holes) == len(movers)
            for to, at in zip(holes, movers):
                moves[s, h, to] = at
                positions[s, h, to], weights[s, h, to] = positions[s, h, at], weights[s, h, at]
    return lengths, positions, weights, moves


def check_evict(held, keep, recent, in_place):
    lengths, positions, weights, moves = evicted(held, keep, recent)
    for name in "kv":
        codes, scales = held.codes[name].clone(), held.scales[name].clone()
        for (s, h, to), at in moves.items():
            a, b = held.table[s, to // held.page], held.table[s, at // held.page]
            if 0 <= a < held.pages and 0 <= b < held.pages:
                codes[a, h, to % held.page], scales[a, h, to % held.page] = held.codes[name][b, h, at % held.page], held.scales[name][b, h, at % held.page]
        setattr(held, "want_" + name, (codes, scales))
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, keep=keep)
    gpu = held.gpu_lengths, held.positions.cuda(), held.weights.cuda()
    out = None if in_place else (torch.full_like(gpu[0], -9), torch.full_like(gpu[1], -9), torch.full_like(gpu[2], -9.0))
    got = ctx.kv4_evict(held.cache, held.gpu_table, *gpu, keep, recent=recent, out=out)
    assert all(a is b for a, b in zip(got, gpu if in_place else out))
    assert got[0].tolist() == lengths
    for s, n in enumerate(lengths):
        for g, w, first in ((got[1], positions, held.positions), (got[2], weights, held.weights)):
            g = g[s].cpu().numpy()
            assert np.array_equal(g[:, :n], w[s, :, :n], equal_nan=True)
            assert np.array_equal(g[:, n:], first[s, :, n:].numpy(), equal_nan=True) if in_place else (g[:, n:] == -9).all()
    if not in_place:
        assert gpu[0].tolist() == held.lengths and torch.equal(gpu[1].cpu(), held.positions)
    for name, codes, scales in (("k", held.cache.k_codes, held.cache.k_scales), ("v", held.cache.v_codes, held.cache.v_scales)):
        want = getattr(held, "want_" + name)
        assert torch.equal(codes.cpu(), want[0]) and torch.equal(scales.cpu().view(torch.int16), want[1].view(torch.int16))


@pytest.mark.parametrize("in_place", [False, True], ids=["elsewhere", "in_place"])
@pytest.mark.parametrize("lengths,keep,recent,kv_heads,dim,page", [
    ([1], 0, 0, 1, 64, 16), ([1], 1, 1, 1, 64, 16), ([2], 1, 0, 1, 64, 16), ([17, 16, 5, 0], 16, 4, 2, 64, 16), ([65], 64, 8, 4, 128, 64), ([300, 100], 100, 100, 2, 40, 32),
    ([300, 100], 99, 10, 2, 96, 16), ([1023, 1024, 1025], 512, 33, 1, 8, 48), ([5000, 1], 17, 0, 1, 16, 64), ([5000], 4990, 100, 2, 256, 128), ([40, 50], 100, 3, 2, 64, 16),
    ([4097], 4096, 64, 2, 128, 64), ([9000, 8000], 3000, 50, 1, 8, 16)])
def test_evict(lengths, keep, recent, kv_heads, dim, page, in_place):
    rng = np.random.default_rng(len(lengths) + keep)
    held = Held(rng, lengths, kv_heads, dim, page, places=3)
    for s, n in enumerate(lengths):  # positions in any order, as evictions leave them
        for h in range(kv_heads):
            held.positions[s, h, :n] = torch.from_numpy(rng.permutation(n) + 10 * s).int()
    check_evict(held, keep, recent, in_place)


@pytest.mark.parametrize("weights", ["equal", "two", "zeros", "signs", "nan", "inf", "close", "positions"])
def test_evict_weights_that_are_hard_to_order(weights):
    rng = np.random.default_rng(8)
    held = Held(rng, [700, 200], 2, 64, 16)
    w = held.weights
    if weights == "equal":
        w.fill_(0.25)
    elif weights == "two":
        w.copy_(torch.from_numpy(rng.integers(0, 2, w.shape)).float())
    elif weights == "zeros":
        w.copy_(torch.where(torch.from_numpy(rng.random(w.shape) < 0.5), 0.0, -0.0))
    elif weights == "signs":
        w.copy_(torch.from_numpy(rng.standard_normal(w.shape) * 10.0 ** rng.integers(-40, 38, w.shape)).float())
    elif weights == "nan":
        w[torch.from_numpy(rng.random(w.shape) < 0.3)] = math.nan
        w[torch.from_numpy(rng.random(w.shape) < 0.3)] = -math.nan
    elif weights == "inf":
        w[torch.from_numpy(rng.random(w.shape) < 0.3)] = math.inf
        w[torch.from_numpy(rng.random(w.shape) < 0.3)] = -math.inf
    elif weights == "close":  # the last bits decide
        w.copy_(torch.from_numpy((rng.integers(0, 300, w.shape) + 0x3F800000).astype(np.int32)).view(torch.float32))
    else:
        held.positions.copy_(torch.from_numpy(rng.choice([-2 ** 31, -1, 0, 2 ** 31 - 1], held.positions.shape)).int())
    check_evict(held, 150, 20, False)


def test_evict_with_pages_that_are_none():
    held = Held(np.random.default_rng(9), [200], 2, 64, 16)
    held.table[0, 3], held.table[0, 10] = -1, held.pages
    held.gpu_table = ints(held.table)
    check_evict(held, 100, 10, False)


# together

def test_a_run_of_them_together():
    """prompts read and appended, steps that add weight up, evictions between them, eagerly and in a captured graph; against attention in 64 bits over the values that the
    cache was told to hold, by position"""
    rng = np.random.default_rng(10)
    heads, kv_heads, dim, page, keep = 4, 2, 64, 16, 40
    prompts, steps = [50, 9], 24
    of = 6
    cache = oz.KV4Cache.empty(2 * of, kv_heads, page, dim)
    table = ints(rng.permutation(2 * of).reshape(2, of))
    capacity = of * page
    positions, weights = torch.zeros((2, kv_heads, capacity), dtype=torch.int32, device="cuda"), torch.zeros((2, kv_heads, capacity), device="cuda")
    lengths, seen = ints(prompts), ints(prompts)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, table, tokens=sum(prompts), heads=heads, weights=True, keep=keep)
    make = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, dim))).bfloat16().cuda()
    q, k, v = make(59, heads), make(59, kv_heads), make(59, kv_heads)
    cu = ints([0, 50, 59])
    held = torch.empty_like(k), torch.empty_like(v)
    at = torch.cat([torch.arange(n) for n in prompts]).int().cuda()
    oz.kv4_append(cache, k, v, cu, table, lengths, at=at, positions=positions, weights=weights, held=held)
    # the whole prompt's attention over what is held is the cache's own
    one, two = oz.attention(q, *held, cu).float(), ctx.kv4_attention(cache, q, cu, table, lengths).float()
    assert (one - two).abs().max() <= 2.0 ** -4 * held[1].abs().max().float()
    past = [[(held[0][a:b].clone(), held[1][a:b].clone())] for a, b in ((0, 50), (50, 59))]

    q1, k1, v1, out = make(2, heads), make(2, kv_heads), make(2, kv_heads), torch.empty((2, heads, dim), dtype=torch.bfloat16, device="cuda")
    held1 = torch.empty_like(k1), torch.empty_like(v1)
    cu1 = ints([0, 1, 2])

    def step():
        lengths.add_(1)
        oz.kv4_append(cache, k1, v1, cu1, table, lengths, at=seen, positions=positions, weights=weights, held=held1)
        seen.add_(1)
        ctx.kv4_attention(cache, q1, cu1, table, lengths, weights=weights, out=out)
        before.copy_(lengths)
        standing.copy_(positions)
        ctx.kv4_evict(cache, table, lengths, positions, weights, keep, recent=8)

    before, standing = torch.zeros_like(lengths), torch.zeros_like(positions)
    graph = None
    for i in range(steps):
        for t, n in ((q1, heads), (k1, kv_heads), (v1, kv_heads)):
            t.copy_(make(2, n))
        if i == steps // 2:
            graph = torch.cuda.CUDAGraph()
            state = [t.clone() for t in (lengths, seen)]
            with torch.cuda.graph(graph):
                step()
            assert torch.equal(lengths, state[0]) and torch.equal(seen, state[1])
        if graph:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        for s in range(2):
            past[s].append((held1[0][s : s + 1].clone(), held1[1][s : s + 1].clone()))
            keys, values = (torch.cat([p[j] for p in past[s]]).double().cpu() for j in (0, 1))
            for h in range(kv_heads):
                at = standing[s, h, : before[s]].long().cpu()
                assert len(set(at.tolist())) == len(at) and int(at.max()) == int(seen[s]) - 1
                x = q1[s].double().cpu()[h * 2 : h * 2 + 2] @ keys[at, h].T * dim ** -0.5
                want = torch.softmax(x, 1) @ values[at, h]
                # (held values are rounded to bf16 here, unrounded in the cache: 2^-8 of keys and values, and the result's own rounding)
                assert (out[s].double().cpu()[h * 2 : h * 2 + 2] - want).abs().max() <= 2.0 ** -4 * values.abs().max()
                assert len(set(positions[s, h, : lengths[s]].tolist())) == int(lengths[s])
    assert lengths.tolist() == [keep, 9 + steps]


def test_two_sequences_alike_and_equal_calls_give_equal_bits():
    rng = np.random.default_rng(11)
    held = Held(rng, [900, 900], 2, 128, 64)
    held.table[1] = held.table[0]
    table = ints(held.table)
    q = torch.from_numpy(rng.standard_normal((1, 8, 128))).bfloat16().cuda().repeat(2, 1, 1)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, table, tokens=2, heads=8)
    first = ctx.kv4_attention(held.cache, q, ints([0, 1, 2]), table, held.gpu_lengths)
    assert torch.equal(first[0], first[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = ctx.kv4_attention(held.cache, q, ints([0, 1, 2]), table, held.gpu_lengths, stream=side)
    side.synchronize()
    assert torch.equal(first, again)


def test_the_registered_workspace():
    """kv4_attention and kv4_evict outside a context"""
    rng = np.random.default_rng(12)
    held = Held(rng, [600], 2, 64, 16)
    q = torch.from_numpy(rng.standard_normal((1, 4, 64))).bfloat16()
    need = max(oz.kv4_attention_workspace_bytes(held.cache, held.gpu_table, 1, 4, weights=True), oz.kv4_evict_workspace_bytes(held.cache, held.gpu_table, 100))
    buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    oz.set_workspace(buf.data_ptr() + -buf.data_ptr() % 256, need)
    try:
        weights = held.weights.cuda()
        out = oz.kv4_attention(held.cache, q.cuda(), ints([0, 1]), held.gpu_table, held.gpu_lengths, weights=weights)
        close(out, formula(held, q.double().numpy(), [0, 1], 0.125), "bf16", 64)
        assert oz.kv4_evict(held.cache, held.gpu_table, held.gpu_lengths, held.positions.cuda(), weights, 100)[0].tolist() == [100]
        oz.set_workspace(buf.data_ptr() + -buf.data_ptr() % 256, 256)
        with pytest.raises(oz.Oz2Error, match="workspace"):
            oz.kv4_attention(held.cache, q.cuda(), ints([0, 1]), held.gpu_table, ints([600]))
    finally:
        oz.set_workspace(None, 0)
