"""How far attention over a cache held in 4 bits may be from its formula where results are FP32, and that the bound tells a kernel with one term fewer from a right one (on the CPU).

Scores are s sum q c + o sum q in FP32, or with c - 7.5 and o + 7.5 s for FP32 queries: sums of terms up to twice those of q (s c + o), of which the matrix cores cut off what
FP32 does not hold instead of rounding it, twice the error of a plain evaluation again.  So errors are up to 4 times those of the formula in FP32 (root of mean squares over
the elements of a call), and beside these p s is rounded to two bf16, with FP32 queries to three: by at most 2^-16 or 2^-24 of it, which is below r = 2^-17 or 2^-25 in the root
of mean squares, each place's by itself: r sqrt(sum (p s c)^2).
Weights of places have the first part alone.  Queries are chosen that their last bf16 term counts: as large as it can be, with the sign of the value, and some keys
have large codes where it is positive and small ones where not.  Or queries and keys are small whole numbers, whose scores are exact: what is left are the
terms of p s."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TERMS = {"f32": 3, "bf16": 1, "f16": 2}
P_TERMS = {"f32": 3, "bf16": 2, "f16": 2}
SHAPES = [(40, 64), (40, 128), (700, 128), (300, 96), (90, 40), (120, 256), (1500, 64)]  # places, dim


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).bfloat16().float().numpy()


def terms(x, n):
    """x as a sum of n bf16, as near as it goes"""
    out, left = [], np.asarray(x, dtype=np.float32)
    for _ in range(n):
        out.append(bf16(left))
        left = left - out[-1]
    return out, left


class Case:
    """rows of queries (rows, dim), codes (n, dim), scales and offsets (n) of keys and values"""

    def __init__(self, rng, n, dim, name, whole=False, rows=24):
        x = rng.uniform(0.6, 1.9, (rows, dim)) * rng.choice([-1.0, 1.0], dim)
        near = x[..., None] * (1 + rng.uniform(-0.01, 0.01, (rows, dim, 64)))
        near = torch.from_numpy(near).to(TYPES[name]).float().numpy()
        left = terms(near, max(TERMS[name] - 1, 1))[1] * np.sign(near)
        self.q = np.take_along_axis(near, left.argmax(2)[..., None], 2)[..., 0]
        codes = lambda: rng.integers(0, 16, (n, dim))
        self.kc, self.vc = codes(), codes()
        aligned = rng.choice(n, 3, replace=False)
        self.kc[aligned] = np.where(self.q[0] > 0, rng.integers(12, 16, (3, dim)), rng.integers(0, 4, (3, dim)))
        self.ks, self.vs = (rng.uniform(0.2, 0.4, n).astype(np.float16) for _ in "kv")
        self.ko, self.vo = ((-7.5 * s.astype(np.float64) * rng.uniform(0.9, 1.1, n)).astype(np.float16) for s in (self.ks, self.vs))
        gain = 5.5 * 0.3 * np.abs(self.q).sum(1).mean()  # (score of an aligned key)
        self.scale = float(np.float32((np.log(n / 3) + 0.3) / gain))
        if whole:
            self.q = rng.integers(-2, 3, (rows, dim)).astype(np.float32)
            self.ks[:], self.ko[:], self.scale = 0.25, rng.integers(-10, -4, n) / 4, 2.0 ** -4

    def formula(self, kind):
        """out, received of a row, p, in a floating type of NumPy"""
        k, v = (c.astype(kind) * s.astype(kind)[:, None] + o.astype(kind)[:, None] for c, s, o in ((self.kc, self.ks, self.ko), (self.vc, self.vs, self.vo)))
        x = (self.q.astype(kind) @ k.T) * kind(self.scale)
        p = np.exp(x - x.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        return p @ v, p


def rms(x):
    return float(np.sqrt(np.mean(np.square(np.asarray(x, dtype=np.float64)))))


def bounds(case, name):
    """out and p in 64 bits, and what the roots of mean squares of their errors may be"""
    out, p = case.formula(np.float64)
    out32, p32 = case.formula(np.float32)
    r = 2.0 ** -25 if name == "f32" else 2.0 ** -17
    rounded = r * np.sqrt(np.square(p) @ np.square(case.vs.astype(np.float64)[:, None] * case.vc))
    return out, p, 4 * rms(out32 - out) + rms(rounded), 4 * rms(p32 - p)


def model(case, name, q_terms, p_terms):
    """the kernel's arithmetic, with sums in FP32"""
    f = np.float32
    centred = name == "f32"
    kc, vc = (c.astype(f) - f(7.5 if centred else 0) for c in (case.kc, case.vc))
    ko, vo = (o.astype(f) + f(7.5 if centred else 0) * s.astype(f) for o, s in ((case.ko, case.ks), (case.vo, case.vs)))
    total = case.q.astype(f).sum(1, dtype=f)
    x = sum((t @ kc.T for t in terms(case.q, q_terms)[0]), f(0)) * case.ks.astype(f) + total[:, None] * ko
    x = x * f(f(case.scale) * f(1.4426950408889634))
    p = np.exp2(x - x.max(1, keepdims=True))
    w = terms(p * case.vs.astype(f), p_terms)[0]
    out = sum((t @ vc for t in w), f(0)) + (p @ vo)[:, None]
    total = p.sum(1, dtype=f, keepdims=True)
    return out / total, p / total


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("whole", [False, True], ids=["", "whole"])
def test_the_bound_tells_terms_that_are_missing(whole, name, shape):
    case = Case(np.random.default_rng(sum(shape)), *shape, name, whole)
    out, p, of_out, of_p = bounds(case, name)
    got = model(case, name, TERMS[name], P_TERMS[name])
    assert rms(got[0] - out) <= of_out and rms(got[1] - p) <= of_p
    if whole or name != "f32":
        assert rms(model(case, name, TERMS[name], P_TERMS[name] - 1)[0] - out) > 1.25 * of_out
    if TERMS[name] > 1 and not whole:
        fewer = model(case, name, TERMS[name] - 1, P_TERMS[name])
        assert rms(fewer[0] - out) > 1.25 * of_out and rms(fewer[1] - p) > 1.25 * of_p
    assert rms(out) > 100 * of_out  # (zeros are no result)
