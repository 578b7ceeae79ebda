"""Attention over packed prompts where one key takes the maximum and thousands lie far below it: what they weigh together counts.

The sink's value is 0, so the result is the others' part alone.  Formula and tolerances: test_gpu_attention; in FP16 p is off by half a step, 2^-11 of it, or, below its normal
range, by 2^-25 where the largest p is 2^7 or more: 2^-32 of that for each of n keys."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_attention import HALF, LEAST, TYPES, U
from test_gpu_kv4 import ints


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim,heads", [(64, 1), (128, 1), (128, 16), (200, 1), (64, 20)])
@pytest.mark.parametrize("first", [True, False], ids=["first", "last"])
def test_many_keys_far_below_one(first, dim, heads, name):
    rng = np.random.default_rng(dim)
    for n in (700, 3500, 20000) if name != "f32" and heads == 1 else (700, 3500):
        v = torch.from_numpy(rng.uniform(0.5, 1.5, (n, 1, dim))).to(TYPES[name])
        sink = 0 if first else n - 1
        v[sink] = 0.0
        q, k = torch.zeros((n, heads, dim), dtype=TYPES[name]), torch.zeros((n, 1, dim), dtype=TYPES[name])
        q[..., 0], k[sink, 0, 0] = 1.0, 16.0
        for down in (10.0, 17.3, 20.6, 22.4, 23.6, 24.4, 25.2, 27.7):  # powers of two
            scale = down * math.log(2.0) / 16.0
            got = oz.attention(q.cuda(), k.cuda(), v.cuda(), ints([0, n]), scale=scale, causal=False).double().cpu().numpy()
            p = 2.0 ** -down / (1.0 + (n - 1) * 2.0 ** -down)
            want = p * v.double().numpy().sum((0, 1))
            h = 0.0 if name == "f32" else HALF[name]
            slack = 2 * (2 * (dim + 16) * U * 16 * scale + h + (n + 72) * U) * 2 * want + (n * 2.0 ** -32 * 1.5 if name == "f16" else 0.0)
            tol = slack + HALF[name] * (want + slack) + LEAST[name]
            off = np.abs(got - want)
            assert (off <= tol).all(), "%g below, %d keys: off by %.3g, %.3g of the tolerance" % (down, n, off.max(), (off / tol).max())
