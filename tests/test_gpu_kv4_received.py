"""What places of a cache receive where a row of the call is not finite: the places that the row sees receive a NaN, all others what the other rows give them."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_kv4 import TYPES, U, Held, formula, ints


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("what", [math.nan, math.inf])
@pytest.mark.parametrize("length,bad", [(40, 1), (700, 20)])
@pytest.mark.parametrize("heads", [4, 60])
def test_places_that_an_odd_row_does_not_see(heads, length, bad, what, name):
    """`length` places of which the new tokens are the last four; one page is none; the second new token's row of head 0 is not finite"""
    rng = np.random.default_rng(length)
    held = Held(rng, [length, 30], 2, 64, 16)
    held.table[0, bad] = -1
    held.gpu_table = ints(held.table)
    q = torch.from_numpy(rng.standard_normal((5, heads, 64))).to(TYPES[name])
    cu = [0, 4, 5]
    clean = q.double().numpy()
    q[1, 0, 3] = what
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=5, heads=heads, weights=True)
    received = held.weights.cuda()
    ctx.kv4_attention(held.cache, q.cuda(), ints(cu), held.gpu_table, held.gpu_lengths, weights=received)
    got, before = received.double().cpu().numpy(), held.weights.double().numpy()
    want = formula(held, clean, cu, 0.125)
    place = np.arange(held.capacity)
    sees = (place < length - 2) & (place // 16 != bad)
    assert np.isnan(got[0, 0, sees]).all()
    rest = np.ones(got.shape, bool)
    rest[0, 0, sees] = False
    # (the other rows' part: none of the odd one is in places that it does not see)
    assert (np.abs(got - before - want[4]) <= 2 * want[5] + 2 * U * (before + want[4]))[rest].all()
    hidden = np.zeros(got.shape, bool)
    hidden[0, :, bad * 16 : bad * 16 + 16], hidden[0, :, length:] = True, True
    assert np.array_equal(got[hidden], before[hidden])
