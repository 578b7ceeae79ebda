"""Attention over a cache held in 4 bits with results in FP32, within bounds that a kernel with one bf16 term fewer of q or of p s would not keep: test_kv4_error_bounds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_kv4 import ints
from test_kv4_error_bounds import SHAPES, TYPES, Case, bounds, rms


@pytest.mark.parametrize("whole", [False, True], ids=["", "whole"])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_errors(shape, name, whole):
    rng = np.random.default_rng(sum(shape))
    case = Case(rng, *shape, name, whole)
    (n, dim), rows, page = shape, case.q.shape[0], 16
    of = -(-n // page)
    table = rng.permutation(of + 1)[None, :of]
    t = np.arange(n)
    parts = []
    for codes, scale, offset in ((case.kc, case.ks, case.ko), (case.vc, case.vs, case.vo)):
        held, pairs = np.full((of + 1, 1, page, dim // 2), 0xff, dtype=np.uint8), np.full((of + 1, 1, page, 2), np.nan, dtype=np.float16)
        held[table[0, t // page], 0, t % page] = codes[:, 0::2] | codes[:, 1::2] << 4
        pairs[table[0, t // page], 0, t % page] = np.stack((scale, offset), axis=1)
        parts += [torch.from_numpy(held).cuda(), torch.from_numpy(pairs).cuda()]
    cache = oz.KV4Cache(*parts)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, ints(table), tokens=1, heads=rows, weights=True)
    q = torch.from_numpy(case.q[None]).to(TYPES[name])
    assert np.array_equal(q.float().numpy()[0], case.q)
    out, received = torch.empty((1, rows, dim), device="cuda"), torch.zeros((1, 1, of * page), device="cuda")
    ctx.kv4_attention(cache, q.cuda(), ints([0, 1]), ints(table), ints([n]), scale=case.scale, weights=received, out=out)
    want, p, of_out, of_p = bounds(case, name)
    off = rms(out[0].double().cpu().numpy() - want)
    assert off <= of_out, "%.3g of the bound" % (off / of_out)
    # (what a place receives is a sum over the rows, in FP32)
    off, bound = rms(received[0, 0, :n].double().cpu().numpy() - p.sum(0)), rows * of_p + 2.0 ** -24 * rows * rms(p.sum(0))
    assert off <= bound, "%.3g of the bound of weights" % (off / bound)
