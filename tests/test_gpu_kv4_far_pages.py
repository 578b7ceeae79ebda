"""Caches whose pages begin behind 2^32 bytes: results that show which page was read.

Every token has a direction of its own as key, and queries point at some of them so that each has nearly all weight: then the result is that token's value, in which every
element is its own.  Tolerances: errors of a result are below 2^-16 of sum p s c, with FP32 queries less (test_kv4_error_bounds); 2^-12 of the values' size is far above that,
and far below what another token's value differs by."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_kv4 import ints

PAGES, HEADS, PAGE, DIM = 9000, 4, 1024, 256  # 4.7 GB of codes of keys, as many of values, 147 MB of scales each


def test_values_of_far_pages():
    rng = np.random.default_rng(7)
    cache = oz.KV4Cache.empty(PAGES, HEADS, PAGE, DIM)
    table = np.array([[8999, 3, 8500, 8998, -1], [0, 8997, 8400, -1, -1]], dtype=np.int32)
    lengths, tokens, cu = [3500, 2100], 5600, [0, 3500, 5600]
    k = torch.from_numpy(rng.choice([-1.0, 1.0], (tokens, HEADS, DIM)).astype(np.float32)).cuda()
    v = torch.from_numpy(rng.uniform(-1.0, 1.0, (tokens, HEADS, DIM)).astype(np.float32)).cuda()
    held = torch.empty_like(k), torch.empty_like(v)
    positions = torch.full((2, HEADS, 5 * PAGE), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros((2, HEADS, 5 * PAGE), device="cuda")
    at = torch.cat([torch.arange(3500), torch.arange(2100)]).int().cuda()
    gpu_table, on_lengths = ints(table), ints(lengths)
    oz.kv4_append(cache, k, v, ints(cu), gpu_table, on_lengths, at=at, positions=positions, weights=weights, held=held)
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, gpu_table, tokens=2, heads=HEADS * 8, weights=True, keep=2000)

    def check(places_of):
        """the tokens of 8 places of every page and head: positions that hold them -> their values"""
        for places in places_of:
            token = torch.stack([torch.stack([cu[s] + positions[s, h, places[s]].long() for h in range(HEADS)]) for s in range(2)])  # (2, heads, 8)
            pick = lambda x: torch.stack([torch.stack([x[token[s, h], h] for h in range(HEADS)]) for s in range(2)])
            # a key meets itself with 256, others with 16 or so: 240 / 4 nats apart
            q = pick(k).reshape(2, HEADS * 8, DIM)
            out = ctx.kv4_attention(cache, q, ints([0, 1, 2]), gpu_table, on_lengths, scale=0.25)
            want = pick(held[1]).reshape(2, HEADS * 8, DIM)
            assert (out - want).abs().max() <= 2.0 ** -12
            other = pick(held[1].roll(1, 0)).reshape(2, HEADS * 8, DIM)  # (no other token's values would pass, nor zeros)
            assert ((want - other).abs().amax(2) > 0.25).all() and (want.abs().amax(2) > 0.25).all()

    some = lambda n: torch.from_numpy(rng.integers(0, n, (2, 8))).cuda()
    ends = [torch.tensor([[0, 1023, 1024, 2047, 2048, 3 * PAGE - 1, 3 * PAGE, 3499], [0, 1023, 1024, 2047, 2048, 2049, 2099, 5]], device="cuda")]
    check(ends + [torch.stack((some(3500)[0], some(2100)[1])) for _ in range(4)])

    # weights that are known: every third place is worth little
    worth = torch.from_numpy(rng.permutation(2 * HEADS * 5 * PAGE).reshape(2, HEADS, 5 * PAGE).astype(np.float32)).cuda()
    weights.copy_(worth)
    parts = {n: getattr(cache, n) for n in ("k_codes", "k_scales", "v_codes", "v_scales")}
    pages = torch.tensor([p for p in table.flatten() if p >= 0], device="cuda")
    before = {n: t[pages].clone() for n, t in parts.items()}
    index = {int(p): i for i, p in enumerate(pages.tolist())}
    ctx.kv4_evict(cache, gpu_table, on_lengths, positions, weights, 2000, recent=10)
    assert on_lengths.tolist() == [2000, 2000]
    for s in range(2):
        n = lengths[s]
        for h in range(HEADS):
            value = worth[s, h, :n].cpu().numpy().astype(np.float64)
            value[n - 10 :] += 1e9
            stay = np.zeros(n, bool)
            stay[np.argsort(-value, kind="stable")[:2000]] = True
            source = np.arange(2000)
            source[~stay[:2000]] = 2000 + np.flatnonzero(stay[2000:])
            assert np.array_equal(positions[s, h, :2000].cpu().numpy(), source)
            to = np.arange(2000)
            for name, t in parts.items():
                now = t[torch.from_numpy(table[s, to // PAGE].astype(np.int64)).cuda(), h, torch.from_numpy(to % PAGE).cuda()]
                was = before[name][torch.tensor([index[int(p)] for p in table[s, source // PAGE]], device="cuda"), h, torch.from_numpy(source % PAGE).cuda()]
                assert torch.equal(now.view(torch.uint8), was.view(torch.uint8)), (name, s, h)
    check([some(2000) for _ in range(5)])
