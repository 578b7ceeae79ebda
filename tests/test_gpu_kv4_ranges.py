"""Caches held in 4 bits where a call is of another size than the tests beside the formula: many sequences, long appends, caches beyond 2^32 bytes, long evictions.
Formulas, tolerances and their derivation: test_gpu_kv4."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_kv4 import TYPES, U, Held, appended, check, check_evict, close, formula, ints


@pytest.mark.parametrize("name,weights", [("bf16", True), ("f32", False)])
def test_many_sequences(name, weights):
    """more than 64, and more than 4096, some without places or new tokens"""
    rng = np.random.default_rng(1)
    for n, heads, kv_heads, dim in ((65, 4, 2, 64), (200, 2, 1, 40), (4200, 1, 1, 8)):
        check(rng.integers(0, 40, n).tolist(), rng.integers(0, 3, n).tolist(), heads, kv_heads, dim, 16, name, weights, seed=n)


@pytest.mark.parametrize("name", TYPES)
def test_large_groups(name):
    for heads, kv_heads, new in ((48, 1, 3), (257, 1, 1), (200, 2, 2)):
        check([90, 33], [new, 1], heads, kv_heads, 64, 16, name, True, seed=heads)


def test_chunks_of_one_place_and_of_many():
    """lengths around the parts that a long sequence is cut into, beside short ones"""
    for n in (1023, 1024, 1025, 4095, 4097):
        check([n, 1, 129], [1, 1, 1], 4, 1, 64, 64, "f16", True, seed=n)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("kv_heads,dim,page", [(2, 64, 48), (1, 256, 16), (3, 40, 64)])
def test_appends_of_many_tokens(kv_heads, dim, page, name):
    """several vectors a lane: ends of sequences and of pages inside a workgroup's run, tokens without a place, rows behind the last sequence"""
    rng = np.random.default_rng(kv_heads)
    lanes = 8
    while lanes * 8 < dim:
        lanes *= 2
    tokens = 4096 * (256 // lanes) // kv_heads + 300
    cuts = np.sort(rng.integers(0, tokens - 40, 60))
    cu = np.concatenate([[0, 0, 1, 3], np.maximum(cuts, 3), [tokens - 37]]).astype(np.int64)
    news = np.diff(cu)
    lengths = [int(n) + int(rng.integers(-2, 50)) if n else int(rng.integers(0, 9)) for n in news]
    lengths = [max(n, 0) for n in lengths]
    of = [-(-n // page) for n in lengths]
    pages, most = sum(of) + 1, max(of) + 1
    table, order, begin = np.full((len(lengths), most), -1, dtype=np.int32), rng.permutation(pages), 0
    for s, n in enumerate(of):
        table[s, :n] = order[begin : begin + n]
        begin += n
    cache = oz.KV4Cache.empty(pages, kv_heads, page, dim)
    cache.k_codes.fill_(0x5a), cache.v_codes.fill_(0xa5), cache.k_scales.fill_(9.0), cache.v_scales.fill_(-9.0)
    want = {n: (c.cpu().clone(), s.cpu().clone()) for n, c, s in (("k", cache.k_codes, cache.k_scales), ("v", cache.v_codes, cache.v_scales))}
    k, v = (torch.from_numpy(rng.standard_normal((tokens, kv_heads, dim)).astype(np.float32)).to(TYPES[name]) for _ in "kv")
    held = tuple(torch.full(k.shape, 7.0, dtype=k.dtype, device="cuda") for _ in "kv")
    at = torch.arange(tokens, dtype=torch.int32)
    positions = torch.full((len(lengths), kv_heads, most * page), -5, dtype=torch.int32)
    places = positions.clone()
    gpu = positions.cuda()
    oz.kv4_append(cache, k.cuda(), v.cuda(), ints(cu), ints(table), ints(lengths), at=at.cuda(), positions=gpu, held=held)
    row = np.repeat(np.arange(len(news)), news)
    place = np.asarray(lengths)[row] - (cu[row + 1] - np.arange(cu[-1]))
    has = place >= 0
    token, row, place = np.arange(cu[-1])[has], row[has], place[has]
    page_of, in_page = table[row, place // page], place % page
    for n, x, back in (("k", k, held[0]), ("v", v, held[1])):
        c, s, o = appended(x)
        want[n][0][page_of, :, in_page] = torch.from_numpy(c[token][:, :, 0::2] | c[token][:, :, 1::2] << 4)
        want[n][1][page_of, :, in_page] = torch.from_numpy(np.stack((s[token], o[token]), axis=2))
        value = c * s.astype(np.float64)[..., None] + o.astype(np.float64)[..., None]
        got = back.double().cpu().numpy()
        half = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name]
        assert (np.abs(got - value)[: cu[-1]] <= ((half + 2 * U) * np.abs(value) + 2.0 ** -24)[: cu[-1]]).all() and (got[cu[-1] :] == 7.0).all()
    places[row, :, place] = at[token][:, None]
    for n, c, s in (("k", cache.k_codes, cache.k_scales), ("v", cache.v_codes, cache.v_scales)):
        assert torch.equal(c.cpu(), want[n][0]) and torch.equal(s.cpu().view(torch.int16), want[n][1].view(torch.int16))
    assert torch.equal(gpu.cpu(), places)


@pytest.mark.parametrize("lengths,keep,recent,kv_heads,page", [([40000, 33000, 5], 20000, 100, 1, 64), ([70000], 69990, 0, 2, 128), ([33000, 32768, 32769], 32760, 32760, 1, 16),
                                                               ([35000], 0, 0, 1, 256), ([20000, 100], 19000, 7, 2, 64)])
@pytest.mark.parametrize("in_place", [False, True], ids=["elsewhere", "in_place"])
def test_long_evictions(lengths, keep, recent, kv_heads, page, in_place):
    rng = np.random.default_rng(keep)
    held = Held(rng, lengths, kv_heads, 8, page, places=3)
    for s, n in enumerate(lengths):
        for h in range(kv_heads):
            held.positions[s, h, :n] = torch.from_numpy(rng.permutation(n)).int()
            held.weights[s, h, : n // 2] = held.weights[s, h, : n // 2].round()  # (many alike)
    check_evict(held, keep, recent, in_place)


def test_a_cache_beyond_32_bits():
    """pages whose codes begin behind 2^32 bytes: appended to, read, evicted from"""
    pages, kv_heads, page, dim = 9000, 4, 1024, 256  # 4.7 GB of codes of keys
    cache = oz.KV4Cache.empty(pages, kv_heads, page, dim)
    rng = np.random.default_rng(7)
    table = np.array([[8999, 3, 8500, 8998, -1], [0, 8997, 8400, -1, -1]], dtype=np.int32)
    lengths, tokens = [3500, 2100], 5600
    k, v = (torch.from_numpy(rng.standard_normal((tokens, kv_heads, dim)).astype(np.float32)).bfloat16() for _ in "kv")
    held = tuple(torch.empty((tokens, kv_heads, dim), device="cuda") for _ in "kv")
    cu = [0, 3500, 5600]
    positions, weights = torch.zeros((2, kv_heads, 5 * page), dtype=torch.int32, device="cuda"), torch.zeros((2, kv_heads, 5 * page), device="cuda")
    at = torch.cat([torch.arange(3500), torch.arange(2100)]).int().cuda()
    oz.kv4_append(cache, k.cuda().float(), v.cuda().float(), ints(cu), ints(table), ints(lengths), at=at, positions=positions, weights=weights, held=held)
    hk, hv = held
    q = torch.from_numpy(rng.standard_normal((2, 8, dim)).astype(np.float32)).cuda()
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, ints(table), tokens=2, heads=8, weights=True, keep=2000)
    out = ctx.kv4_attention(cache, q, ints([0, 1, 2]), ints(table), ints(lengths), weights=weights)

    def plain(rows):  # FP32 operands as the cache holds them; sums in 64 bits
        want = torch.empty((2, 8, dim), dtype=torch.float64, device="cuda")
        got = []
        for s in range(2):
            for h in range(8):
                i = rows[s][h // 2]
                p = torch.softmax(hk[i, h // 2].double() @ q[s, h].double() / 16.0, 0)
                want[s, h] = p @ hv[i, h // 2].double()
                got.append(p)
        return want, got

    everything = [[torch.arange(cu[s], cu[s + 1], device="cuda")] * kv_heads for s in range(2)]
    want, p = plain(everything)
    # codes of up to 15 s + |o| below 16 times the values' range: the bound of the formula's test with S = 4 sum |q| and A = 47 s + |o| <= 30
    slack = 2 * (2 * (dim + 48) * U * (0.0625 * 30 * q.abs().sum(2, keepdim=True).double()) + U + 3600 * U) * 40
    assert ((out.double() - want).abs() <= slack).all()
    for s in range(2):
        for h in range(kv_heads):
            n = lengths[s]
            assert torch.allclose(weights[s, h, :n].double(), p[8 * s + 2 * h] + p[8 * s + 2 * h + 1], rtol=1e-3, atol=1e-9)
    on_lengths = ints(lengths)
    ctx.kv4_evict(cache, ints(table), on_lengths, positions, weights, 2000, recent=10)
    assert on_lengths.tolist() == [2000, 2000]
    out = ctx.kv4_attention(cache, q, ints([0, 1, 2]), ints(table), on_lengths)
    want, _ = plain([[cu[s] + positions[s, h, :2000].long() for h in range(kv_heads)] for s in range(2)])
    assert ((out.double() - want).abs() <= slack).all()


def test_contexts_side_by_side():
    """two contexts on streams of their own and a captured step of a third, under way together, each as if alone"""
    rng = np.random.default_rng(9)
    sets = []
    for i in range(3):
        held = Held(rng, [3000 + i, 700], 2, 128, 64)
        q = torch.from_numpy(rng.standard_normal((2, 8, 128))).bfloat16().cuda()
        ctx = oz.Context()
        ctx.allocate_kv4_workspace(held.cache, held.gpu_table, tokens=2, heads=8, weights=True)
        sets.append((held, q, ctx, ints([0, 1, 2]), torch.empty_like(q), torch.zeros(held.weights.shape, device="cuda")))
    run = lambda s, **more: s[2].kv4_attention(s[0].cache, s[1], s[3], s[0].gpu_table, s[0].gpu_lengths, weights=s[5], out=s[4], **more)
    want = []
    for s in sets:
        run(s)
        want.append((s[4].clone(), s[5].clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(sets[2])
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(4):
        for s in sets:
            s[4].zero_(), s[5].zero_()
        torch.cuda.synchronize()
        run(sets[0], stream=streams[0]), run(sets[1], stream=streams[1])
        with torch.cuda.stream(streams[2]):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s[4], w[0]) and torch.equal(s[5], w[1]) for s, w in zip(sets, want))


def test_a_sequence_of_as_many_places_as_there_may_be():
    """65535 chunks, of which the first and the last have pages; a place that nobody sees receives nothing"""
    rng = np.random.default_rng(10)
    n = 65535 * 4096
    held = Held(rng, [3 * 4096], 1, 64, 4096, spare=0)
    table = torch.full((1, 65535), -1, dtype=torch.int32)
    table[0, 0], table[0, 65533], table[0, 65534] = (int(x) for x in held.table[0])
    q = torch.from_numpy(rng.standard_normal((1, 2, 64))).bfloat16()
    ctx, weights = oz.Context(), torch.zeros((1, 1, n), device="cuda")
    ctx.allocate_kv4_workspace(held.cache, table.cuda(), tokens=1, heads=2, weights=True)
    out = ctx.kv4_attention(held.cache, q.cuda(), ints([0, 1]), table.cuda(), ints([n]), weights=weights)
    want = formula(held, q.double().numpy(), [0, 1], 0.125)
    close(out, want, "bf16", 64)
    got = torch.cat((weights[0, 0, :4096], weights[0, 0, 65533 * 4096 :])).double().cpu().numpy()
    assert (np.abs(got - want[4][0, 0]) <= 2 * want[5][0, 0] + 2 * U * want[4][0, 0]).all()
    assert not weights[0, 0, 4096 : 65533 * 4096].any()


def test_more_rows_than_a_launch_has_workgroups_for_weights():
    """many sequences and heads of a long table: places are received in turns"""
    rng = np.random.default_rng(11)
    sequences, kv_heads, page, places = 600, 1000, 16, 2048  # 600000 pairs, 8 turns each of which 6 go to a workgroup
    cache = oz.KV4Cache.empty(2, kv_heads, page, 8)
    cache.k_scales.fill_(0.25), cache.v_scales.fill_(0.5)
    cache.k_codes.copy_(torch.from_numpy(rng.integers(0, 256, cache.k_codes.shape, dtype=np.uint8)))
    cache.v_codes.copy_(torch.from_numpy(rng.integers(0, 256, cache.v_codes.shape, dtype=np.uint8)))
    table = np.full((sequences, places // page), -1, dtype=np.int32)
    table[:, 0], table[::3, 100] = 0, 1
    lengths = np.where(np.arange(sequences) % 3 == 0, 1616, 16)
    weights = torch.zeros((sequences, kv_heads, places), device="cuda")
    q = torch.from_numpy(rng.standard_normal((1, kv_heads, 8))).bfloat16().expand(sequences, -1, -1).contiguous()
    ctx = oz.Context()
    ctx.allocate_kv4_workspace(cache, ints(table), tokens=sequences, heads=kv_heads, weights=True)
    out = ctx.kv4_attention(cache, q.cuda(), ints(np.arange(sequences + 1)), ints(table), ints(lengths), weights=weights)
    for first in (0, 1):  # sequences are alike by threes
        same = torch.arange(first, sequences, 3, device="cuda")
        assert torch.equal(out[same], out[first].expand(len(same), -1, -1)) and torch.equal(weights[same], weights[first].expand(len(same), -1, -1))
    total = weights[:2].double().sum(2).cpu().numpy()
    assert (np.abs(total - 1) <= (40 + 72) * U * 2).all()
    assert not weights[0, :, 16:1600].any() and not weights[0, :, 1616:].any() and (weights[0, :, 1600:1616] > 0).all() and not weights[1, :, 16:].any()
