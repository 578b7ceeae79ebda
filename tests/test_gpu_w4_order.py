"""Layers of experts on the matrix cores: the order of a token's sums follows from the sizes of the call alone, so what other tokens choose
changes no bit of its result, and equal calls give equal bits.  Inner dimensions here are several runs of blocks and several chunks long."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def stack(gen, experts, n, k, group):
    codes = torch.randint(0, 256, (experts, n, (k + 1) // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = (torch.rand((experts, n, -(-k // group)), device="cuda", generator=gen) + 0.5) / (4 * k ** 0.5)
    return oz.W4Matrix(codes, scales, k=k, group=group)


def layer_of(gen, experts, top_k, d, f, group):
    """expert e is chosen for what feature e of a token holds"""
    router = torch.eye(experts, d, device="cuda")
    return oz.MoeLayer(router, stack(gen, experts, f, d, group), stack(gen, experts, f, d, group), stack(gen, experts, d, f, group), top_k)


def tokens_of(gen, choices, experts, d, x_type):
    x = torch.randn((len(choices), d), device="cuda", generator=gen)
    x[:, :experts] *= 0.1
    return choose(x.to(TYPES[x_type]), range(len(choices)), choices)


def choose(x, tokens, choices):
    """the tokens' features so that these experts are chosen, in that order"""
    for t, experts in zip(tokens, choices):
        x[t, x[t] >= 4] = 0.0
        for j, e in enumerate(experts):
            x[t, e] = 16.0 - j
    return x


def call(layer, x):
    ctx = oz.Context()
    ctx.allocate_moe_workspace(layer, x.shape[0])
    out = torch.full(x.shape, float("nan"), device="cuda")
    y, ids, weights = ctx.w4_moe(layer, x, out=out)
    torch.cuda.synchronize()
    return y, ids, weights


def same_but_for(token, layer, x, other):
    """the results of all tokens but one where this one makes another choice; and they are there"""
    a = call(layer, x)
    x = choose(x.clone(), [token], [other])
    b = call(layer, x)
    assert a[1][token].tolist() != b[1][token].tolist() == list(other)
    keep = [i for i in range(x.shape[0]) if i != token]
    assert all(torch.equal(u[keep], v[keep]) for u, v in zip(a[1:], b[1:])) and bool(a[0].isfinite().all())
    off = (a[0][keep] != b[0][keep]).any(dim=1)
    assert not bool(off.any()), "tokens %s differ" % [keep[i] for i in off.nonzero().flatten().tolist()]


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("t,experts", [(16, 12), (24, 48)])
def test_the_rank_of_an_expert_among_the_chosen_changes_nothing(t, experts, x_type):
    """Five runs of blocks each way, at most four tokens an expert: one expert more is chosen, of a lower index than all others."""
    print(t, experts, x_type, flush=True)
    gen = torch.Generator("cuda").manual_seed(41)
    layer = layer_of(gen, experts, 2, 1300, 1400, 64)
    others = experts - 1
    choices = [(1 + 2 * i % others, 1 + (2 * i + 1) % others) for i in range(t)]
    x = tokens_of(gen, choices, experts, 1300, x_type)
    same_but_for(2, layer, x, (0, choices[2][1]))


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("t,experts,sharing,d,f", [(30, 4, 29, 1408, 1400), (32, 48, 9, 1300, 2100)])
def test_how_many_tokens_share_an_expert_changes_nothing(t, experts, sharing, d, f, x_type):
    """`sharing` tokens have the same two experts, in several lots of as many as the matrix cores take at a time; without one of them, each behind it is
    one place further ahead.  The chosen experts are the same."""
    print(t, experts, sharing, d, f, x_type, flush=True)
    gen = torch.Generator("cuda").manual_seed(42)
    layer = layer_of(gen, experts, 2, d, f, 128)
    rest = [e for e in range(experts) if e not in (1, 2)]
    choices = [(1, 2) if i < sharing else (rest[2 * i % len(rest)], rest[(2 * i + 1) % len(rest)]) for i in range(t)]
    x = tokens_of(gen, choices, experts, d, x_type)
    same_but_for(0, layer, x, choices[sharing])


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
def test_equal_calls_give_equal_bits_where_many_tokens_share_an_expert(x_type):
    """more places than a wave deals out at a time"""
    gen = torch.Generator("cuda").manual_seed(43)
    layer = layer_of(gen, 5, 4, 1408, 1400, 128)
    choices = [[(i + j) % 5 for j in range(4)] for i in range(32)]
    x = tokens_of(gen, choices, 5, 1408, x_type)
    first = [v.clone() for v in call(layer, x)]
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(call(layer, x), first))
