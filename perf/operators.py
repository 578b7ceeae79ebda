"""Performance cases of the products with weights held in 4 bits: what programs that answer with a model make of them, over the range they
do it in.

A weight is w[i, l] = scale[i, g] * (code[i, l] - zero[i, g]) with one scale (and, if there are any, one zero point) for each group g = l // group of
a row; codes are two to a byte, the even l in the low half, and where there are no zero points they are 8.  A case is one call of
  op "matvec"  y := alpha W x + beta c for t vectors x, W n x k
     "moe"     a whole layer of experts for t tokens: logits by the router, the top_k experts of each token, their gated products, the weighted sum
with types of the activations ("x") and of the scales, and for a layer d x f experts, how scores are formed, whether a selection bias is there
and how many of the tokens are padding.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MATVEC = dict(op="matvec", x="bf16", scales="bf16", group=128, zeros=False, alpha=1.0, beta=0.0)
MOE = dict(op="moe", x="bf16", scales="bf16", group=128, zeros=False, score="softmax", renormalize=True, factor=1.0, bias=False,
           activation="silu", padding=0)


def _matvec(name, n, k, t, **more):
    return dict(MATVEC, name=name, n=n, k=k, t=t, **more)


def _moe(name, t, experts, top_k, d, f, **more):
    return dict(MOE, name=name, t=t, experts=experts, top_k=top_k, d=d, f=f, **more)


def listed():
    return [
        # the smallest projection of a decoder's step, one token: latency decides
        _matvec("matvec_1024x1024", 1024, 1024, 1),
        # the ordinary one, one token
        _matvec("matvec_4096x4096", 4096, 4096, 1),
        # four sequences at odd sizes (rows that do not start on a whole word), small groups with zero points, added to a residual, all in FP32
        _matvec("matvec_3001x2777_t4_f32", 3001, 2777, 4, x="f32", scales="f32", group=32, zeros=True, beta=1.0),
        # a wide projection with zero points in half precision
        _matvec("matvec_16384x4096_f16", 16384, 4096, 1, x="f16", scales="f16", group=64, zeros=True),
        # sixteen sequences answered together
        _matvec("matvec_8192x8192_t16", 8192, 8192, 16),
        # the output layer over a large vocabulary: reading the weights is everything
        _matvec("matvec_65536x8192", 65536, 8192, 1, group=32),
        # one token through few, wide experts
        _moe("moe_t1_e8_top2_2048x4096", 1, 8, 2, 2048, 4096),
        # one token through many narrow experts
        _moe("moe_t1_e128_top8_2048x1024", 1, 128, 8, 2048, 1024),
        # a few tokens at odd sizes in FP32, gelu
        _moe("moe_t3_e9_top3_1000x777_f32", 3, 9, 3, 1000, 777, x="f32", scales="f32", group=32, zeros=True, activation="gelu"),
        # four sequences: most of their experts are different ones
        _moe("moe_t4_e64_top6_4096x1024_f16", 4, 64, 6, 4096, 1024, x="f16", scales="f16", group=64),
        # a batch with three padded places, sigmoid scores and a bias that balances the experts
        _moe("moe_t16_e64_top6_2048x1408", 16, 64, 6, 2048, 1408, zeros=True, score="sigmoid", bias=True, factor=2.5, padding=3),
        # the largest batch and layer: nearly every expert is wanted by somebody
        _moe("moe_t32_e128_top8_4096x2048", 32, 128, 8, 4096, 2048, group=32),
    ]


MOST_BYTES = 1.5e9


def draw(rng):
    def size(low, high):
        v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        return v if rng.random() < 0.5 else max(64, v // 64 * 64)

    while True:
        x = rng.choice(["bf16", "bf16", "f16", "f32"])
        kind = dict(x=x, scales=rng.choice([x, x, "f32"]), group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.4)
        t = rng.choice([1, 1, 2, 3, 4, 5, 8, 12, 16, 23, 32])
        if rng.random() < 0.5:
            c = dict(MATVEC, n=size(64, 65536), k=size(64, 16384), t=t, beta=rng.choice([0.0, 0.0, 1.0]), **kind)
        else:
            experts = rng.choice([4, 8, 9, 16, 60, 64, 128])
            c = dict(MOE, t=t, experts=experts, top_k=rng.randint(1, min(8, experts)), d=size(256, 4096), f=size(256, 4096),
                     score=rng.choice(["softmax", "sigmoid"]), renormalize=rng.random() < 0.7, bias=rng.random() < 0.3,
                     activation=rng.choice(["silu", "silu", "gelu"]), padding=rng.choice([0, 0, t // 4]), **kind)
            # what the plain form holds at once: the experts of every token
            if c["t"] * c["top_k"] * c["d"] * c["f"] > 32 * 8 * 4096 * 2048:
                continue
        if work(c)["bytes"] <= MOST_BYTES:
            return c


def _weights(gen, case, rows, k, stack=()):
    groups = -(-k // case["group"])
    codes = torch.randint(0, 256, (*stack, rows, (k + 1) // 2), dtype=torch.uint8, device=DEVICE, generator=gen)
    # as a rounding of weights of variance 1 / k to 15 steps gives them
    scales = torch.rand((*stack, rows, groups), device=DEVICE, generator=gen).add_(0.5).mul_(0.25 / math.sqrt(k)).to(TYPES[case["scales"]])
    zeros = torch.randint(5, 12, (*stack, rows, groups), dtype=torch.uint8, device=DEVICE, generator=gen) if case["zeros"] else None
    return codes, scales, zeros


def _activations(gen, t, k, dtype):
    """normal values, one feature in fifty ten times as large, as the inputs of projections have them"""
    x = torch.randn((t, k), device=DEVICE, generator=gen)
    x *= torch.where(torch.rand((k,), device=DEVICE, generator=gen) < 0.02, 10.0, 1.0)
    return x.to(TYPES[dtype])


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    t = case["t"]
    if case["op"] == "matvec":
        n, k = case["n"], case["k"]
        return dict(w=_weights(gen, case, n, k), x=_activations(gen, t, k, case["x"]),
                    c=torch.randn((t, n), device=DEVICE, generator=gen).to(TYPES[case["x"]]) if case["beta"] else None)
    experts, d, f = case["experts"], case["d"], case["f"]
    s = dict(x=_activations(gen, t, d, case["x"]),
             router=(torch.randn((experts, d), device=DEVICE, generator=gen) / math.sqrt(d)).to(TYPES[case["x"]]),
             bias=torch.randn((experts,), device=DEVICE, generator=gen) * 0.1 if case["bias"] else None,
             gate=_weights(gen, case, f, d, (experts,)), up=_weights(gen, case, f, d, (experts,)), down=_weights(gen, case, d, f, (experts,)),
             active=None)
    if case["padding"]:
        s["active"] = torch.arange(t, device=DEVICE) < t - case["padding"]
    return s


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    t, dtype = case["t"], TYPES[case["x"]]
    if not own:
        return s
    import paper_2504_08009_amd as oz

    if case["op"] == "matvec":
        s["matrix"] = oz.W4Matrix(*s["w"], k=case["k"], group=case["group"])
        s["y"] = torch.empty((t, case["n"]), dtype=dtype, device=DEVICE)
        return s
    d, f, group = case["d"], case["f"], case["group"]
    s["layer"] = oz.MoeLayer(s["router"], oz.W4Matrix(*s["gate"], k=d, group=group), oz.W4Matrix(*s["up"], k=d, group=group),
                             oz.W4Matrix(*s["down"], k=f, group=group), case["top_k"], bias=s["bias"], score=case["score"],
                             renormalize=case["renormalize"], factor=case["factor"], activation=case["activation"])
    s["ctx"] = oz.Context()
    s["ctx"].allocate_moe_workspace(s["layer"], t, device=DEVICE)
    s["y"] = torch.empty((t, d), dtype=dtype, device=DEVICE)
    s["ids"] = torch.empty((t, case["top_k"]), dtype=torch.int32, device=DEVICE)
    s["weights"] = torch.empty((t, case["top_k"]), dtype=torch.float32, device=DEVICE)
    return s


def _values(w, k, group):
    """the weights that codes, scales and zero points stand for, in FP32"""
    codes, scales, zeros = w
    q = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)[..., :k].float()
    g = torch.arange(k, device=codes.device) // group
    q -= 8.0 if zeros is None else zeros[..., g].float()
    return q.mul_(scales[..., g].float())


def _chosen(s):
    """experts and weights of every token: (t, top_k) each, -1 and 0 in a place without an expert"""
    logits = s["x"].float() @ s["router"].float().t()
    if s["score"] == "softmax":
        e = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        p = e / e.sum(dim=1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-logits))
    key = p if s["bias"] is None else p + s["bias"]
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, : s["top_k"]]
    there = key.gather(1, ids) != -math.inf
    if s["active"] is not None:
        there &= s["active"][:, None]
    weights = torch.where(there, p.gather(1, ids), 0.0)
    if s["renormalize"]:
        total = weights.sum(dim=1, keepdim=True)
        weights = torch.where(total == 0, 0.0, weights / total)
    return torch.where(there, ids, -1).int(), weights * s["factor"]


def _of_experts(w, ids):
    return tuple(None if v is None else v[ids] for v in w)


def _product(w, x, k, group):
    """W x of every place: (places, rows) from (places, k)"""
    return (_values(w, k, group) * x[:, None, :]).sum(dim=2) if x.shape[0] <= 4 else torch.bmm(_values(w, k, group), x[:, :, None])[:, :, 0]


def run(s):
    if own:
        import paper_2504_08009_amd as oz

        if s["op"] == "matvec":
            return oz.w4_matvec(s["matrix"], s["x"], alpha=s["alpha"], beta=s["beta"], c=s["c"], out=s["y"])
        y, ids, weights = s["ctx"].w4_moe(s["layer"], s["x"], active=s["active"], out=s["y"], ids=s["ids"], weights=s["weights"])
        return {"y": y, "ids": ids, "weights": weights}
    if s["op"] == "matvec":
        y = s["x"].float() @ _values(s["w"], s["k"], s["group"]).t() * s["alpha"]
        if s["c"] is not None:
            y += s["beta"] * s["c"].float()
        return y.to(s["x"].dtype)
    t, top_k, d, f, group = s["t"], s["top_k"], s["d"], s["f"], s["group"]
    ids, weights = _chosen(s)
    places = ids.clamp(min=0).flatten().long()
    x = s["x"].float().repeat_interleave(top_k, dim=0)
    g = _product(_of_experts(s["gate"], places), x, d, group)
    u = _product(_of_experts(s["up"], places), x, d, group)
    h = u * (g / (1.0 + torch.exp(-g)) if s["activation"] == "silu" else 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5))))
    y = _product(_of_experts(s["down"], places), h, f, group).view(t, top_k, d)
    y = torch.where(ids[:, :, None] >= 0, y * weights[:, :, None], 0.0).sum(dim=1)
    return {"y": y.to(s["x"].dtype), "ids": ids, "weights": weights}


def work(case):
    """Bytes: codes, scales and zero points of the weights that are wanted, inputs and results once.  Of a layer of experts those are the
    experts that t tokens choose when each chooses evenly among all of them."""
    size = {"bf16": 2, "f16": 2, "f32": 4}

    def weights(rows, k):
        return rows * ((k + 1) // 2 + -(-k // case["group"]) * (size[case["scales"]] + (1 if case["zeros"] else 0)))

    t, a = case["t"], size[case["x"]]
    if case["op"] == "matvec":
        n, k = case["n"], case["k"]
        return {"bytes": float(weights(n, k) + a * t * (k + n * (2 if case["beta"] else 1))), "flops": 2.0 * n * k * t}
    experts, top_k, d, f = case["experts"], case["top_k"], case["d"], case["f"]
    t -= case["padding"]
    wanted = experts * (1.0 - (1.0 - top_k / experts) ** t)
    return {"bytes": wanted * (2 * weights(f, d) + weights(d, f)) + a * (experts * d + 2 * case["t"] * d) + case["t"] * top_k * 8.0,
            "flops": 2.0 * t * experts * d + 6.0 * t * top_k * d * f}


def _product64(w, x, k, group):
    """x (t, k) times the rows of w in 64 bits: the even and the odd inner indexes apart, a group's scale applied to its sum"""
    codes, scales, zeros = w
    groups, half = -(-k // group), group // 2
    t = x.shape[0]
    padded = torch.zeros((t, groups * group), dtype=torch.float64, device=x.device)
    padded[:, :k] = x
    pairs = padded.view(t, groups, half, 2)
    even, odd = pairs[..., 0].permute(1, 2, 0).contiguous(), pairs[..., 1].permute(1, 2, 0).contiguous()
    sums = padded.view(t, groups, group).sum(dim=2).t()
    out = torch.empty((t, codes.shape[0]), dtype=torch.float64, device=x.device)
    for r in range(0, codes.shape[0], 2048):
        c = torch.zeros((min(2048, codes.shape[0] - r), groups * half), dtype=torch.uint8, device=x.device)
        c[:, : codes.shape[1]] = codes[r : r + 2048]
        c = c.view(c.shape[0], groups, half).permute(1, 0, 2).contiguous()
        q = torch.matmul((c % 16).double(), even) + torch.matmul((c // 16).double(), odd)
        z = 8.0 if zeros is None else zeros[r : r + 2048].double().t()[:, :, None]
        out[:, r : r + 2048] = (scales[r : r + 2048].double().t()[:, :, None] * (q - z * sums[:, None, :])).sum(dim=0).t()
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    x = s["x"].double()
    if case["op"] == "matvec":
        y = case["alpha"] * _product64(s["w"], x, case["k"], case["group"])
        return y if s["c"] is None else y + case["beta"] * s["c"].double()
    t, top_k, d, f, group = case["t"], case["top_k"], case["d"], case["f"], case["group"]
    p = torch.matmul(x, s["router"].double().t())
    p = torch.softmax(p, dim=1) if case["score"] == "softmax" else torch.sigmoid(p)
    key = (p if s["bias"] is None else p + s["bias"].double()).tolist()
    p = p.tolist()
    ids, weights = torch.full((t, top_k), -1, dtype=torch.int32), torch.zeros((t, top_k), dtype=torch.float64)
    for i in range(t - case["padding"]):
        best = sorted(range(case["experts"]), key=lambda e: (-key[i][e], e))[:top_k]
        total = sum(p[i][e] for e in best) if case["renormalize"] else 1.0
        for j, e in enumerate(best):
            ids[i, j], weights[i, j] = e, case["factor"] * p[i][e] / total
    y = torch.zeros((t, d), dtype=torch.float64, device=DEVICE)
    for e in sorted(set(ids.flatten().tolist()) - {-1}):
        at, j = (v.tolist() for v in torch.where(ids == e))
        one = {m: tuple(None if v is None else v[e] for v in s[m]) for m in ("gate", "up", "down")}
        g, u = _product64(one["gate"], x[at], d, group), _product64(one["up"], x[at], d, group)
        h = u * (g * torch.sigmoid(g) if case["activation"] == "silu" else torch.nn.functional.gelu(g))
        y[at] += weights[at, j].to(DEVICE)[:, None] * _product64(one["down"], h, f, group)
    return {"y": y, "ids": ids, "weights": weights}
