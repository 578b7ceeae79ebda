"""Steps of a decoder without attention, its weights in 4 bits, one captured HIP graph a step.

    python examples/decode_w4.py [--tokens 4] [--layers 2] [--width 1024] [--experts 16] [--steps 16]

Each layer mixes a token's values by two products with a residual (oz2_w4_matvec, the second with beta = 1), then adds a layer
of experts (oz2_w4_moe); the last product gives the logits over the vocabulary, whose largest chooses the next token.  Weights are random.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2504_08009_amd as oz

GROUP = 64


def quantize(w, group=GROUP):
    """Codes and scales of the nearest values s (q - 8) to w (..., n, k), k a multiple of the group."""
    parts = w.float().unflatten(-1, (-1, group))
    s = (parts.abs().amax(-1, keepdim=True) / 7).clamp_min(1e-12).bfloat16().float()
    q = ((parts / s).round().clamp(-8, 7) + 8).to(torch.uint8).flatten(-2)
    return (q[..., 0::2] | q[..., 1::2] << 4).contiguous(), s.squeeze(-1).bfloat16().contiguous()


def weights(gen, *shape):
    w = torch.randn(shape, generator=gen, device="cuda") / shape[-1] ** 0.5
    codes, scales = quantize(w)
    return oz.W4Matrix(codes, scales, group=GROUP)


class Decoder:
    """All tensors of a step are made here, so that a captured step finds them where they were."""

    def __init__(self, tokens, layers, width, inner, experts, top_k, vocabulary, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.embedding = torch.randn((vocabulary, width), generator=gen, device="cuda").bfloat16()
        self.layers = []
        for _ in range(layers):
            router = (torch.randn((experts, width), generator=gen, device="cuda") / width ** 0.5).bfloat16()
            moe = oz.MoeLayer(router, weights(gen, experts, inner, width), weights(gen, experts, inner, width), weights(gen, experts, width, inner), top_k)
            self.layers.append((weights(gen, inner, width), weights(gen, width, inner), moe))
        self.head = weights(gen, vocabulary, width)
        self.ctx = oz.Context()
        self.ctx.allocate_moe_workspace(self.layers[0][2], tokens)
        make = lambda n: torch.empty((tokens, n), dtype=torch.bfloat16, device="cuda")
        self.x, self.inner, self.mixed, self.expert = make(width), make(inner), make(width), make(width)
        self.logits = torch.empty((tokens, vocabulary), device="cuda")
        self.token = torch.arange(tokens, device="cuda") % vocabulary
        self.graph = None

    def step(self):
        self.x.copy_(self.embedding[self.token])
        for up, down, moe in self.layers:
            oz.w4_matvec(up, self.x, out=self.inner)
            self.inner.relu_()
            oz.w4_matvec(down, self.inner, beta=1.0, c=self.x, out=self.mixed)
            self.ctx.w4_moe(moe, self.mixed, out=self.expert)
            torch.add(self.mixed, self.expert, out=self.x)
        oz.w4_matvec(self.head, self.x, out=self.logits)
        self.token.copy_(self.logits.argmax(1))

    def capture(self):
        start = self.token.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()  # once outside: kernels are loaded
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()
        self.token.copy_(start)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in [("tokens", 4), ("layers", 2), ("width", 1024), ("inner", 2048), ("experts", 16), ("top-k", 4), ("vocabulary", 8192), ("steps", 16)]:
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    d = Decoder(a.tokens, a.layers, a.width, a.inner, a.experts, a.top_k, a.vocabulary)
    first = d.token.clone()
    eager = []
    for _ in range(a.steps):
        d.step()
        eager.append(d.token.tolist())
    d.token.copy_(first)
    d.capture()
    torch.cuda.synchronize()
    begin, replayed = time.perf_counter(), []
    for _ in range(a.steps):
        d.graph.replay()
        replayed.append(d.token.tolist())
    print("%d steps of %d tokens, %.0f us a step; the same tokens as without the graph: %s" %
          (a.steps, a.tokens, (time.perf_counter() - begin) / a.steps * 1e6, replayed == eager))
    return 0 if replayed == eager else 1


if __name__ == "__main__":
    sys.exit(main())
