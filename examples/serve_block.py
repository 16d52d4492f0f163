"""A whole block of a serving program on this library: the attention layer of serve_layer.py with base weights in 8 bits, norms and a layer of experts.

    python examples/serve_block.py [--tokens N]

A step, for all tokens of the batch at once (h: the residual stream):
  n8 = norm(h)                              in 8 bits: norm.run
  q, k, v = n8 Wq, n8 Wk, n8 Wv             weights.matmul, then the users' adapters on the norm in the element type: pool.delta
  attention over the 4-bit cache            cache.append, cache.attend
  o = a8 Wo                                 a8: the attention's rows in 8 bits (rows.quantise), and the o slot's adapters
  h = h + o;  n, n8 = norm(h)               norm.run twice (the router reads the element type, the experts 8 bits)
  which experts                             routing.route on the logits n Wr (torch)
  y = act(n8 Wg) * (n8 Wu) Wd, by expert    weights.grouped with rows gathered, rows.quantise with the gate, weights.grouped
  h = h + sum over a token's experts of y   norm.run with places: the sum is part of the next block's norm
Weights are random; nothing is compared here (tests/test_gpu_serve_block.py does that).
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2512_20210_amd as plora  # noqa: E402
from serve_layer import DT, Layer, Users  # noqa: E402


def weights8(w, stream):
    """Weights [.., n, k] of the element type in 8 bits."""
    n, k = w.shape[-2:]
    codes = torch.empty(w.shape, device="cuda", dtype=torch.float8_e4m3fn)
    scales = torch.empty(*w.shape[:-2], -(-n // 128), -(-k // 128), device="cuda")
    return plora.Fp8Weights(codes, scales).quantise(w.contiguous(), stream)


def rows8(n, k):
    return plora.Fp8Rows(torch.empty(n, k, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(-(-k // 128), n, device="cuda"))


class Block:
    """A Layer whose base products are in 8 bits, its norms, and `experts` gated experts of which a token takes top_k."""

    def __init__(self, experts=8, top_k=2, wide=512, seed=1, **kw):
        self.layer = layer = Layer(seed=seed, **kw)
        stream = torch.cuda.current_stream().cuda_stream
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        hidden = layer.base[0].shape[0]
        self.experts, self.top_k, self.wide, self.hidden = experts, top_k, wide, hidden
        self.base = [weights8(w.t(), stream) for w in layer.base]

        def randn(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(DT)

        self.up = weights8(randn(experts, 2 * wide, hidden), stream)  # gate's rows, then up's
        self.down = weights8(randn(experts, hidden, wide), stream)
        self.router = randn(experts, hidden)
        self.norms = [plora.NormWeights((1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).to(DT), eps=1e-5) for _ in range(3)]

    def step(self, batch, token_adapters, h):
        """h [tokens, hidden] -> (the next h, the next block's norm of it, what lies between)."""
        layer, n, stream = self.layer, h.shape[0], torch.cuda.current_stream().cuda_stream
        first = plora.BlockNorm(self.norms[0])
        x, x8 = torch.empty_like(h), rows8(n, self.hidden)
        first.run(h, out=x, stream=stream)
        first.run(h, out8=x8, stream=stream)
        q, k, v = (w.matmul(x8, torch.empty(n, w.n, device="cuda", dtype=DT), stream) for w in self.base[:3])
        work = [torch.empty(n, layer.rank, device="cuda") for _ in range(3)]
        lora = layer.pool.batch_begin(token_adapters, stream)
        layer.pool.delta(lora, 0, [x, x, x], work, [q, k, v], stream)
        q, k, v = (t.view(n, -1, layer.head_dim) for t in (q, k, v))
        a = torch.empty_like(q)
        layer.cache.append(batch, k, v, layer.rotary, stream)
        layer.cache.attend(batch, q, a, layer.head_dim ** -0.5, layer.workspace, rotary=layer.rotary, stream=stream)
        flat = a.view(n, -1)
        a8 = rows8(n, flat.shape[1]).quantise(flat, stream=stream)
        o = self.base[3].matmul(a8, torch.empty(n, self.hidden, device="cuda", dtype=DT), stream)
        layer.pool.delta(lora, 3, [flat], work[:1], [o], stream)
        layer.pool.batch_end(lora)

        middle, m8 = torch.empty_like(h), rows8(n, self.hidden)
        h1 = torch.empty_like(h)
        second = plora.BlockNorm(self.norms[1])
        second.run(o, residual=h, hidden=h1, out=middle, stream=stream)
        second.run(o, residual=h, out8=m8, stream=stream)
        routing, up, gated, down = self.experts_of(middle, m8, stream)
        h2, after = torch.empty_like(h), torch.empty_like(h)
        plora.BlockNorm(self.norms[2]).run(down, residual=h1, hidden=h2, out=after, places=routing.places, place_weights=routing.weights, stream=stream)
        return h2, after, dict(x8=x8, q=q, k=k, v=v, a=a, a8=a8, o=o, h1=h1, middle=middle, m8=m8, routing=routing, up=up, gated=gated, down=down)

    def experts_of(self, x, x8, stream):
        n, k = x.shape[0], self.top_k
        i32 = dict(device="cuda", dtype=torch.int32)
        size = plora.Routing.workspace_bytes(n, self.experts)
        routing = plora.Routing(torch.empty(n, k, **i32), torch.empty(n, k, device="cuda"), torch.empty(self.experts + 1, **i32), torch.empty(n * k, **i32),
                                torch.empty(n, k, **i32), torch.empty(size, device="cuda", dtype=torch.uint8) if size else None)
        routing.route(x @ self.router.t(), stream=stream)
        up = self.up.grouped(x8, routing.offsets, torch.empty(n * k, 2 * self.wide, device="cuda", dtype=DT), routing.rows, stream)
        gated = rows8(n * k, self.wide).quantise(up, plora.PLORA_ACT_SILU, stream)
        down = self.down.grouped(gated, routing.offsets, torch.empty(n * k, self.hidden, device="cuda", dtype=DT), None, stream)
        return routing, up, gated, down

    def close(self):
        self.layer.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=64, help="decode steps after the prompts")
    a = ap.parse_args()
    block = Block()
    users = Users(block.layer, [0, 1, 2, 3, -1])  # the last one has no adapter
    h = torch.randn(500, 1024, device="cuda").to(DT)
    h, _, _ = block.step(*users.batch([100, 37, 1, 250, 112]), h)
    h = h[-5:].contiguous()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens):
        h, _, _ = block.step(*users.batch([1] * 5), h)
        h = h / h.float().std().to(DT)  # (one block over and over: kept in range)
    torch.cuda.synchronize()
    print("prompts of 500 tokens, then %d steps of 5 users: %.0f us a step" % (a.tokens, (time.perf_counter() - t) / a.tokens * 1e6))
    block.close()


if __name__ == "__main__":
    main()
