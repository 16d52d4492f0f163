"""One attention layer of a serving program on this library: prompts, then decode steps, for a few users with adapters of their own.

    python examples/serve_layer.py [--tokens N]

A step, for all tokens of the batch at once:
  q, k, v = x Wq, x Wk, x Wv      the base model's products (torch), then the users' adapters: pool.delta over the q, k, v slots
  k, v into the 4-bit cache       k rotated by its positions on the way: cache.append
  attention over the cache        q rotated on the way: cache.attend
  out = o Wo                      and the adapters of the o slot
Weights are random; nothing is compared here (tests/test_gpu_serve_layer.py does that).
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_20210_amd as plora  # noqa: E402

DT = torch.bfloat16


class Layer:
    """Weights, adapters and the KV cache of one layer with grouped heads."""

    def __init__(self, hidden=1024, heads=8, kv_heads=2, head_dim=128, adapters=4, rank=16, page_tokens=64, n_pages=64, max_pos=4096, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.page_tokens = heads, kv_heads, head_dim, page_tokens
        out = [heads * head_dim, kv_heads * head_dim, kv_heads * head_dim, hidden]  # q, k, v, o
        d_in = [hidden, hidden, hidden, heads * head_dim]
        self.base = [(torch.randn(a, b, generator=g, device="cuda") * a ** -0.5).to(DT) for a, b in zip(d_in, out)]
        page = 64 << 10
        per = sum(d_in) + sum(out)
        self.pool = plora.PagedLoraPool(page, adapters * -(-rank * per * 2 // page), d_in, out, plora.PLORA_BF16, adapters, rank)
        self.blobs = [(torch.randn(rank * per, generator=g, device="cuda") * 0.03).to(DT).cpu().pin_memory() for _ in range(adapters)]
        for i, b in enumerate(self.blobs):
            self.pool.load(i, rank, 1.0, b)
        self.rank, self.dims = rank, list(zip(d_in, out))
        table = torch.empty(max_pos, head_dim // 2, 2, device="cuda")
        self.rotary = plora.Rotary.make(table, plora.RotaryConfig(base=10000.0), stream=torch.cuda.current_stream().cuda_stream)
        self.pages = torch.zeros(n_pages, plora.PagedKvCache.page_bytes(kv_heads, head_dim, page_tokens), device="cuda", dtype=torch.uint8)
        self.cache = plora.PagedKvCache(plora.PLORA_BF16, kv_heads, head_dim, page_tokens, self.pages)
        self.workspace = torch.empty(16 << 20, device="cuda", dtype=torch.uint8)

    def step(self, batch, token_adapters, x):
        """x [tokens, hidden] -> ([tokens, hidden], (q, k, v, attention)): batch is a KvBatch that already counts these tokens."""
        n, stream = x.shape[0], torch.cuda.current_stream().cuda_stream
        q, k, v = (x @ w for w in self.base[:3])
        work = [torch.empty(n, self.rank, device="cuda") for _ in range(3)]
        lora = self.pool.batch_begin(token_adapters, stream)
        self.pool.delta(lora, 0, [x, x, x], work, [q, k, v], stream)
        q, k, v = (t.view(n, -1, self.head_dim) for t in (q, k, v))
        o = torch.empty_like(q)
        self.cache.append(batch, k, v, self.rotary, stream)
        self.cache.attend(batch, q, o, self.head_dim ** -0.5, self.workspace, rotary=self.rotary, stream=stream)
        flat = o.view(n, -1)
        out = flat @ self.base[3]
        self.pool.delta(lora, 3, [flat], work[:1], [out], stream)
        self.pool.batch_end(lora)
        return out, (q, k, v, o)

    def close(self):
        torch.cuda.synchronize()
        self.pool.close()


class Users:
    """Which pages each user's sequence has: what a scheduler keeps."""

    def __init__(self, layer, adapters):
        self.layer, self.adapters = layer, list(adapters)
        self.free = list(range(layer.pages.shape[0]))[::-1]
        self.pages = [[] for _ in self.adapters]
        self.length = [0] * len(self.adapters)

    def batch(self, new):
        """(KvBatch, adapter of every token) of a step in which user i brings new[i] tokens."""
        for i, n in enumerate(new):
            self.length[i] += n
            while len(self.pages[i]) * self.layer.page_tokens < self.length[i]:
                self.pages[i].append(self.free.pop())
        table = np.full((len(new), max(1, max(len(p) for p in self.pages))), -1, np.int32)
        for i, p in enumerate(self.pages):
            table[i, :len(p)] = p
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        to = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (start, self.length, table)]
        return plora.KvBatch(*to, int(start[-1]), max(max(new), 1), max(self.length)), np.repeat(np.asarray(self.adapters, np.int32), new)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=64, help="decode steps after the prompts")
    a = ap.parse_args()
    layer = Layer()
    users = Users(layer, [0, 1, 2, 3, -1])  # the last one has no adapter
    x = torch.randn(500, 1024, device="cuda").to(DT)
    out, _ = layer.step(*users.batch([100, 37, 1, 250, 112]), x)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens):
        out, _ = layer.step(*users.batch([1] * 5), out[-5:].contiguous())
    torch.cuda.synchronize()
    print("prompts of 500 tokens, then %d steps of 5 users: %.0f us a step, sequences of %s tokens" % (a.tokens, (time.perf_counter() - t) / a.tokens * 1e6, users.length))
    layer.close()


if __name__ == "__main__":
    main()
