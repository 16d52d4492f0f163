"""examples/serve_layer.py: prompts, chunks and decode steps of one layer against the same layer in 64 bits.

Bounds: what the cache keeps of k and v is taken as the library's rows choose it (the oracle's choice of the k and v that the step
returns, rotated in fp32), so attention is held to the roundings of a bf16 result, 2^-8, of its weights and of q, as a
2-norm; q, k, v and the output to the roundings of two bf16 results in a row (base product, then the adapters' update).
"""
import importlib.util
import os

import numpy as np
import pytest

from oracle import kv as O

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def norm(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


def test_layer_against_64_bits():
    import torch
    spec = importlib.util.spec_from_file_location("serve_layer", os.path.join(ROOT, "examples", "serve_layer.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    layer = M.Layer()
    users = M.Users(layer, [2, -1, 0])
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    base = [f64(w) for w in layer.base]
    blobs = [f64(b) for b in layer.blobs]
    r, d = layer.rank, layer.head_dim

    def adapted(slot, x, adapters):
        y = x @ base[slot]
        at = r * sum(a + b for a, b in layer.dims[:slot])
        di, do = layer.dims[slot]
        for t, i in enumerate(adapters):
            if i >= 0:
                A, B = blobs[i][at:at + r * di].reshape(r, di), blobs[i][at + r * di:at + r * (di + do)].reshape(r, do)
                y[t] += (x[t] @ A.T) @ B
        return y

    cs = O.angles(O.frequencies(d), np.arange(400)).astype(np.float32)
    kept = [([], []) for _ in range(3)]  # rows as the cache stands for them, rotated keys and values
    gen = torch.Generator(device="cuda").manual_seed(3)
    for new in ([70, 33, 0], [1, 1, 1], [5, 0, 40], [1, 1, 1]):
        batch, adapters = users.batch(new)
        x = torch.randn(sum(new), 1024, device="cuda", generator=gen).to(torch.bfloat16)
        out, (q, k, v, o) = layer.step(batch, adapters, x)
        x64 = f64(x)
        for slot, t in ((0, q), (1, k), (2, v)):
            assert norm(f64(t).reshape(len(x64), -1), adapted(slot, x64, adapters)) < 4e-3
        at = 0
        for i, n in enumerate(new):
            places = np.arange(users.length[i] - n, users.length[i])
            rows = slice(at, at + n)
            at += n
            if not n:
                continue
            turned = O.rotate(f64(k[rows]).astype(np.float32), cs[places], False)
            for store, y in zip(kept[i], (turned, f64(v[rows]))):
                for row in y:
                    c, s, m = O.chosen(row, 32)
                    store.append(m[:, None] + s[:, None].astype(np.float64) * c)
            ref, _, _ = O.attend(O.rotate(f64(q[rows]), cs[places].astype(np.float64), False), np.array(kept[i][0]), np.array(kept[i][1]), d ** -0.5, places)
            assert norm(f64(o[rows]), ref) < 2.5e-3
        assert norm(f64(out), adapted(3, f64(o).reshape(len(x64), -1), adapters)) < 4e-3
    layer.close()
