"""examples/serve_block.py: prompts and decode steps of a whole block, each operator against 64 bits on what the one before it gave.

Bounds: codes of 8 bits are within half a step, 2^-4 of a value and 2^-10 of the scale; results of products as a 2-norm within the rounding of
two bf16 results in a row (base product, adapters) or one; choices of experts equal those of the same logits.
"""
import importlib.util
import os
import sys

import numpy as np
import pytest

from oracle import base as O

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        spec = importlib.util.spec_from_file_location("serve_block", os.path.join(ROOT, "examples", "serve_block.py"))
        M = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(M)
    finally:
        sys.path.pop(0)
    return M


def near(a, b, most):
    return np.linalg.norm(a - b) <= most * np.linalg.norm(b)


def test_block_against_64_bits():
    import torch
    M = example()
    block = M.Block(adapters=2)
    layer = block.layer
    users = M.Users(layer, [1, -1, 0])
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    raw = lambda t: t.view(torch.uint8).cpu().numpy()  # noqa: E731
    val = lambda r: O.row_values(raw(r.codes), r.scales.cpu().numpy())  # noqa: E731
    base = [O.weight_values(raw(w.codes), w.scales.cpu().numpy()) for w in block.base]
    for w, b in zip(base, layer.base):  # [out][in] of the same weights
        assert (np.abs(w - f64(b).T) <= 2.0 ** -4 * np.abs(f64(b).T) + 2.0 ** -10 * np.abs(f64(b)).max() / 448 * 1.01).all()
    up, down = ([O.weight_values(raw(w.codes[e]), w.scales[e].cpu().numpy()) for e in range(block.experts)] for w in (block.up, block.down))
    norms = [dict(weight=f64(p.kept[0]), eps=1e-5) for p in block.norms]
    blobs = [f64(b) for b in layer.blobs]
    r = layer.rank

    def adapted(slot, y, x, adapters):
        at = r * sum(a + b for a, b in layer.dims[:slot])
        di, do = layer.dims[slot]
        for t, i in enumerate(adapters):
            if i >= 0:
                A, B = blobs[i][at:at + r * di].reshape(r, di), blobs[i][at + r * di:at + r * (di + do)].reshape(r, do)
                y[t] += (x[t] @ A.T) @ B
        return y

    def eight(rows, y):
        s = np.repeat(rows.scales.double().cpu().numpy(), 128, 0)[:rows.k].T
        assert (np.abs(val(rows) - y) <= (2.0 ** -4 + 1e-4) * np.abs(y) + 2.0 ** -10 * s).all()

    gen = torch.Generator(device="cuda").manual_seed(3)
    for new in ([70, 33, 200], [1, 1, 1], [5, 0, 40]):
        batch, adapters = users.batch(new)
        h = (2 * torch.randn(sum(new), 1024, device="cuda", generator=gen)).to(torch.bfloat16)
        h2, after, m = block.step(batch, adapters, h)
        h64 = f64(h)
        x64 = O.norm(h64, **norms[0])
        eight(m["x8"], x64)
        for slot, name in ((0, "q"), (1, "k"), (2, "v")):
            ref = adapted(slot, val(m["x8"]) @ base[slot].T, x64, adapters)
            assert near(f64(m[name]).reshape(ref.shape), ref, 4e-3)
        flat = f64(m["a"]).reshape(len(h64), -1)
        eight(m["a8"], flat)
        assert near(f64(m["o"]), adapted(3, val(m["a8"]) @ base[3].T, flat, adapters), 4e-3)
        h1 = h64 + f64(m["o"])
        assert near(f64(m["h1"]), h1, 2.0 ** -8) and near(f64(m["middle"]), O.norm(h1, **norms[1]), 2.0 ** -8)
        eight(m["m8"], O.norm(h1, **norms[1]))
        logits = f64(m["middle"] @ block.router.t())
        e, w, offsets, rows, places = O.route(logits, block.top_k)
        got = m["routing"]
        for a, b in ((got.experts, e), (got.offsets, offsets), (got.rows, rows), (got.places, places)):
            assert (a.cpu().numpy() == b).all()
        assert np.abs(f64(got.weights) - w).max() < 1e-5
        x = val(m["m8"])
        ups, downs = np.zeros((len(rows), 2 * block.wide)), np.zeros((len(rows), 1024))
        gated = val(m["gated"])
        for i in range(block.experts):
            a, b = offsets[i], offsets[i + 1]
            ups[a:b] = x[rows[a:b]] @ up[i].T
            downs[a:b] = gated[a:b] @ down[i].T
        assert near(f64(m["up"]), ups, 2.0 ** -8)
        eight(m["gated"], O.activated(f64(m["up"]), "silu"))
        assert near(f64(m["down"]), downs, 2.0 ** -8)
        last = f64(m["h1"]) + O.gathered(f64(m["down"]), places, w)
        assert near(f64(h2), last, 2.0 ** -8) and near(f64(after), O.norm(last, **norms[2]), 2.0 ** -8)
    block.close()


def test_experts_in_a_graph_and_beside_another_stream():
    """A layer of experts recorded once and replayed on changing rows, with eager work between; the same calls on two streams at once."""
    import torch
    M = example()
    block = M.Block()
    n = 300
    gen = torch.Generator(device="cuda").manual_seed(4)
    draw = lambda: torch.randn(n, 1024, device="cuda", generator=gen).to(torch.bfloat16)  # noqa: E731

    def run(x, keep):
        stream = torch.cuda.current_stream().cuda_stream
        x8 = M.rows8(n, 1024)
        norm = M.plora.BlockNorm(block.norms[0])
        mid = torch.empty_like(x)
        norm.run(x, out=mid, stream=stream)
        norm.run(x, out8=x8, stream=stream)
        routing, _, _, down = block.experts_of(mid, x8, stream)
        out, hidden = torch.empty_like(x), torch.empty_like(x)
        norm.run(down, residual=x, hidden=hidden, out=out, places=routing.places, place_weights=routing.weights, stream=stream)
        keep.append((x8, mid, routing, down))
        return hidden, out

    keep, x = [], draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(x, keep)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = run(x, keep)
    for _ in range(4):
        x.copy_(draw())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in recorded]
        want = run(x, keep)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    xs = [draw(), draw()]
    want = [run(v, keep) for v in xs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(run(xs[i], keep))
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(pair, want[i]))
    block.close()
