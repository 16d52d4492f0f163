"""Calls of the base layer's operators that their contract allows, beside those of test_gpu_base.py: results in place of every input that may be one, one row for
all, one row gathered by all, masks of a type's lowest value, products in a graph.  Bounds as there."""
import numpy as np
import pytest

import test_gpu_base as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [264, 2056, 9224])
@pytest.mark.parametrize("hidden,out", [("block", None), ("gate", None), (None, "residual"), (None, "gate"), ("block", "residual"), ("gate", "block"), ("residual", "gate"),
                                        ("residual", "block"), ("block", "gate"), ("gate", "residual")])
def test_norm_in_place_of_each_input(dtype, dim, hidden, out):
    import torch
    rng = np.random.default_rng(dim)
    kw, norm, *_ = B.norm_case(rng, dtype, 37, dim, gate="rows", post=B.RMS, pre=B.LAYER)
    want = [torch.empty_like(kw["block"]) for _ in range(2)]
    norm.run(hidden=want[0], out=want[1], stream=B.stream(), **kw)
    mine = {name: t.clone() for name, t in kw.items()}
    norm.run(hidden=hidden and mine[hidden], out=out and mine[out], stream=B.stream(), **mine)
    for name, w in ((hidden, want[0]), (out, want[1])):
        assert name is None or torch.equal(mine[name], w)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_norm_of_gathered_rows_in_place_of_residual_and_gate(dtype):
    import torch
    kw, norm, *_ = B.norm_case(np.random.default_rng(1), dtype, 19, 520, top_k=3, gate="rows", post=B.RMS, pre=B.RMS)
    want = [torch.empty_like(kw["residual"]) for _ in range(2)]
    norm.run(hidden=want[0], out=want[1], stream=B.stream(), **kw)
    mine = {name: t.clone() for name, t in kw.items()}
    norm.run(hidden=mine["residual"], out=mine["gate"], stream=B.stream(), **mine)
    assert torch.equal(mine["residual"], want[0]) and torch.equal(mine["gate"], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_one_row_for_all(dtype):
    """Inputs of stride 0 give what the row repeated gives."""
    import torch
    P = B.lib()
    n, d = 33, 1032
    rng = np.random.default_rng(3)
    block, residual, gate = (B.put(rng.normal(size=(1, d)), dtype)[0].expand(n, d) for _ in range(3))
    weight, _ = B.put(rng.normal(size=d), dtype)
    norm = P.BlockNorm(P.NormWeights(weight), P.NormWeights(eps=1e-5))
    got, want = ([torch.empty(n, d, device="cuda", dtype=block.dtype) for _ in range(2)] for _ in range(2))
    norm.run(block, residual, *got, gate=gate, stream=B.stream())
    norm.run(block.contiguous(), residual.contiguous(), *want, gate=gate.contiguous(), stream=B.stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    r, codes, scales = B.empty_rows(n, d)
    s, codes2, scales2 = B.empty_rows(n, d)
    r.quantise(block, stream=B.stream())
    s.quantise(block.contiguous(), stream=B.stream())
    assert torch.equal(codes, codes2) and torch.equal(scales, scales2)
    logits = block[:, :60]
    a, b = B.routing(n, 60, 4), B.routing(n, 60, 4)
    a.route(logits, stream=B.stream())
    b.route(logits.contiguous(), stream=B.stream())
    for name in ("experts", "weights", "offsets", "rows", "places"):
        assert torch.equal(getattr(a, name), getattr(b, name))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("total,n,k", [(20, 136, 272), (700, 264, 1040), (700, 5128, 144)])
def test_one_row_gathered_by_all(dtype, total, n, k):
    import torch
    P = B.lib()
    rng = np.random.default_rng(total)
    x, xv = B.made_rows(rng, 1, k)
    w, wv = B.made_weights(rng, n, k, 3)
    rows = np.zeros(total, int)
    rows[5] = 1
    out = torch.empty(total, n, device="cuda", dtype=getattr(torch, B.DT[dtype][1]))
    edge = [0, total // 3, total // 3 + 1, total]
    w.grouped(x, B.ints(edge), out, B.ints(rows), B.stream())
    got = B.host(out)
    assert np.isnan(got[5]).all()
    for e in range(3):
        r = [i for i in range(edge[e], edge[e + 1]) if i != 5]
        B.check_product(got[r], xv[rows[r]], wv[e], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,e,k", [(6, 5, 5), (40, 64, 8), (70, 100, 6), (64, 300, 20), (130, 700, 4)])
def test_routing_of_extreme_logits(dtype, n, e, k):
    """Masks of the type's lowest value are values like others (chosen last, by their index, with p = 0 beside ordinary ones); zeros of both signs are alike; values that
    are hardly any, or as large as there are."""
    import torch
    info = torch.finfo(getattr(torch, B.DT[dtype][1]))
    rng = np.random.default_rng(n * e)
    x = rng.normal(size=(n, e))
    x[0] = info.min
    x[1, :] = info.min
    x[1, e // 2] = 3
    x[2] = np.where(np.arange(e) % 2, 0.0, -0.0)
    x[3] = rng.choice([info.min, info.max, 0, -info.smallest_normal, info.smallest_normal, -np.inf], e)
    x[4] = info.smallest_normal * rng.choice([0, 0.5, -0.5, 0.25, -0.25], e)
    x[5] = info.max
    t, x64 = B.put(x, dtype)
    for renormalise in (True, False):
        r = B.routing(n, e, k)
        r.route(t, renormalise, 1.5, B.stream())
        experts, w, offsets, rows, places = B.O.route(x64, k, renormalise, 1.5)
        for got, want in ((r.experts, experts), (r.offsets, offsets), (r.rows, rows), (r.places, places)):
            assert (got.cpu().numpy() == want).all()
        got = B.host(r.weights)
        # as in check_route; where a difference of logits passes fp32 both exponentials are 0
        spread = np.where(np.isfinite(x64), x64, 0)
        off = np.minimum(2 * (spread.max(1) - spread.min(1)), 2 * 104) + 40
        assert (np.abs(got - w) <= off[:, None] * B.U * np.abs(w) + 2e-38).all()


@pytest.mark.parametrize("t,n,k", [(1, 8200, 1424), (5, 264, 1040), (40, 264, 2064), (300, 1032, 528), (200, 16392, 1424)])
def test_products_in_a_graph(t, n, k):
    """Recorded once, replayed over new rows and new weights, with eager calls between."""
    import torch
    P = B.lib()
    g = torch.Generator(device="cuda").manual_seed(t)
    x, w = torch.empty(t, k, device="cuda"), torch.empty(n, k, device="cuda")
    x8, codes, scales = B.empty_rows(t, k)
    w8 = P.Fp8Weights(torch.empty(n, k, device="cuda", dtype=torch.uint8), torch.empty(-(-n // 128), -(-k // 128), device="cuda"))
    out = torch.empty(t, n, device="cuda", dtype=torch.bfloat16)

    def run():
        s = torch.cuda.current_stream().cuda_stream
        w8.quantise(w, s)
        x8.quantise(x, stream=s)
        w8.matmul(x8, out, s)

    def fill():
        for a in (x, w):
            a.copy_(torch.randn(a.shape, generator=g, device="cuda"))

    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(got.float().abs().sum() > 0)
