"""Every kernel of the 8-bit products in every type, over few blocks of K and over many (base_tiles.py), against 64 bits.  Bounds as in test_gpu_base.py; the
reference and the bound are products in 64 bits on the GPU."""
import numpy as np
import pytest

import test_gpu_base as B
from base_tiles import EXPERTS, calls

pytestmark = pytest.mark.gpu


def codes_of(gen, *shape):
    """All codes but NaN alike, and the values that they stand for in 64 bits."""
    import torch
    codes = torch.randint(0, 254, shape, generator=gen, device="cuda", dtype=torch.uint8)
    codes += (codes > 126).to(torch.uint8)  # 0 .. 126, 128 .. 254
    every = np.arange(256)
    return codes, torch.from_numpy(B.O.values(np.where(every % 128 == 127, 0, every))).cuda()


def scales_of(gen, *shape):
    import torch
    return torch.exp(torch.randn(*shape, generator=gen, device="cuda"))


def check(got, x, w, dtype):
    """test_gpu_base.product_bound's terms, on the GPU."""
    import torch
    ref = x @ w.t()
    eps = B.DT[dtype][0]
    off = eps * ref.abs() + (128 * 2 + 3 * -(-x.shape[1] // 128)) * B.U * (x.abs() @ w.abs().t()) + 1e-37
    if dtype == "fp16":
        off += 2.0 ** -25
    if dtype != "fp32":
        gx, gw = (v.abs().view(len(v), -1, 8).amax(-1) for v in (x, w))
        off += 7 * 2.0 ** -13 * (gx @ gw.t()) * (1 + eps)
    got = got.double()
    if dtype == "fp16":  # as in test_gpu_base.check_product: from 65520 on, the middle behind fp16's largest value, a rounding gives inf
        over = torch.isinf(got)
        assert bool((ref.abs() + off >= 65520)[over].all() and (torch.sign(got) == torch.sign(ref))[over].all() and (ref.abs() - off < 65520)[~over].all())
        got, ref, off = (v.masked_fill(over, 0) for v in (got, ref, off))
    assert bool(((got - ref).abs() <= off).all())
    if dtype != "fp32":
        assert float(torch.linalg.norm(got - ref)) <= eps * float(torch.linalg.norm(ref))


def rows_and_values(gen, t, k):
    codes, table = codes_of(gen, t, k)
    s = scales_of(gen, -(-k // 128), t) / (30 * k)  # (fp16: results stay in range)
    return codes, s, table[codes.long()] * s.double().repeat_interleave(128, 0)[:k].t()


def weight_values(table, codes, s):
    n, k = codes.shape
    return table[codes.long()] * s.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kernel,t,n,k", calls(False))
def test_products(dtype, kernel, t, n, k):
    import torch
    P = B.lib()
    gen = torch.Generator(device="cuda").manual_seed(t * n + k)
    xc, xs, xv = rows_and_values(gen, t, k)
    wc, table = codes_of(gen, n, k)
    ws = scales_of(gen, -(-n // 128), -(-k // 128))
    out = torch.full((t + 1, n + 8), 7.0, device="cuda", dtype=getattr(torch, B.DT[dtype][1]))
    w, x = P.Fp8Weights(wc, ws), P.Fp8Rows(xc, xs)
    w.matmul(x, out[:t, :n], B.stream())
    assert bool((out[t:] == 7).all() and (out[:, n:] == 7).all())
    check(out[:t, :n], xv, weight_values(table, wc, ws), dtype)
    again = torch.empty(t, n, device="cuda", dtype=out.dtype)
    assert torch.equal(w.matmul(x, again, B.stream()), out[:t, :n])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kernel,t,n,k", calls(True))
def test_products_by_expert(dtype, kernel, t, n, k):
    """One expert with half of the rows, one with none; rows gathered (some not there) and not."""
    import torch
    P = B.lib()
    gen = torch.Generator(device="cuda").manual_seed(t * n + k)
    xc, xs, xv = rows_and_values(gen, t, k)
    wc, table = codes_of(gen, EXPERTS, n, k)
    ws = scales_of(gen, EXPERTS, -(-n // 128), -(-k // 128))
    w, x = P.Fp8Weights(wc, ws), P.Fp8Rows(xc, xs)
    offsets = [0, 1, 1 + t // 2, 1 + t // 2, 3 + t // 2, t]
    rows = torch.randint(0, t, (t,), generator=gen, device="cuda", dtype=torch.int32)
    rows[t // 3], rows[t - 1] = -1, t
    for r in (None, rows):
        out = torch.full((t, n + 8), 7.0, device="cuda", dtype=getattr(torch, B.DT[dtype][1]))
        w.grouped(x, B.ints(offsets), out[:, :n], r, B.stream())
        assert bool((out[:, n:] == 7).all())
        there = torch.ones(t, dtype=torch.bool, device="cuda") if r is None else (r >= 0) & (r < t)
        assert bool(torch.isnan(out[~there, :n]).all())
        source = xv if r is None else xv[r.clamp(0, t - 1).long()]
        for e in range(EXPERTS):
            a, b = offsets[e], offsets[e + 1]
            if a < b:
                mine = there[a:b]
                check(out[a:b, :n][mine], source[a:b][mine], weight_values(table, wc[e], ws[e]), dtype)
