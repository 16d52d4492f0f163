"""The base layer's operators on the GPU against the oracle: rows and weights in 8 bits, products, experts' products, routing, norms.

Bounds, from the arithmetic (a step of a rounding: eps / 2 of the type):
  codes      equal bytes, where the choice runs in 32 bits on the inputs; behind an activation or a norm the value is off by some units of
             32 bits first, so a code may be its neighbour: half a step of the code (2^-4 relative, 2^-10 scales below the normal codes) and that.
  products   products of codes are exact; each of the 128 additions inside a block loses at most 2^-23 of the block's sum of magnitudes, each
             of a row's blocks 3 roundings (two scales, one multiply-add) of 2^-24.
  norms      a sum of squares over 16384 channels is 64 additions a thread and 8 between threads: 72 * 2^-24 relative, the root halves it;
             the parts of hidden are 4 roundings and one for each expert's row.
"""
import numpy as np
import pytest

from oracle import base as O

pytestmark = pytest.mark.gpu

DT = {"bf16": (2.0 ** -8, "bfloat16"), "fp16": (2.0 ** -11, "float16"), "fp32": (2.0 ** -24, "float32")}
U = 2.0 ** -24


def lib():
    import paper_2512_20210_amd as P
    return P


def put(x, dtype="fp32"):
    """numpy -> GPU tensor of the element type, and what its elements are in 64 bits."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, DT[dtype][1])).cuda()
    return t, t.double().cpu().numpy()


def ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def empty_rows(n, k, wide=0):
    """Fp8Rows whose codes have `wide` bytes behind every row."""
    import torch
    codes = torch.full((n, k + wide), 0x55, device="cuda", dtype=torch.uint8)
    scales = torch.full((-(-k // 128), n + (3 if wide else 0)), 7.0, device="cuda")
    return lib().Fp8Rows(codes[:, :k], scales[:, :n]), codes, scales


def made_rows(rng, n, k):
    """Random rows in 8 bits: Fp8Rows and their values."""
    import torch
    x = rng.normal(size=(n, k)) * np.exp(rng.normal(size=(n, 1)))
    c, s = O.rows(x)
    return lib().Fp8Rows(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()), O.row_values(c, s)


def made_weights(rng, n, k, experts=None):
    import torch
    got = [O.weights(rng.normal(size=(n, k)) * np.exp(0.3 * rng.normal(size=(n, 1)))) for _ in range(experts or 1)]
    c, s = (np.stack([g[i] for g in got]) for i in (0, 1))
    v = np.stack([O.weight_values(*g) for g in got])
    if experts is None:
        c, s, v = c[0], s[0], v[0]
    return lib().Fp8Weights(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()), v


# ---- rows and weights in 8 bits -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,k", [(1, 8), (1, 4096), (3, 136), (17, 128), (33, 1000), (300, 264), (700, 4104), (2, 13824)])
def test_rows_of_values(dtype, n, k):
    import torch
    rng = np.random.default_rng(n * k)
    x = rng.normal(size=(n, k)) * np.exp(2 * rng.normal(size=(n, k)))
    x[0, :min(k, 128)] *= 1e-4
    x[-1, k // 2:k // 2 + 4] = 0
    t, x64 = put(x, dtype)
    c, s = O.rows(x64.astype(np.float32))
    for wide in (0, 24):
        r, codes, scales = empty_rows(n, k, wide)
        r.quantise(t, stream=stream())
        assert (codes[:, :k].cpu().numpy() == c).all() and (scales[:, :n].cpu().numpy() == s).all()
        assert (codes[:, k:] == 0x55).all() and (scales[:, n:] == 7).all()
    wide = torch.full((n, k + 8), float("nan"), device="cuda", dtype=t.dtype)
    wide[:, :k] = t
    r, codes, _ = empty_rows(n, k)
    r.quantise(wide[:, :k], stream=stream())
    assert (codes.cpu().numpy() == c).all()


def test_rows_of_values_that_are_not_ordinary():
    import torch
    x = np.zeros((9, 384), np.float32)
    x[0, 3], x[1, 130], x[2, 383], x[3, 0] = np.inf, -np.inf, np.nan, 3.4e38
    x[4, :128] = 2.0 ** -100
    x[5, :128] = 2.0 ** -101
    x[6, 128:256] = 1e-40
    x[7] = -0.0
    x[8, 5:9] = [448, 448 * (1 - 2.0 ** -24), -432, 2.0 ** -10]
    c, s = O.rows(x)
    r, codes, scales = empty_rows(9, 384)
    r.quantise(torch.from_numpy(x).cuda(), stream=stream())
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True) and (codes.cpu().numpy() == c).all()
    assert np.isnan(s).sum() == 3 and s[0, 5] == 0 and s[0, 4] > 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,k", [(1, 8), (5, 1000), (64, 2048), (600, 1384)])
def test_gated_rows(dtype, act, n, k):
    P = lib()
    rng = np.random.default_rng(n + k)
    x = rng.normal(size=(n, 2 * k)) * 3
    x[0, :8] = [-200, 200, 0, -0.0, 1e-3, -1e-3, 60, -60]
    t, x64 = put(x, dtype)
    y = O.activated(x64, act)
    r, codes, scales = empty_rows(n, k)
    r.quantise(t, {"silu": P.PLORA_ACT_SILU, "gelu": P.PLORA_ACT_GELU}[act], stream())
    # the exponential's argument z is rounded (gelu: 5 times) before it is taken: |z| * 2^-24 each, and 5 roundings behind it
    a = x64[:, :k]
    z = np.abs(a) if act == "silu" else np.abs(2 * 0.7978845608 * (a + 0.044715 * a ** 3))
    off = (np.where(z < 100, 6 * z, 0) + 8) * U * np.abs(y) + 1e-37
    c, s = codes.cpu().numpy(), scales.cpu().numpy().astype(np.float64)
    wide = np.repeat(s, 128, 0)[:k].T
    got = O.values(c) * wide
    # the largest |y| of a block and the largest slip in it: its scale
    pad = lambda v: np.pad(v, ((0, 0), (0, -k % 128))).reshape(n, -1, 128).max(-1).T  # noqa: E731
    assert (np.abs(s * 448 - pad(np.abs(y))) <= pad(off) + 2 * U * pad(np.abs(y))).all()
    assert (np.abs(got - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * wide + 1.1 * off + 4 * U * np.abs(y)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("experts,n,k", [(None, 8, 16), (None, 128, 128), (None, 136, 400), (3, 264, 1040), (None, 1000, 4096)])
def test_weights(dtype, experts, n, k):
    import torch
    P = lib()
    shape = (n, k) if experts is None else (experts, n, k)
    t, w64 = put(np.random.default_rng(n).normal(size=shape), dtype)
    codes = torch.full(shape, 0x55, device="cuda", dtype=torch.uint8)
    scales = torch.full((*shape[:-2], -(-n // 128), -(-k // 128)), float("nan"), device="cuda")
    P.Fp8Weights(codes, scales).quantise(t, stream())
    got_c, got_s, w = (v.reshape(-1, *v.shape[-2:]) for v in (codes.cpu().numpy(), scales.cpu().numpy(), w64))
    for e in range(experts or 1):
        c, s = O.weights(w[e].astype(np.float32))
        assert (got_c[e] == c).all() and (got_s[e] == s).all()


# ---- products -----------------------------------------------------------------------------------------

def product_bound(x, w, ref, dtype):
    kb = -(-x.shape[1] // 128)
    return DT[dtype][0] * np.abs(ref) + (128 * 2 + 3 * kb) * U * (np.abs(x) @ np.abs(w).T) + 1e-37


SIZES = [(1, 8, 16), (1, 4096, 4096), (2, 264, 144), (5, 1000, 2048), (16, 128, 128), (17, 136, 272), (33, 1024, 5120), (64, 72, 4096), (65, 512, 1040),
         (100, 2048, 400), (129, 264, 1552), (200, 5120, 512), (256, 1000, 1024), (300, 520, 13824), (513, 776, 2064), (1000, 4104, 272), (2100, 1288, 1168)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", SIZES)
def test_product(dtype, t, n, k):
    import torch
    rng = np.random.default_rng(t + n + k)
    x, xv = made_rows(rng, t, k)
    w, wv = made_weights(rng, n, k)
    ref = xv @ wv.T
    out = torch.full((t + 1, n + 8), 7.0, device="cuda", dtype=getattr(torch, DT[dtype][1]))
    w.matmul(x, out[:t, :n], stream())
    assert (np.abs(host(out[:t, :n]) - ref) <= product_bound(xv, wv, ref, dtype)).all()
    assert (out[t:] == 7).all() and (out[:, n:] == 7).all()


def test_product_of_rows_in_wider_ones():
    import torch
    P = lib()
    rng = np.random.default_rng(5)
    c, s = O.rows(rng.normal(size=(70, 400)))
    codes = torch.full((70, 432), 0x7f, device="cuda", dtype=torch.uint8)  # NaN behind every row
    codes[:, :400] = torch.from_numpy(c).cuda()
    scales = torch.full((4, 80), float("nan"), device="cuda")
    scales[:, :70] = torch.from_numpy(s).cuda()
    w, wv = made_weights(rng, 264, 400)
    xv = O.row_values(c, s)
    ref = xv @ wv.T
    out = torch.empty(70, 264, device="cuda")
    w.matmul(P.Fp8Rows(codes[:, :400], scales[:, :70]), out, stream())
    assert (np.abs(host(out) - ref) <= product_bound(xv, wv, ref, "fp32")).all()


@pytest.mark.parametrize("t", [1, 20, 64, 130, 300])
def test_nan_stays_in_its_row_and_channels(t):
    import torch
    P = lib()
    rng = np.random.default_rng(t)
    x = rng.normal(size=(t, 384)).astype(np.float32)
    x[t // 2, 200] = np.inf
    c, s = O.rows(x)
    r = P.Fp8Rows(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda())
    w, _ = made_weights(rng, 272, 384)
    out = torch.empty(t, 272, device="cuda", dtype=torch.bfloat16)
    bad = torch.isnan(w.matmul(r, out, stream()))
    assert bad[t // 2].all() and bad.sum() == 272
    x[t // 2, 200] = 1
    r.quantise(torch.from_numpy(x).cuda(), stream=stream())
    w.scales[1, 2] = float("nan")
    bad = torch.isnan(w.matmul(r, out, stream()))
    assert bad[:, 128:256].all() and not bad[:, :128].any() and not bad[:, 256:].any()


@pytest.mark.parametrize("t", [1, 40, 200, 600])
def test_a_row_does_not_depend_on_the_others_and_repeats(t):
    """The same bits again, and for rows whose neighbours change."""
    import torch
    rng = np.random.default_rng(t)
    x, _ = made_rows(rng, t, 1040)
    w, _ = made_weights(rng, 520, 1040)
    a, b = (torch.empty(t, 520, device="cuda") for _ in range(2))
    w.matmul(x, a, stream())
    w.matmul(x, b, stream())
    assert torch.equal(a, b)
    if t > 1:
        x.codes[:t // 2] = x.codes[:t // 2].flip(1)
        w.matmul(x, b, stream())
        assert torch.equal(a[t // 2:], b[t // 2:])


GROUPS = [([3], 8, 16), ([0, 5, 0, 1], 136, 272), ([1] * 9, 520, 400), ([40, 0, 3, 129, 64, 65, 0], 264, 1040), ([300, 20, 257], 520, 2048), ([0, 0, 700], 1032, 272),
          ([1, 2, 0] * 45, 72, 144), ([7] * 70, 136, 4096), ([0] * 6, 72, 144)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("sizes,n,k", GROUPS, ids=[str(i) for i in range(len(GROUPS))])
def test_grouped(dtype, gather, sizes, n, k):
    import torch
    P = lib()
    rng = np.random.default_rng(len(sizes) + n)
    total = sum(sizes)
    have = max(1, total // 2 if gather else total + 2)
    x, xv = made_rows(rng, have, k)
    w, wv = made_weights(rng, n, k, len(sizes))
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    rows = rng.integers(0, have, total + 2)
    if gather and total > 4:
        rows[1], rows[total - 2] = -1, have
    out = torch.full((total + 2, n), 7.0, device="cuda", dtype=getattr(torch, DT[dtype][1]))
    w.grouped(x if have >= total + 2 or gather else P.Fp8Rows(x.codes, x.scales), ints(offsets), out, ints(rows) if gather else None, stream())
    got = host(out)
    assert (got[total:] == 7).all()  # rows of no group
    for e in range(len(sizes)):
        for r in range(offsets[e], offsets[e + 1]):
            src = rows[r] if gather else r
            if not 0 <= src < have:
                assert np.isnan(got[r]).all()
                continue
            ref = xv[src] @ wv[e].T
            assert (np.abs(got[r] - ref) <= product_bound(xv[src][None], wv[e], ref, dtype)).all()


@pytest.mark.parametrize("offsets", [[0, -5, 40, 1000, 90], [-3, -1, 0, 0, 5], [10, 20, 20, 30, 2000000000], [50, 40, 30, 20, 10]])
def test_offsets_out_of_range(offsets):
    """Each is held to the rows there are; a group that ends ahead of its start is empty."""
    import torch
    rng = np.random.default_rng(1)
    x, xv = made_rows(rng, 90, 144)
    w, wv = made_weights(rng, 72, 144, 4)
    out = torch.full((90, 72), 7.0, device="cuda")
    w.grouped(x, ints(offsets), out, None, stream())
    held = np.clip(offsets, 0, 90)
    of = np.full(90, -1)
    claims = np.zeros(90, int)
    for e in range(4):
        of[held[e]:held[e + 1]] = e
        claims[held[e]:held[e + 1]] += 1
    got = host(out)
    for r in range(90):
        if claims[r] > 1:
            continue
        if of[r] < 0:
            assert (got[r] == 7).all()
        else:
            ref = xv[r] @ wv[of[r]].T
            assert (np.abs(got[r] - ref) <= product_bound(xv[r][None], wv[of[r]], ref, "fp32")).all()


# ---- routing ------------------------------------------------------------------------------------------

def routing(n, e, k):
    import torch
    P = lib()
    size = P.Routing.workspace_bytes(n, e)
    r = P.Routing(ints(np.full((n, k), -9)), torch.full((n, k), -9.0, device="cuda"), ints(np.full(e + 1, -9)), ints(np.full(n * k, -9)), ints(np.full((n, k), -9)),
                  torch.full((size,), 0xAB, device="cuda", dtype=torch.uint8) if size else None)
    return r


def check_route(r, logits64, k, renormalise, scale):
    e, w, o, rows, p = O.route(logits64, k, renormalise, scale)
    assert (r.experts.cpu().numpy() == e).all()
    assert (r.offsets.cpu().numpy() == o).all()
    assert (r.places.cpu().numpy() == p).all()
    assert (r.rows.cpu().numpy() == rows).all()
    got = host(r.weights)
    assert (np.isnan(got) == np.isnan(w)).all()
    # p's exponent d is rounded, |d| 2^-24, the exponential 2 units; a sum of up to 22 additions, a quotient, a product
    x = np.where(np.isfinite(logits64), logits64, 0)
    off = (2 * (x.max(1) - x.min(1)) + 40) * U
    ok = ~np.isnan(w)
    assert (np.abs(got - w)[ok] <= (off[:, None] * np.abs(w) + 1e-38)[ok]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (1, 8, 2), (5, 64, 6), (63, 65, 8), (64, 256, 8), (65, 64, 4), (130, 7, 7), (300, 128, 32), (1000, 512, 3),
                                   (700, 1024, 8), (4097, 60, 2), (5000, 200, 6)])
def test_routing(dtype, n, e, k):
    import torch
    rng = np.random.default_rng(n + e + k)
    x = np.round(rng.normal(size=(n, e)) * 4) / 4 if dtype == "bf16" else rng.normal(size=(n, e)) * 2  # bf16: many ties
    x[rng.random(n) < 0.15] = -np.inf
    if e > 4:
        x[rng.random((n, e)) < 0.05] = -np.inf
        x[n // 2, 1:] = -np.inf
        x[n // 3, e // 2] = np.nan
        x[n // 4, e // 3] = np.inf
    t, x64 = put(x, dtype)
    r = routing(n, e, k)
    r.route(t, True, 1.0, stream())
    check_route(r, x64, k, True, 1.0)
    wide = torch.full((n, e + 3), 50.0, device="cuda", dtype=t.dtype)
    wide[:, 1:e + 1] = t
    r = routing(n, e, k)
    r.route(wide[:, 1:e + 1], False, 2.5, stream())
    check_route(r, x64, k, False, 2.5)


def test_routing_of_no_tokens():
    import torch
    P = lib()
    r = P.Routing(ints(np.zeros((0, 2))), torch.zeros(0, 2, device="cuda"), ints([5] * 9), ints([]), ints(np.zeros((0, 2))))
    r.route(torch.zeros(0, 8, device="cuda"), stream=stream())
    assert (r.offsets == 0).all()


@pytest.mark.parametrize("chunks", [64, 65, 300])
def test_routing_over_many_chunks(chunks):
    """Both ways in which the chunks' counts are summed, at the size where they change: against torch's stable sort."""
    import torch
    n, e, k = chunks * 64 - 5, 33, 3
    g = torch.Generator(device="cuda").manual_seed(chunks)
    x = torch.randn(n, e, device="cuda", generator=g)
    r = routing(n, e, k)
    r.route(x, stream=stream())
    best = torch.sort(x, descending=True, stable=True)[1][:, :k]
    assert torch.equal(r.experts.long(), best)
    order = torch.sort(best.reshape(-1), stable=True)[1]
    assert torch.equal(r.rows.long(), order // k)
    assert torch.equal(r.places.reshape(-1).long()[order], torch.arange(n * k, device="cuda"))
    assert torch.equal(r.offsets[1:].long(), torch.bincount(best.reshape(-1), minlength=e).cumsum(0)) and r.offsets[0] == 0


# ---- norms between blocks -----------------------------------------------------------------------------

def norm_case(rng, dtype, n, d, top_k=0, residual=True, gate=None, post=None, pre=None, scale=1.0, block_rows=None):
    """Inputs on the GPU and the results in 64 bits with their bounds: (kwargs of run, BlockNorm, hidden, y, bound of hidden, bound of y)."""
    P = lib()
    m = n if not top_k else (block_rows if block_rows is not None else n * top_k)
    block, b64 = put(rng.normal(size=(m, d)) * 3, dtype)
    kw = dict(block=block)
    mag = np.abs(b64)
    if top_k:
        places = rng.integers(-1, m + 1, (n, top_k))
        pw = rng.random((n, top_k)).astype(np.float32)
        pw[(places < 0) | (places >= m)] = np.nan
        kw.update(places=ints(places), place_weights=put(pw)[0])
        u, mag = O.gathered(b64, places, pw), O.gathered(mag, places, pw)
    else:
        u = b64
    du = (top_k + 1) * U * mag
    make = {}
    for name, spec in (("post", post), ("pre", pre)):
        if spec is None:
            make[name] = (None, None)
            continue
        opt = dict(spec)
        w, w64 = put(1 + 0.3 * rng.normal(size=d), dtype) if opt.pop("weight", True) else (None, None)
        b, bias64 = put(rng.normal(size=d), dtype) if opt.pop("bias", False) else (None, None)
        make[name] = (P.NormWeights(w, b, **opt), dict(weight=w64, bias=bias64, **opt))

    def applied(v, dv, o):
        y = O.norm(v, **o)
        if o.get("center"):
            dv = dv + 75 * U * np.abs(v).mean(-1, keepdims=True) + U * np.abs(v)
            v = v - v.mean(-1, keepdims=True)
        ms = (v * v).mean(-1, keepdims=True) + o["eps"]
        f = 1.0 if o["weight"] is None else np.abs(o.get("offset", 0.0) + o["weight"])
        z = np.abs(v) / np.sqrt(ms) * f
        # the row's own error moves the mean square too: at most the relative 2-norm of it
        rel = np.sqrt((dv * dv).mean(-1, keepdims=True) / ms) + 45 * U
        return y, dv / np.sqrt(ms) * f + rel * z + 4 * U * (z + np.abs(y))

    if post is not None:
        u, du = applied(u, du, make["post"][1])
    h, dh = scale * u, abs(scale) * (du + U * np.abs(u))
    if gate is not None:
        g, g64 = put(rng.normal(size=(n, d) if gate == "rows" else d), dtype)
        kw["gate"] = g
        h, dh = h * g64, dh * np.abs(g64) + U * np.abs(h * g64)
    if residual:
        r, r64 = put(rng.normal(size=(n, d)) * 5, dtype)
        kw["residual"] = r
        h = h + r64
        dh = dh + U * np.abs(h)
    y, dy = applied(h, dh, make["pre"][1]) if pre is not None else (h, dh)
    return kw, P.BlockNorm(make["pre"][0], make["post"][0], scale), h, y, dh, dy


RMS = dict(eps=1e-6)
LAYER = dict(eps=1e-5, center=True, bias=True)
NORMS = [(1, 8, dict(pre=RMS)), (1, 4096, dict(pre=RMS)), (5, 128, dict(pre=dict(eps=1e-6, offset=1.0), gate="rows")), (7, 136, dict(pre=LAYER, post=LAYER, gate="one", scale=0.5)),
         (33, 264, dict(pre=RMS, post=RMS, residual=False)), (9, 520, dict(post=RMS, gate="rows", scale=-2.0)), (4, 1032, dict(pre=dict(eps=1e-6, weight=False), top_k=2)),
         (3, 2048, dict(pre=LAYER, top_k=8)), (18, 4104, dict(pre=RMS, post=LAYER, top_k=1)), (2, 6152, dict(pre=RMS, post=RMS, gate="rows", top_k=3)),
         (5, 8200, dict(pre=LAYER, post=RMS, gate="rows")), (2, 16384, dict(pre=LAYER, post=LAYER, gate="rows", top_k=5)), (300, 64, dict(pre=RMS)), (1030, 40, dict(pre=LAYER, top_k=4)),
         (6, 5120, dict()), (3, 1000, dict(top_k=3, block_rows=1, residual=False))]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,d,spec", NORMS, ids=["%dx%d" % c[:2] for c in NORMS])
def test_norm(dtype, n, d, spec):
    import torch
    rng = np.random.default_rng(n * d)
    kw, norm, h, y, dh, dy = norm_case(rng, dtype, n, d, **spec)
    dt = kw["block"].dtype
    eps = DT[dtype][0]
    hidden, out = (torch.full((n + 1, d + 8), 7.0, device="cuda", dtype=dt) for _ in range(2))
    norm.run(hidden=hidden[:n, :d], out=out[:n, :d], stream=stream(), **kw)
    assert (np.abs(host(hidden[:n, :d]) - h) <= dh + eps * (np.abs(h) + dh) + 2.0 ** -25).all()
    assert (np.abs(host(out[:n, :d]) - y) <= dy + eps * (np.abs(y) + dy) + 2.0 ** -25).all()  # (fp16: half a step of its smallest)
    for t in (hidden, out):
        assert (t[n:] == 7).all() and (t[:, d:] == 7).all()
    # in 8 bits, hidden in place of the residual (or not written)
    r, codes, scales = empty_rows(n, d, 8)
    inplace = kw["residual"].clone() if "residual" in kw else None
    norm.run(**{**kw, "residual": inplace}, hidden=inplace, out8=r, stream=stream())
    if inplace is not None:
        assert torch.equal(inplace, hidden[:n, :d])
    s = scales[:, :n].cpu().numpy().astype(np.float64)
    wide = np.repeat(s, 128, 0)[:d].T
    got = O.values(codes[:, :d].cpu().numpy()) * wide
    assert (np.abs(got - y) <= 2.0 ** -4 * (np.abs(y) + dy) + 2.0 ** -10 * wide + dy + 4 * U * np.abs(y)).all()
    top = np.pad(np.abs(y), ((0, 0), (0, -d % 128))).reshape(n, -1, 128).max(-1).T
    slip = np.pad(dy, ((0, 0), (0, -d % 128))).reshape(n, -1, 128).max(-1).T
    assert (np.abs(448 * s - top) <= slip + 2 * U * top).all()
    assert (codes[:, d:] == 0x55).all() and (scales[:, n:] == 7).all()


def test_norm_in_place_of_the_block_and_rows_with_nan():
    import torch
    P = lib()
    rng = np.random.default_rng(2)
    block, b = put(rng.normal(size=(6, 264)), "fp16")
    block[3, 7] = float("nan")
    norm = P.BlockNorm(P.NormWeights())
    want = torch.empty_like(block)
    norm.run(block, out=want, stream=stream())
    r, codes, scales = empty_rows(6, 264)
    norm.run(block, out8=r, stream=stream())
    norm.run(block, out=block, stream=stream())
    assert torch.equal(block.view(torch.int16), want.view(torch.int16))
    assert torch.isnan(block[3]).all() and torch.isnan(block).sum() == 264
    assert torch.isnan(scales[:, 3]).all() and torch.isnan(scales).sum() == 3


def test_no_rows():
    import torch
    P = lib()
    e = torch.empty(0, 64, device="cuda")
    P.BlockNorm().run(e, hidden=e, stream=stream())
    r = P.Fp8Rows(torch.empty(0, 64, device="cuda", dtype=torch.uint8), torch.empty(1, 0, device="cuda"))
    r.quantise(e, stream=stream())
    w, _ = made_weights(np.random.default_rng(0), 8, 64, 2)
    w.grouped(r, ints([0, 0, 0]), torch.empty(0, 8, device="cuda"), None, stream())
