"""The base layer's operators on the GPU against the oracle: rows and weights in 8 bits, products, experts' products, routing, norms.

Bounds, from the arithmetic (a step of a rounding: eps / 2 of the type):
  codes      equal bytes, where the choice runs in 32 bits on the inputs; behind an activation or a norm the value is off by some units of
             32 bits first, so a code may be its neighbour: half a step of the code (2^-4 relative, 2^-10 scales below the normal codes) and that.
  products   products of codes are exact.  fp32: each of the 128 additions inside a block loses at most 2^-23 of the block's sum of magnitudes.
             16-bit types: of 8 neighbouring products the matrix unit keeps the bits down to 2^-13 of the largest one's power of two, so each of the
             7 others loses less than 2^-13 of the largest; the 16 sums of 8 are added as above.  Each of a row's blocks has 3 roundings
             (two scales, one multiply-add) of 2^-24.  As a 2-norm the error stays below what the results' own rounding may have at most.
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
    off = DT[dtype][0] * np.abs(ref) + (128 * 2 + 3 * kb) * U * (np.abs(x) @ np.abs(w).T) + 1e-37
    if dtype == "fp16":
        off += 2.0 ** -25  # half a step of its smallest values
    if dtype != "fp32":
        gx, gw = (np.abs(v).reshape(len(v), -1, 8).max(-1) for v in (x, w))  # k is a multiple of 16
        off += 7 * 2.0 ** -13 * (gx @ gw.T) * (1 + DT[dtype][0])
    return off


def check_product(got, x, w, dtype):
    ref = x @ w.T
    off = product_bound(x, w, ref, dtype)
    if dtype == "fp16":  # 65520 is the middle between fp16's largest value and the power of two behind it: from there on a rounding gives inf
        over = np.isinf(got)
        assert (np.abs(ref) + off >= 65520)[over].all() and (np.sign(got) == np.sign(ref))[over].all() and (np.abs(ref) - off < 65520)[~over].all()
        got, ref, off = (np.where(over, 0, v) for v in (got, ref, off))
    assert (np.abs(got - ref) <= off).all()
    if dtype != "fp32":
        assert np.linalg.norm(got - ref) <= DT[dtype][0] * np.linalg.norm(ref)


SIZES = [(1, 8, 16), (1, 4096, 4096), (2, 264, 144), (5, 1000, 2048), (16, 128, 128), (17, 136, 272), (33, 1024, 5120), (64, 72, 4096), (65, 512, 1040),
         (100, 2048, 400), (129, 264, 1552), (200, 5120, 512), (256, 1000, 1024), (300, 520, 13824), (513, 776, 2064), (1000, 4104, 272), (2100, 1288, 1168)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", SIZES)
def test_product(dtype, t, n, k):
    import torch
    rng = np.random.default_rng(t + n + k)
    x, xv = made_rows(rng, t, k)
    w, wv = made_weights(rng, n, k)
    out = torch.full((t + 1, n + 8), 7.0, device="cuda", dtype=getattr(torch, DT[dtype][1]))
    w.matmul(x, out[:t, :n], stream())
    check_product(host(out[:t, :n]), xv, wv, dtype)
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
    out = torch.empty(70, 264, device="cuda")
    w.matmul(P.Fp8Rows(codes[:, :400], scales[:, :70]), out, stream())
    check_product(host(out), xv, wv, "fp32")


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
            check_product(got[r][None], xv[src][None], wv[e], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(7, 520, 13840), (16, 16392, 2576), (3, 32776, 1040), (12, 32776, 144)])
def test_few_rows_of_many_blocks_or_channels(dtype, t, n, k):
    test_product(dtype, t, n, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("k", [16, 528, 1408, 1424])
def test_many_experts_of_few_blocks(dtype, k):
    """Two wavefronts share K up to 1408 values, then four."""
    test_grouped(dtype, k != 528, [int(v) for v in np.random.default_rng(k).integers(0, 10, 40)], 1032, k)


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
            check_product(got[r][None], xv[r][None], wv[of[r]], "fp32")


def random_codes(rng, *shape):
    """All codes but NaN alike: sizes over 16 powers of two."""
    c = rng.integers(0, 127, shape, dtype=np.uint8)
    return c | (rng.integers(0, 2, shape, dtype=np.uint8) << 7)


# rows, channels, values: each of the kernels that the rule chooses from (few rows: 3, tiles: 8), and an odd end everywhere
KINDS = [(9, 72, 528), (9, 4104, 528), (9, 72, 144), (17, 72, 2064), (2070, 264, 4112), (17, 72, 144), (2070, 520, 2064), (1500, 2056, 144), (1030, 5128, 144),
         (2070, 2056, 2064), (1030, 7176, 144)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", KINDS)
def test_product_of_each_kernel(dtype, t, n, k):
    import torch
    P = lib()
    rng = np.random.default_rng(t * n + k)
    xc, wc = random_codes(rng, t, k), random_codes(rng, n, k)
    xs, ws = (np.exp(rng.normal(size=z)).astype(np.float32) for z in ((-(-k // 128), t), (-(-n // 128), -(-k // 128))))
    put_ = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    out = torch.full((t + 1, n + 8), 7.0, device="cuda", dtype=torch.float32 if dtype == "fp32" else getattr(torch, DT[dtype][1]))
    xs /= 30 * k  # (fp16: results stay in range)
    P.Fp8Weights(put_(wc), put_(ws)).matmul(P.Fp8Rows(put_(xc), put_(xs)), out[:t, :n], stream())
    got = host(out)
    assert (got[t:] == 7).all() and (got[:, n:] == 7).all()
    check_product(got[:t, :n], O.row_values(xc, xs), O.weight_values(wc, ws), dtype)


GROUPED_KINDS = [(9, 72, 528), (9, 1032, 528), (9, 72, 144), (100, 72, 2064), (100, 2056, 4112), (100, 72, 144), (413, 2056, 2064), (1500, 2056, 144), (257, 13832, 144),
                 (600, 5128, 2064), (413, 13832, 144)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,n,k", GROUPED_KINDS)
def test_grouped_of_each_kernel(dtype, t, n, k):
    """Five experts, one of them with half of the rows, one with none; rows gathered and not."""
    import torch
    P = lib()
    rng = np.random.default_rng(t * n + k)
    xc, wc = random_codes(rng, t, k), random_codes(rng, 5, n, k)
    xs, ws = (np.exp(rng.normal(size=z)).astype(np.float32) for z in ((-(-k // 128), t), (5, -(-n // 128), -(-k // 128))))
    xs /= 30 * k
    put_ = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    x, w = P.Fp8Rows(put_(xc), put_(xs)), P.Fp8Weights(put_(wc), put_(ws))
    offsets = np.array([0, 1, 1 + t // 2, 1 + t // 2, 3 + t // 2, t])
    rows = rng.integers(0, t, t)
    xv = O.row_values(xc, xs)
    for r in (None, rows):
        out = torch.full((t, n), 7.0, device="cuda", dtype=getattr(torch, DT[dtype][1]))
        w.grouped(x, ints(offsets), out, None if r is None else ints(r), stream())
        got = host(out)
        for e in range(5):
            a, b = offsets[e], offsets[e + 1]
            if a < b:
                check_product(got[a:b], xv[a:b] if r is None else xv[r[a:b]], O.weight_values(wc[e], ws[e]), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(413, 7176, 144), (257, 7176, 1040), (600, 13832, 144)])
def test_product_of_more_kernels(dtype, t, n, k):
    """Tiles of 64 x 128, 128 x 128 and the largest (fp32: 256 x 128)."""
    test_product_of_each_kernel(dtype, t, n, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(9, 2056, 528), (316, 1032, 8208), (413, 4104, 1040), (600, 7176, 144), (1030, 4104, 2064), (1030, 7176, 144)])
def test_grouped_of_more_kernels(dtype, t, n, k):
    """Few rows x 32 channels, tiles of 64 x 64 with two sets, 128 x 128, 128 x 256, 256 x 128 and the largest (fp32: another one)."""
    test_grouped_of_each_kernel(dtype, t, n, k)


def test_one_expert_of_very_many_rows():
    """More rows than 32-bit floats count (the rule's sizes of groups)."""
    import torch
    P = lib()
    rng = np.random.default_rng(12)
    total, k, n = (1 << 25) + 8, 16, 8
    xc, wc = random_codes(rng, 64, k), random_codes(rng, 1, n, k)
    codes = torch.from_numpy(xc).cuda().repeat(total // 64 + 1, 1)[:total].contiguous()
    w = P.Fp8Weights(torch.from_numpy(wc).cuda(), torch.ones(1, 1, 1, device="cuda"))
    out = torch.zeros(total, n, device="cuda")
    w.grouped(P.Fp8Rows(codes, torch.ones(1, total, device="cuda")), ints([0, total]), out, stream=stream())
    expected = O.row_values(xc, np.ones((1, 64), np.float32))
    check_product(host(out[:64]), expected, O.weight_values(wc[0], np.ones((1, 1), np.float32)), "fp32")
    assert (out[64:] == out[:64].repeat(total // 64, 1)[:total - 64]).all()


def test_rows_far_apart():
    """x's rows behind 2 and 4 GiB, and results behind 4 GiB."""
    import torch
    P = lib()
    rng = np.random.default_rng(8)
    n, k, total, step = 136, 272, 5000, 1 << 20
    codes = torch.empty(total, step, device="cuda", dtype=torch.uint8)
    pick = np.concatenate([rng.integers(0, total, 30), [0, 2047, 2048, 4095, 4096, total - 1]])
    xc, xs = random_codes(rng, total, k), np.exp(rng.normal(size=(3, total))).astype(np.float32)
    codes[:, :k] = torch.from_numpy(xc).cuda()
    x = P.Fp8Rows(codes[:, :k], torch.from_numpy(xs).cuda())
    xv = O.row_values(xc, xs)
    w, wv = made_weights(rng, n, k, 2)
    wide = torch.empty(len(pick), 1 << 26, device="cuda")  # 256 MiB a row
    w.grouped(x, ints([0, 20, len(pick)]), wide[:, :n], ints(pick), stream())
    got = host(wide[:, :n])
    check_product(got[:20], xv[pick[:20]], wv[0], "fp32")
    check_product(got[20:], xv[pick[20:]], wv[1], "fp32")
    one = P.Fp8Weights(w.codes[0], w.scales[0])
    out = torch.empty(total, n, device="cuda", dtype=torch.bfloat16)
    one.matmul(x, out, stream())
    check_product(host(out), xv, wv[0], "bf16")
    few = codes[::625]  # 8 rows, 655 MB from one to the next
    few.copy_(codes[:8])
    out = torch.empty(8, n, device="cuda")
    one.matmul(P.Fp8Rows(few[:, :k], x.scales[:, :8]), out, stream())
    check_product(host(out), xv[:8], wv[0], "fp32")
    many = codes.view(-1, 1 << 23)[:600, :k]  # 600 rows, 8 MiB from one to the next: a tile's rows pass 2 GiB
    many.copy_(torch.from_numpy(xc[:600]).cuda())
    out = torch.empty(600, n, device="cuda")
    one.matmul(P.Fp8Rows(many, x.scales[:, :600]), out, stream())
    check_product(host(out), xv[:600], wv[0], "fp32")


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
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (1, 8, 2), (5, 64, 6), (63, 65, 8), (64, 256, 8), (65, 64, 4), (130, 7, 7), (300, 128, 32), (200, 130, 9), (256, 1024, 2), (257, 16, 16), (1, 513, 8), (64, 512, 8), (64, 1000, 32), (1100, 300, 17), (1000, 512, 3),
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


@pytest.mark.parametrize("e", [8, 1000])
def test_routing_of_no_tokens(e):
    import torch
    P = lib()
    r = P.Routing(ints(np.zeros((0, 2))), torch.zeros(0, 2, device="cuda"), ints([5] * (e + 1)), ints([]), ints(np.zeros((0, 2))))
    r.route(torch.zeros(0, e, device="cuda"), stream=stream())
    assert (r.offsets == 0).all()


@pytest.mark.parametrize("chunks", [15, 16, 17, 64, 300])
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


def test_one_row_of_a_wider_tensor():
    """A row cut out of a tensor whose width is no multiple of 16 bytes: its stride does not matter."""
    import torch
    P = lib()
    rng = np.random.default_rng(4)
    wide, w64 = put(rng.normal(size=(1, 403)), "bf16")
    x = wide[:, :400]
    out = torch.empty(1, 413, device="cuda", dtype=torch.bfloat16)[:, :400]
    P.BlockNorm(P.NormWeights()).run(x, out=out, stream=stream())
    ref = O.norm(w64[:, :400])
    assert (np.abs(host(out) - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5).all()
    r, codes, scales = empty_rows(1, 400)
    r.quantise(x, stream=stream())
    c, s = O.rows(w64[:, :400].astype(np.float32))
    assert (codes.cpu().numpy() == c).all() and (scales.cpu().numpy() == s).all()
    w, wv = made_weights(rng, 264, 400)
    y = torch.empty(1, 271, device="cuda")[:, :264]
    w.matmul(r, y, stream())
    check_product(host(y), O.row_values(c, s), wv, "fp32")


def test_wrappers_refuse():
    """Tensors that are not on the GPU, of other types, sizes or strides."""
    import torch
    P = lib()
    f = lambda *z, d=torch.bfloat16: torch.zeros(*z, device="cuda", dtype=d)  # noqa: E731
    i = lambda *z: torch.zeros(*z, device="cuda", dtype=torch.int32)  # noqa: E731
    u8 = torch.uint8
    rows = P.Fp8Rows(f(4, 256, d=u8), f(2, 4, d=torch.float32))
    w = P.Fp8Weights(f(264, 256, d=u8), f(3, 2, d=torch.float32))
    ws = P.Fp8Weights(f(2, 264, 256, d=u8), f(2, 3, 2, d=torch.float32))
    route = P.Routing(i(4, 2), f(4, 2, d=torch.float32), i(9), i(8), i(4, 2))
    norm = P.BlockNorm(P.NormWeights(f(256)))
    x = f(4, 256)
    bad = [
        lambda: P.Fp8Rows(f(4, 256, d=u8), f(2, 5, d=torch.float32)), lambda: P.Fp8Rows(f(4, 256, d=u8), f(3, 4, d=torch.float32)),
        lambda: P.Fp8Rows(f(4, 256), f(2, 4, d=torch.float32)), lambda: P.Fp8Rows(f(4, 512, d=u8)[:, ::2], f(2, 4, d=torch.float32)),
        lambda: P.Fp8Rows(f(4, 256, d=u8), f(2, 4)), lambda: P.Fp8Rows(f(4, 256, d=u8).cpu(), f(2, 4, d=torch.float32)),
        lambda: P.Fp8Weights(f(264, 256, d=u8), f(2, 2, d=torch.float32)), lambda: P.Fp8Weights(f(264, 512, d=u8)[:, :256], f(3, 2, d=torch.float32)),
        lambda: rows.quantise(x.cpu()), lambda: rows.quantise(f(4, 264)), lambda: rows.quantise(x, P.PLORA_ACT_SILU), lambda: rows.quantise(f(4, 256, d=torch.float64)),
        lambda: rows.quantise(x, 7), lambda: w.quantise(f(264, 512)[:, :256]), lambda: w.quantise(f(264, 264)),
        lambda: w.matmul(rows, f(4, 256)), lambda: w.matmul(rows, f(5, 264)), lambda: w.matmul(rows, f(4, 264).cpu()), lambda: ws.matmul(rows, f(4, 264)),
        lambda: w.matmul(P.Fp8Rows(f(4, 272, d=u8), f(3, 4, d=torch.float32)), f(4, 264)), lambda: w.matmul(rows, f(4, 268)[:, :264]),
        lambda: ws.grouped(rows, i(2), f(4, 264)), lambda: ws.grouped(rows, i(3).long(), f(4, 264)), lambda: ws.grouped(rows, i(3), f(5, 264)),
        lambda: ws.grouped(rows, i(3), f(8, 264), i(7)), lambda: ws.grouped(rows, i(3).cpu(), f(4, 264)),
        lambda: route.route(f(4, 9)), lambda: route.route(f(5, 8)), lambda: route.route(f(4, 8).cpu()), lambda: P.Routing(i(4, 2), f(4, 2), i(9), i(8), i(4, 2)),
        lambda: P.Routing(i(4, 2), f(4, 2, d=torch.float32), i(9), i(7), i(4, 2)), lambda: P.Routing(i(4, 9), f(4, 9, d=torch.float32), i(9), i(36), i(4, 9)).route(f(4, 8)),
        lambda: P.Routing(i(70, 2), f(70, 2, d=torch.float32), i(9), i(140), i(70, 2)).route(f(70, 8)),  # no workspace
        lambda: norm.run(x), lambda: norm.run(x, out=f(4, 264)), lambda: norm.run(x, out=f(4, 256, d=torch.float16)), lambda: norm.run(x, out=x.cpu()),
        lambda: norm.run(f(4, 264), out=f(4, 264)), lambda: norm.run(x, out=f(4, 256), out8=rows), lambda: norm.run(x, out=f(4, 256), residual=f(3, 256)),
        lambda: norm.run(x, out=f(2, 256), places=i(2, 2)), lambda: norm.run(x, out=f(4, 256), place_weights=f(4, 2, d=torch.float32)),
        lambda: norm.run(x, out=x, places=i(4, 2), place_weights=f(4, 2, d=torch.float32)), lambda: norm.run(x, hidden=x, out=x),
        lambda: P.NormWeights(f(256), f(255)), lambda: P.NormWeights(f(256), f(256, d=torch.float16)), lambda: P.NormWeights(f(512)[::2]),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(P.PloraError):
            call()
            print("call %d was not refused" % n)
