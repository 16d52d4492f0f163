"""Rotary positions, the paged 4-bit KV cache and attention over it, on the GPU against the oracle's 64 bits.

Bounds, from the arithmetic: a rotation is two products and a sum in fp32 (3 roundings of at most |a| + |b| each), then one
rounding to the element type.  The cache's bytes are the choice that fp32 makes with one rounding per operation, so they are
compared for equality with the same choice on the CPU.  Attention rounds each weight to 11 bits (22 in fp32), so an output moves by at
most that much of sum(weight * |values|); logits are sums of 32-bit products (and a rotated q is held to 11 bits where the type
has 8), so a weight's relative error is at most that of its logit, whose terms add up to X; then one rounding to the
element type.
"""
import numpy as np
import pytest

from oracle import kv as O

pytestmark = pytest.mark.gpu

DT = {"bf16": (2.0 ** -8, "bfloat16"), "fp16": (2.0 ** -11, "float16"), "fp32": (2.0 ** -24, "float32")}  # most relative error of one rounding


def lib():
    import paper_2512_20210_amd as P
    return P


def code_of(dtype):
    P = lib()
    return {"bf16": P.PLORA_BF16, "fp16": P.PLORA_F16, "fp32": P.PLORA_F32}[dtype]


def put(x, dtype):
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


def table_of(rot, positions, **kw):
    import torch
    cs = O.angles(O.frequencies(rot, **kw), np.arange(positions)).astype(np.float32)
    return torch.from_numpy(cs).cuda(), cs


# ---- rotation -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("name,kw", [("NONE", {}), ("LINEAR", dict(factor=4.0)), ("NTK", dict(factor=8.0)),
                                     ("TURNS", dict(factor=8.0, low=1.0, high=4.0, original_len=8192))])
@pytest.mark.parametrize("rot,n", [(2, 5), (20, 33), (128, 70001)])
def test_angle_table(name, kw, rot, n):
    import torch
    P = lib()
    if name == "NTK" and rot == 2:
        kw, name = {}, "NONE"
    table = torch.full((n, rot // 2, 2), float("nan"), device="cuda")
    P.Rotary.make(table, P.RotaryConfig(base=50000.0, magnitude=1.25, scaling=getattr(P, "PLORA_ROTARY_" + name), **kw), stream=stream())
    ref = O.angles(O.frequencies(rot, base=50000.0, scaling=name.lower(), **kw), np.arange(n), 1.25)
    # one rounding of values up to 1.25, and angles in 64 bits: at most 70001 * 2^-51 off
    assert np.abs(host(table) - ref).max() <= 2.0 ** -24 + 1e-10


def rotated_bound(x, rot, interleaved, dtype):
    """Per element: 4 roundings (with the table's) of the pair's magnitudes, and the rounding to the type."""
    a = np.abs(x)
    y = np.zeros_like(a)
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    y[..., first] = y[..., second] = a[..., first] + a[..., second]
    return 4 * 2.0 ** -24 * y + DT[dtype][0] * y


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,d,rot", [(1, 1, 8, 2), (1, 32, 128, 128), (7, 5, 80, 20), (3, 2, 80, 32), (65, 3, 96, 24), (300, 4, 64, 48),
                                                (33, 2, 256, 256), (5, 1, 1024, 512), (9, 3, 64, 62)])
def test_rotation(dtype, interleaved, tokens, heads, d, rot):
    import torch
    P = lib()
    rng = np.random.default_rng(tokens * d + rot)
    table, cs = table_of(rot, 1000)
    pos = rng.integers(0, 1000, tokens)
    x, x64 = put(rng.normal(size=(tokens, heads, d)), dtype)
    r = P.Rotary(table, rot, interleaved)
    for inverse in (False, True):
        ref = O.rotate(x64, cs[pos].astype(np.float64), interleaved, inverse)
        out = torch.full_like(x, float("nan"))
        r.rotate(ints(pos), x, out, inverse, stream())
        got = host(out)
        assert (np.abs(got - ref) <= rotated_bound(x64, rot, interleaved, dtype)).all()
        assert (got[..., rot:] == x64[..., rot:]).all()
        y = x.clone()
        r.rotate(ints(pos), y, y, inverse, stream())  # in place
        assert torch.equal(y, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotation_of_strided_rows(dtype):
    """q inside a fused q, k, v row; heads ahead of tokens; one head's row for all (stride 0) as the input."""
    import torch
    P = lib()
    rng = np.random.default_rng(3)
    table, cs = table_of(64, 100)
    r, pos = P.Rotary(table, 64), rng.integers(0, 100, 17)
    wide, w64 = put(rng.normal(size=(17, 12, 64)), dtype)
    ref = O.rotate(w64, cs[pos].astype(np.float64), False)
    before = wide.clone()
    out = torch.zeros(4, 17, 64, device="cuda", dtype=wide.dtype).transpose(0, 1)
    r.rotate(ints(pos), wide[:, 2:6], out, stream=stream())
    bound = rotated_bound(w64, 64, False, dtype)
    assert (np.abs(host(out) - ref[:, 2:6]) <= bound[:, 2:6]).all()
    r.rotate(ints(pos), wide[:, 4:9], wide[:, 4:9], stream=stream())
    assert (np.abs(host(wide[:, 4:9]) - ref[:, 4:9]) <= bound[:, 4:9]).all()
    assert torch.equal(wide[:, :4], before[:, :4]) and torch.equal(wide[:, 9:], before[:, 9:])
    same = torch.empty(17, 3, 64, device="cuda", dtype=wide.dtype)
    r.rotate(ints(pos), before[:, :1].expand(17, 3, 64), same, stream=stream())
    assert (np.abs(host(same) - ref[:, :1]) <= bound[:, :1]).all()


def test_positions_outside_the_table_and_values_that_are_not_finite():
    import torch
    P = lib()
    table, _ = table_of(32, 10)
    x = torch.ones(5, 2, 64, device="cuda", dtype=torch.float16)
    x[4, 0, 0] = float("inf")
    out = torch.zeros_like(x)
    P.Rotary(table, 32).rotate(ints([-1, 9, 10, 2 ** 31 - 1, 0]), x, out, stream=stream())
    nan = torch.isnan(out)
    assert nan[0, :, :32].all() and nan[2, :, :32].all() and nan[3, :, :32].all() and not nan[1].any()
    assert not nan[:, :, 32:].any() and not nan[4, 1].any()
    assert torch.isinf(out[4, 0, 0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    """Against differences of the loss sum(w * rotate(x)) (linear in x, so a wide step is exact up to fp32) and autograd's."""
    import torch
    P = lib()
    g = torch.Generator(device="cuda").manual_seed(1)
    table, _ = table_of(24, 50)
    table = table * 1.5  # a magnitude: the gradient has it too
    r, pos = P.Rotary(table, 24, interleaved), ints(np.arange(13) * 3)
    x, w, dx = (torch.randn(13, 3, 40, device="cuda", generator=g) for _ in range(3))
    grad = torch.empty_like(x)
    r.rotate(pos, w, grad, True, stream())

    def loss(t):
        y = torch.empty_like(t)
        r.rotate(pos, t, y, False, stream())
        return (w.double() * y.double()).sum()
    slope = (loss(x + dx) - loss(x - dx)) / 2
    scale = (w.abs().double() * (x.abs() + dx.abs()).double()).sum()
    assert abs(slope - (grad.double() * dx.double()).sum()) <= 16 * 2.0 ** -24 * scale
    xs = x.double().requires_grad_()
    cs = table.double()[pos.long()][:, None]
    a, b = (xs[..., 0:24:2], xs[..., 1:24:2]) if interleaved else (xs[..., :12], xs[..., 12:24])
    u, v = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
    y = torch.cat([torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1), xs[..., 24:]], -1)
    (y * w.double()).sum().backward()
    assert (grad.double() - xs.grad).abs().max() <= 16 * 2.0 ** -24 * float(w.abs().max()) * 1.5


# ---- the cache ----------------------------------------------------------------------------------------

class Setup:
    """Sequences with `new` tokens behind `ctx` ones, on pages in random order; pages hold random bytes at first."""

    def __init__(self, dtype, kv_heads, d, page, new, ctx, seed=0, spare=2, holes=(), extra_rows=0):
        import torch
        P = lib()
        self.rng = rng = np.random.default_rng(seed)
        self.dtype, self.kvh, self.d, self.page = dtype, kv_heads, d, page
        self.new, self.len = list(new), [n + c for n, c in zip(new, ctx)]
        need = [-(-max(l, 0) // page) for l in self.len]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages)
        cols = max(max(need), 1)
        self.table = np.full((len(need), cols), -1, np.int64)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        for i, c in holes:
            self.table[i, c] = -1 if (i + c) % 2 else n_pages
        self.bytes = rng.integers(0, 256, (n_pages, P.PagedKvCache.page_bytes(kv_heads, d, page)), dtype=np.uint8)
        self.oracle = O.KvOracle(self.bytes.copy(), kv_heads, d, page)
        self.pages = torch.from_numpy(self.bytes).cuda()
        self.cache = P.PagedKvCache(code_of(dtype), kv_heads, d, page, self.pages)
        self.start = np.concatenate([[0], np.cumsum(self.new)])
        self.tokens = int(self.start[-1]) + extra_rows
        self.n_pages = n_pages

    def batch(self, positions=None, length=None, max_len=None, max_new=None):
        P = lib()
        length = self.len if length is None else length
        return P.KvBatch(ints(self.start), ints(length), ints(self.table), self.tokens, max_new or max(max(self.new), 1),
                         max_len or max(max(length), 1), None if positions is None else ints(positions))

    def places(self, i):
        return np.arange(self.len[i] - self.new[i], self.len[i])

    def slot(self, i, place):
        """(page, slot) of a place, page None for a hole or a place that is none."""
        if place < 0:
            return None, 0
        page = self.table[i, place // self.page]
        return (int(page) if 0 <= page < self.n_pages else None), place % self.page

    def fill(self, k, v):
        """The oracle's pages get rows k, v [sequence][place][head][d] (numpy, 64 bits)."""
        for i in range(len(self.new)):
            for place in range(self.len[i]):
                page, slot = self.slot(i, place)
                if page is None:
                    continue
                for h in range(self.kvh):
                    for values, x in ((0, k), (1, v)):
                        c, s, m = O.chosen(x[i][place][h][None], 32)
                        self.oracle.write(page, slot, h, values, c[0], s[0], m[0])

    def to_gpu(self):
        import torch
        self.pages.copy_(torch.from_numpy(self.oracle.p))

    def rows(self, i):
        """(keys, values) that the oracle's pages stand for: [place][head][d]; holes are NaN."""
        out = np.full((2, self.len[i], self.kvh, self.d), np.nan)
        for place in range(self.len[i]):
            page, slot = self.slot(i, place)
            if page is not None:
                for h in range(self.kvh):
                    for values in (0, 1):
                        out[values, place, h] = self.oracle.row(page, slot, h, values)
        return out


CACHES = [("bf16", 2, 128, 64, [1, 1, 1], [0, 31, 64]), ("fp16", 3, 64, 32, [5, 1, 33], [30, 0, 31]), ("fp32", 1, 128, 128, [40, 0, 3], [1, 7, 95]),
          ("bf16", 2, 256, 32, [2, 64], [31, 0]), ("fp16", 1, 256, 256, [31], [1]), ("fp32", 2, 64, 64, [96, 1], [0, 128]),
          ("bf16", 1, 64, 32, [1] * 70, list(range(70)))]


@pytest.mark.parametrize("dtype,kvh,d,page,new,ctx", CACHES)
@pytest.mark.parametrize("interleaved,rot", [(False, 0), (False, 32), (True, 64), (False, 20), (True, 6), (False, "whole"), (True, "whole")])
def test_append_writes_these_bytes_and_no_others(dtype, kvh, d, page, new, ctx, interleaved, rot):
    import torch
    P = lib()
    rot = d if rot == "whole" else rot
    s = Setup(dtype, kvh, d, page, new, ctx, seed=d + rot)
    k, k64 = put(s.rng.normal(size=(s.tokens, kvh, d)) * 3 + 1, dtype)
    v, v64 = put(s.rng.normal(size=(s.tokens, kvh, d)), dtype)
    pos = s.rng.integers(0, 500, s.tokens)
    r, keys = None, k64.astype(np.float32)
    if rot:
        table, cs = table_of(rot, 500)
        r = P.Rotary(table, rot, interleaved)
        keys = O.rotate(keys, cs[pos], interleaved)
    s.cache.append(s.batch(pos), k, v, r, stream())
    for i in range(len(new)):
        for j, place in enumerate(s.places(i)):
            page_, slot = s.slot(i, place)
            for h in range(kvh):
                for values, x in ((0, keys), (1, v64)):
                    x = x[s.start[i] + j, h][None]
                    c, sc, m = O.chosen(x, 32)
                    s.oracle.write(page_, slot, h, values, c[0], sc[0], m[0])
                    # and the values they stand for are within half a step of the 64-bit ones, up to bf16's rounding of scale and min
                    x64 = x if values else (O.rotate(k64, cs[pos].astype(np.float64), interleaved) if rot else k64)[s.start[i] + j, h][None]
                    far = np.abs(m + sc * c - x64).max()
                    assert far <= sc[0] / 2 * (1 + 1e-5) + 2.0 ** -8 * np.abs(x64).max() * 2
    assert torch.equal(s.pages.cpu(), torch.from_numpy(s.oracle.p))
    # read gives these values back
    kb, vb = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    s.cache.read(s.batch(), kb, vb, stream())
    for i in range(len(new)):
        rows = s.rows(i)[:, s.len[i] - new[i]:]
        for got, ref in ((kb, rows[0]), (vb, rows[1])):
            assert torch.equal(got[s.start[i]:s.start[i + 1]].cpu(), torch.from_numpy(ref.astype(np.float32)).to(k.dtype))  # exact in 32 bits, then one rounding


def test_rows_that_hold_no_numbers():
    """Not finite, constant, zero, tiny and huge rows."""
    import torch
    inf, nan, big = np.inf, np.nan, 3e38
    x = np.zeros((11, 1, 64))
    x[0, 0, 5] = nan
    x[1, 0, 63] = inf
    x[2, 0, 0] = -inf
    x[3] = 2.5
    x[5, 0, :2] = -big, big     # a spread that is not finite in 32 bits
    x[6, 0, :2] = 1e-38, 2e-38  # below the smallest scale
    x[7, 0, :2] = -big, -big / 2
    x[8] = np.linspace(-1e-20, 1e-20, 64)
    x[9] = -3.39e38             # its bf16 is the largest finite one
    x[10] = -3.4e38             # its bf16 is not finite
    s = Setup("fp32", 1, 64, 32, [11], [3])
    t, x64 = put(x, "fp32")
    s.cache.append(s.batch(), t, t.clone(), None, stream())
    kb, vb = torch.zeros_like(t), torch.zeros_like(t)
    s.cache.read(s.batch(), kb, vb, stream())
    for values in (0, 1):
        for j, place in enumerate(s.places(0)):
            c, sc, m = O.chosen(x64[j].astype(np.float32), 32)
            s.oracle.write(*s.slot(0, place), 0, values, c[0], sc[0], m[0])
    assert torch.equal(s.pages.cpu(), torch.from_numpy(s.oracle.p))
    for got in (host(kb), host(vb)):
        assert np.isnan(got[[0, 1, 2, 5, 10]]).all() and not np.isnan(got[[3, 4, 6, 7, 8, 9]]).any()
        assert (got[9] == -(2 - 2.0 ** -7) * 2.0 ** 127).all()
        assert (got[3] == 2.5).all() and (got[4] == 0).all() and np.abs(got[6]).max() <= 2e-38
        assert np.abs(got[8] - x64[8]).max() <= 2e-20 / 15 / 2 * 1.02


def test_holes_negative_places_and_rows_of_no_sequence():
    import torch
    s = Setup("bf16", 2, 64, 32, [40, 6, 2, 3], [30, 0, 0, 0], holes=[(0, 1)], extra_rows=4)
    s.len[1], s.len[2] = 4, 0  # two tokens of sequence 1 and both of sequence 2 have no place
    k, k64 = put(s.rng.normal(size=(s.tokens, 2, 64)), "bf16")
    v, v64 = put(s.rng.normal(size=(s.tokens, 2, 64)), "bf16")
    s.cache.append(s.batch(max_len=70), k, v, None, stream())
    kb, vb = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    s.cache.read(s.batch(max_len=70), kb, vb, stream())
    for i in range(4):
        for j, place in enumerate(s.places(i)):
            page, slot = s.slot(i, place)
            got = host(kb)[s.start[i] + j], host(vb)[s.start[i] + j]
            if page is None:
                assert np.isnan(got[0]).all() and np.isnan(got[1]).all()
                continue
            for h in range(2):
                for values, x in ((0, k64), (1, v64)):
                    c, sc, m = O.chosen(x[s.start[i] + j, h][None], 32)
                    s.oracle.write(page, slot, h, values, c[0], sc[0], m[0])
                    assert np.abs(got[values][h] - (m + sc * c)).max() <= 2.0 ** -8 * np.abs(x).max()
    assert torch.equal(s.pages.cpu(), torch.from_numpy(s.oracle.p))
    assert (kb[s.start[-1]:] == 7).all() and (vb[s.start[-1]:] == 7).all()


def test_arrays_out_of_range_touch_nothing_else():
    """Lengths past the table, first rows past the rows, descending first rows: held to what there is."""
    import torch
    P = lib()
    s = Setup("bf16", 1, 64, 32, [3, 2], [60, 5])
    k, _ = put(s.rng.normal(size=(5, 1, 64)), "bf16")
    guard = torch.full((5 + 64, 4, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    out = guard[32:37]
    ws = torch.empty(1 << 16, device="cuda", dtype=torch.uint8)
    for start, length in (([0, 3, 1000], [10 ** 9, 7]), ([0, 4, 2], [63, 2 ** 31 - 1]), ([-5, 3, 5], [-4, 7]), ([2 ** 31 - 1, -1, 5], [63, 7])):
        b = P.KvBatch(ints(start), ints(length), ints(s.table), 5, 3, 64)
        s.cache.append(b, k, k, None, stream())
        s.cache.read(b, k.clone(), k.clone(), stream())
        q, _ = put(s.rng.normal(size=(5, 4, 64)), "bf16")
        s.cache.attend(b, q, out, 0.1, ws, stream=stream())
    torch.cuda.synchronize()
    assert (guard[:32] == 3).all() and (guard[37:] == 3).all()
    assert torch.equal(s.pages[[p for p in range(s.n_pages) if p not in s.table]].cpu(),
                       torch.from_numpy(s.bytes[[p for p in range(s.n_pages) if p not in s.table]]))


# ---- attention ----------------------------------------------------------------------------------------

def check_attention(s, heads, causal=True, window=0, rot=0, interleaved=False, k_std=1.0, v_std=1.0, q_std=1.0, workspace=1 << 22, keys=None, vals=None,
                    q_in=None, scale=None, out_layout="thd", some=None):
    import torch
    P = lib()
    rng, d, dtype = s.rng, s.d, s.dtype
    scale = scale or d ** -0.5
    k = keys or [rng.normal(size=(max(l, 0), s.kvh, d)) * k_std for l in s.len]
    v = vals or [rng.normal(size=(max(l, 0), s.kvh, d)) * v_std for l in s.len]
    s.fill(k, v)
    s.to_gpu()
    q, q64 = put(rng.normal(size=(s.tokens, heads, d)) * q_std if q_in is None else q_in, dtype)
    r, pos = None, rng.integers(0, 300, s.tokens)
    if rot:
        table, cs = table_of(rot, 300)
        r = P.Rotary(table, rot, interleaved)
        q64 = O.rotate(q64, cs[pos].astype(np.float64), interleaved)
    out = torch.full((s.tokens, heads, d) if out_layout == "thd" else (heads, s.tokens, d), 9.0, device="cuda", dtype=q.dtype)
    view = out if out_layout == "thd" else out.transpose(0, 1)
    ws = torch.empty(workspace, device="cuda", dtype=torch.uint8) if workspace else None
    s.cache.attend(s.batch(pos), q, view, scale, ws, causal, window, r, stream())
    got = host(view)
    rounding = DT[dtype][0]
    weight = 2.0 ** -22 if dtype == "fp32" else 2.0 ** -11
    logit = 2.0 ** -18 if dtype == "fp32" else 2.0 ** -11 if dtype == "bf16" and rot else 2.0 ** -16
    for i in range(len(s.new)) if some is None else some:
        rows = slice(s.start[i], s.start[i + 1])
        if not s.new[i]:
            continue
        kk, vv = s.rows(i) if s.len[i] > 0 else np.zeros((2, 1, s.kvh, d))
        holes = [p for p in range(s.len[i]) if s.slot(i, p)[0] is None]
        kk, vv = np.where(np.isfinite(kk), kk, 0), np.where(np.isfinite(vv), vv, 0)
        places = s.places(i) if s.len[i] > 0 else np.full(s.new[i], -1)
        ref, amp, size = O.attend(q64[rows], kk, vv, scale, places, causal, window, holes)
        bound = rounding * np.abs(ref) + (amp * (2 * weight + 2 * logit * size))[..., None] + 1e-30
        s.exact = ref  # of the last sequence
        far = np.abs(got[rows] - ref)
        assert (far <= bound).all(), "sequence %d: %.3g times its bound" % (i, (far / bound).max())
        if s.len[i] <= 0:
            assert (got[rows] == 0).all()
    assert (got[s.start[-1]:] == 9).all()
    return out


ATTEND = [  # kv heads, heads, d, page, new, ctx
    (2, 8, 128, 64, [1, 1, 1, 1, 1], [0, 30, 31, 32, 300]),
    (1, 1, 64, 32, [1, 1], [64, 999]),
    (3, 15, 64, 32, [1, 3, 2, 0, 1], [0, 70, 1, 5, 129]),         # 5 heads a kv head; 3 tokens fill a tile
    (1, 16, 128, 128, [1, 2, 7], [200, 100, 0]),                  # 16 rows and more
    (2, 2, 256, 64, [1, 17, 40], [300, 65, 0]),
    (1, 3, 128, 64, [130, 1, 5], [0, 100, 127]),
    (2, 6, 64, 256, [65, 33], [0, 500]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kvh,heads,d,page,new,ctx", ATTEND)
@pytest.mark.parametrize("causal,window,rot", [(True, 0, 0), (True, 37, 32), (False, 0, 64)])
def test_attention(dtype, kvh, heads, d, page, new, ctx, causal, window, rot):
    check_attention(Setup(dtype, kvh, d, page, new, ctx, seed=heads + d), heads, causal, window, rot, interleaved=rot == 32)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kvh,heads,d,page,new,ctx", ATTEND[:2] + ATTEND[4:6])
@pytest.mark.parametrize("interleaved", [False, True])
def test_attention_with_whole_heads_rotated(dtype, kvh, heads, d, page, new, ctx, interleaved):
    check_attention(Setup(dtype, kvh, d, page, new, ctx, seed=heads + d), heads, rot=d, interleaved=interleaved)


@pytest.mark.parametrize("dtype,most", [("bf16", 2.5e-3), ("fp16", 4e-4), ("fp32", 2e-6)])
@pytest.mark.parametrize("new,rot", [(1, 0), (1, 128), (3, 128), (40, 128)])
def test_error_of_long_rows_as_a_norm(dtype, most, new, rot):
    """2000 keys, some channels of which are loud: the error's 2-norm against the result's.  A result's own rounding is 0.43 units
    in the last place's half (bf16 1.7e-3, fp16 2.1e-4), weights of 11 bits add 2.1e-4 of it, a rotated bf16 row of 11 bits
    2.1e-4 times a logit's size of up to 5; fp32: sums of 128 and 2000 terms, and the exponent of a logit of 10, 2^-24 each."""
    s = Setup(dtype, 1, 128, 64, [new], [2000], seed=5)
    rng = s.rng
    loud = np.where(rng.random(128) < 0.06, 4.0, 1.0)
    keys = [rng.normal(size=(s.len[0], 1, 128)) * loud + 0.5 * rng.normal(size=128)]
    vals = [rng.normal(size=(s.len[0], 1, 128))]
    q_in = 1.5 * rng.normal(size=(new, 4, 128))
    out = host(check_attention(s, 4, rot=rot, keys=keys, vals=vals, q_in=q_in))
    assert np.linalg.norm(out - s.exact) <= most * np.linalg.norm(s.exact)


@pytest.mark.parametrize("workspace", [0, 1000, 40000, 1 << 24])
@pytest.mark.parametrize("heads,new,ctx", [(4, [1, 1], [4000, 100]), (4, [40, 1], [3000, 2500]), (1, [1], [5000])])
def test_parts_of_long_sequences(workspace, heads, new, ctx):
    check_attention(Setup("fp16", 1, 64, 256, new, ctx), heads, workspace=workspace)
    check_attention(Setup("fp16", 1, 64, 32, new, ctx, seed=1), heads, workspace=workspace, window=700, rot=64)


def test_sequences_without_keys_holes_and_rows_of_no_sequence():
    s = Setup("bf16", 2, 64, 32, [2, 3, 40, 5, 1], [0, 0, 60, 0, 40], holes=[(2, 0), (2, 2), (4, 1)], extra_rows=3)
    s.len[0], s.len[3] = 0, 2  # no key at all; three tokens ahead of the first place
    check_attention(s, 4)
    s = Setup("bf16", 2, 64, 32, [1, 1], [63, 31], holes=[(0, 0), (0, 1), (1, 0)])  # nothing but holes
    out = check_attention(s, 4)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_what_is_not_seen_does_not_matter(dtype):
    """Rows behind a token's own place that are not finite or huge, and memory that no row was written to."""
    s = Setup(dtype, 1, 64, 64, [20, 1, 1], [50, 10, 40])
    s.bytes[:] = 255  # every scale and min NaN where no row is
    s.oracle.p[:] = 255
    rng = np.random.default_rng(5)
    k, v = ([rng.normal(size=(l, 1, 64)) for l in s.len] for _ in range(2))
    k[0][60:], v[0][60:] = np.inf, np.nan
    v[0][59] = 1e30
    k[2][:5], v[2][:5] = np.nan, np.inf
    # tokens that see none of these
    import torch
    s.fill(k, v)
    s.to_gpu()
    q, q64 = put(rng.normal(size=(s.tokens, 2, 64)), dtype)
    out = torch.empty_like(q)
    s.cache.attend(s.batch(), q, out, 0.125, None, True, 30, None, stream())
    got = host(out)
    for i, rows in ((0, range(9)), (1, range(1)), (2, range(1))):
        kk, vv = s.rows(i)
        for j in rows:
            see = np.arange(s.len[i])[max(0, s.places(i)[j] - 29):s.places(i)[j] + 1]
            ref, amp, size = O.attend(q64[s.start[i] + j][None], kk[see], vv[see], 0.125, [10 ** 6])
            bound = DT[dtype][0] * np.abs(ref) + (amp * (2.0 ** -10 + 2.0 ** -14 * size))[..., None]
            assert (np.abs(got[s.start[i] + j] - ref) <= bound).all()
    assert np.isnan(got[s.start[0] + 10]).all()  # and those that see them show it


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("q_std,k_std,v_std", [(1e-18, 1e-12, 1.0), (1e15, 1e-14, 1.0), (1.0, 1.0, 1e25), (1.0, 1.0, 1e-25), (60.0, 1.0, 1.0)])
def test_magnitudes(dtype, q_std, k_std, v_std):
    """fp16's range is not a limit of bf16's and fp32's inputs; very sharp softmax."""
    s = Setup(dtype, 1, 128, 64, [1, 20], [200, 90])
    check_attention(s, 2, q_std=q_std, k_std=k_std, v_std=v_std)


def test_values_of_very_different_size_in_one_row():
    """A heavy key with hardly any weight next to light ones, in both orders, and rows of constants (scale 0)."""
    s = Setup("fp32", 1, 64, 64, [1, 1, 1], [99, 99, 99])
    rng = s.rng
    k = [rng.normal(size=(100, 1, 64)) for _ in range(3)]
    v = [rng.normal(size=(100, 1, 64)) for _ in range(3)]
    v[0][10] *= 1e12
    v[1][90] *= 1e12
    v[1][40:60] = 3.0
    v[2][:] = rng.normal(size=(100, 1, 1)) * 1e5
    check_attention(s, 1, keys=k, vals=v, q_std=6.0)


def test_same_bits_wherever_the_pages_lie_and_on_another_stream():
    import torch
    outs = []
    for seed in (0, 1):
        s = Setup("bf16", 2, 128, 32, [1, 30], [700, 50], spare=9 * seed)
        rng = np.random.default_rng(7)
        k, v = ([rng.normal(size=(l, 2, 128)) for l in s.len] for _ in range(2))
        q = rng.normal(size=(s.tokens, 8, 128))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        if seed:
            with torch.cuda.stream(side):
                outs.append(check_attention(s, 8, keys=k, vals=v, q_in=q, out_layout="htd").transpose(0, 1).contiguous())
            torch.cuda.current_stream().wait_stream(side)
        else:
            outs.append(check_attention(s, 8, keys=k, vals=v, q_in=q))
    assert torch.equal(outs[0], outs[1])


def test_places_past_four_gigabytes():
    import torch
    P = lib()
    page = P.PagedKvCache.page_bytes(8, 128, 64)
    n = (5 << 30) // page
    pages = torch.zeros(n, page, device="cuda", dtype=torch.uint8)
    s = Setup("bf16", 8, 128, 64, [70], [3])
    k, k64 = put(s.rng.normal(size=(70, 8, 128)), "bf16")
    far, near = P.PagedKvCache(P.PLORA_BF16, 8, 128, 64, pages), s.cache
    b = s.batch()
    b_far = P.KvBatch(ints(s.start), ints(s.len), ints([[n - 1, n - 2]]), 70, 70, s.len[0])
    s.pages.zero_()
    res = []
    for cache, bb in ((near, b), (far, b_far)):
        cache.append(bb, k, k, None, stream())
        kb, vb, out = (torch.zeros_like(k) for _ in range(3))
        cache.read(bb, kb, vb, stream())
        cache.attend(bb, k, out, 0.1, None, stream=stream())
        res.append((kb, vb, out))
    assert all(torch.equal(x, y) for x, y in zip(*res))
    assert int(pages[:n - 2].max()) == 0


def test_a_captured_step_replayed():
    """append and attend of a decode step as a graph, replayed over lengths that grow, between eager work."""
    import torch
    P = lib()
    s = Setup("bf16", 2, 128, 64, [1, 1, 1], [10, 62, 500], spare=6)
    s.table = np.concatenate([s.table, np.full((3, 1), -1)], 1)
    free = [p for p in range(s.n_pages) if p not in s.table]
    for i, l in enumerate(s.len):
        s.table[i, -(-l // 64)] = free[i]
    rng = np.random.default_rng(2)
    s.fill(*[[rng.normal(size=(l, 2, 128)) for l in s.len] for _ in range(2)])
    s.to_gpu()
    table, _ = table_of(128, 600)
    r = P.Rotary(table, 128)
    length = ints(s.len)
    b = P.KvBatch(ints(s.start), length, ints(s.table), 3, 1, 600)
    q, k, v = (torch.zeros(3, h, 128, device="cuda", dtype=torch.bfloat16) for h in (8, 2, 2))
    out, ws = torch.zeros_like(q), torch.empty(1 << 22, device="cuda", dtype=torch.uint8)

    def step():
        s.cache.append(b, k, v, r, stream())
        s.cache.attend(b, q, out, 0.09, ws, rotary=r, stream=stream())
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for it in range(5):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda"))
        before = s.pages.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, pages = out.clone(), s.pages.clone()
        s.pages.copy_(before)
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(s.pages, pages)
        length += 1


def test_random_shapes():
    rng = np.random.default_rng(11)
    for n in range(30):
        kvh, rep = int(rng.integers(1, 4)), int(rng.integers(1, 9))
        d = int(rng.choice([64, 128, 256]))
        seqs = int(rng.integers(1, 6))
        new = [int(x) for x in rng.integers(0, rng.choice([2, 8, 50]), seqs)]
        ctx = [int(x) for x in rng.integers(0, rng.choice([3, 100, 400]), seqs)]
        if not sum(new):
            new[0] = 1
        s = Setup(str(rng.choice(["bf16", "fp16", "fp32"])), kvh, d, int(rng.choice([32, 64, 128, 256])), new, ctx, seed=n)
        causal = bool(rng.random() < 0.7)
        print("case", n, s.dtype, kvh, rep, d, s.page, new, ctx, causal, flush=True)
        check_attention(s, kvh * rep, causal, int(rng.integers(1, 200)) if causal and rng.random() < 0.4 else 0, int(rng.choice([0, 32, 64])),
                        workspace=int(rng.choice([0, 1 << 22])))
