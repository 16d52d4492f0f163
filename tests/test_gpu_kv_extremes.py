"""Attention over the KV cache where sizes, lengths and settings are far apart or at their limits, against the oracle's 64 bits.  The bounds
are those of test_gpu_kv.py, from the arithmetic, where an input gives no other reason."""
import numpy as np
import pytest

from test_gpu_kv import DT, Setup, check_attention, host, ints, put, stream

pytestmark = pytest.mark.gpu

# One sequence in every kernel and form of it: tokens, tokens ahead of them, query heads, workspace.
FORMS = {"few, 4 rows, 16 wavefronts": (1, 1100, 2, 0), "few, 4 rows, 4 wavefronts": (1, 2300, 2, 0), "few, 8 rows": (2, 700, 4, 0),
         "few, 16 rows": (4, 700, 4, 0), "few, parts": (1, 4500, 2, 1 << 22), "many": (40, 500, 2, 0), "many, parts": (40, 3000, 2, 1 << 24)}


def one(form, dtype, d=64, seed=0):
    """(Setup of one sequence, query heads, workspace, places)"""
    new, ctx, heads, workspace = FORMS[form]
    return Setup(dtype, 1, d, 64, [new], [ctx], seed=seed), heads, workspace, new + ctx


# ---- values of very different size ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("signs", ["one", "both"])
def test_constant_rows_behind_rows_of_zeros(form, dtype, signs):
    """Values of scale 0: their weights meet their min only.  All logits are about the same."""
    s, heads, workspace, n = one(form, dtype)
    c = 1e9 * np.where((np.arange(n) % 2 == 0) | (signs == "one"), 1.0, -0.75)
    c[:n // 2] = 0
    check_attention(s, heads, vals=[np.broadcast_to(c[:, None, None], (n, 1, 64))], q_std=0.1, workspace=workspace)


# ---- settings at their limits -------------------------------------------------------------------------

@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4, 2 ** 30, 50])
@pytest.mark.parametrize("new,length,heads", [([9, 1], [4, 60], 1), ([40, 3], [31, 70], 2), ([200, 1], [150, 1], 1)])
def test_wide_windows_and_negative_places(window, new, length, heads):
    """The window's first place lies before 0, by up to 2^31 and a few."""
    check_attention(Setup("bf16", 1, 64, 32, new, [l - n for l, n in zip(length, new)]), heads, window=window)


@pytest.mark.parametrize("new,ctx", [([1, 1], [4000, 9]), ([40, 1], [300, 77])])
def test_a_max_len_far_above_the_table(new, ctx):
    """max_len is a bound: the table holds 64 or 5 pages."""
    s = Setup("bf16", 1, 64, 64, new, ctx)
    plain = s.batch
    s.batch = lambda positions=None: plain(positions, max_len=2 ** 31 - 1)
    check_attention(s, 2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("light", [0.0, 1e-25])
@pytest.mark.parametrize("stripe", [16, 32, 64, "light first", "heavy first"])
def test_light_and_heavy_values_of_the_same_weight(form, dtype, light, stripe):
    """Values of 1e25 and next to nothing, in steps, columns, wavefronts and parts of their own: what the sums are held against differs by
    up to 2^180, the weights do not."""
    s, heads, workspace, n = one(form, dtype)
    at = np.arange(n)
    heavy = at >= n // 2 if stripe == "light first" else at < n // 2 if stripe == "heavy first" else at // stripe % 2 == 1
    v = (2 + 0.3 * s.rng.normal(size=(n, 1, 64))) * np.where(heavy, 1e25, light)[:, None, None]
    check_attention(s, heads, vals=[v], q_std=0.1, workspace=workspace)


def test_weights_of_millions_of_keys_without_values():
    """Keys whose values are 0 leave the reference far below, so their weights are large numbers: 2^23 of them, then 256 values of 1.  The pages
    in between are the same one.  Bound: a lane's sum has 2^15 additions, each rounded by 2^-24 of it at most."""
    import torch
    import paper_2512_20210_amd as P
    from oracle import kv as O
    columns = (1 << 15) + 2
    pages = np.zeros((3, P.PagedKvCache.page_bytes(1, 64, 256)), np.uint8)
    o = O.KvOracle(pages, 1, 64, 256)
    key = 7.5 * np.log(2) / (64 * 0.125)  # logit of 7.5 to base 2 with a q of ones
    for page, (k, v) in enumerate(((0, 0), (key, 0), (key, 1))):
        for values, x in ((0, k), (1, v)):
            c, sc, m = O.chosen(np.full((1, 64), x), 32)
            for slot in range(256):
                o.write(page, slot, 0, values, c[0], sc[0], m[0])
            if page == 1 and not values:
                held = float(m[0])
    table = torch.ones(1, columns, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -1] = 0, 2
    cache = P.PagedKvCache(P.PLORA_F32, 1, 64, 256, torch.from_numpy(pages).cuda())
    length = columns * 256
    batch = P.KvBatch(ints([0, 1]), ints([length]), table, 1, 1, length)
    q, out = torch.ones(1, 1, 64, device="cuda"), torch.zeros(1, 1, 64, device="cuda")
    cache.attend(batch, q, out, 0.125, None, stream=stream())
    ref = 256 / (256 * np.exp(-8 * held) + 256 * (columns - 1))
    assert np.abs(host(out) / ref - 1).max() <= 2.0 ** -9 + 2.0 ** -18


# ---- more rows than the call says --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_new,new,ctx,heads,kvh", [(1, [2, 1, 5, 1], [4000, 300, 3000, 0], 4, 1), (1, [3, 1], [30, 100], 8, 8), (2, [2, 7, 1], [2000, 900, 90], 8, 2),
                                                       (3, [1, 3, 4, 90], [900, 5000, 40, 4000], 8, 1), (30, [31, 1, 500], [3000, 7, 20], 2, 1)])
@pytest.mark.parametrize("workspace", [0, 1 << 24])
def test_more_tokens_than_max_new(dtype, max_new, new, ctx, heads, kvh, workspace):
    """The first max_new tokens of a sequence have their results, the others may be left out; nothing of the workspace's contents shows."""
    import torch
    from oracle import kv as O
    s = Setup(dtype, kvh, 64, 64, new, ctx, seed=max_new)
    s.fill(*([s.rng.normal(size=(l, kvh, 64)) for l in s.len] for _ in range(2)))
    s.to_gpu()
    q, q64 = put(s.rng.normal(size=(s.tokens, heads, 64)), dtype)
    out = torch.full_like(q, 9.0)
    ws = torch.full((workspace // 4,), float("nan"), device="cuda") if workspace else None
    s.cache.attend(s.batch(max_new=max_new), q, out, 0.125, ws, stream=stream())
    got = host(out)
    for i in range(len(new)):
        rows = slice(s.start[i], s.start[i + 1])
        ref, amp, size = O.attend(q64[rows], *s.rows(i), 0.125, s.places(i))
        bound = DT[dtype][0] * np.abs(ref) + (amp * (2.0 ** -10 + 2.0 ** -15 * size))[..., None]
        right, alone = np.abs(got[rows] - ref) <= bound, got[rows] == 9
        assert right[:max_new].all()
        assert (right[max_new:].all(-1) | alone[max_new:].all(-1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("q_std,k_std", [(1e-34, 1e34), (1e-34, 1e36), (3e-35, 3e36), (1e-30, 1e30), (1e28, 1e-28)])
def test_large_keys_and_small_queries(form, dtype, q_std, k_std):
    """Logits of the order of 1 to 100: sizes of one side that fp32's sums of codes could not take meet the other side first."""
    s, heads, workspace, n = one(form, dtype, d=128)
    check_attention(s, heads, q_std=q_std, k_std=k_std, workspace=workspace)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
def test_large_keys_among_ordinary_ones(form, dtype):
    s, heads, workspace, n = one(form, dtype, d=128)
    keys = s.rng.normal(size=(n, 1, 128)) * np.where(s.rng.random((n, 1, 1)) < 0.1, 1e36, 1e3)
    check_attention(s, heads, q_std=1e-34, keys=[keys], workspace=workspace)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("scale,q_std", [(1e-40, 1e-3), (1e-12, 1e-36), (1e-38, 60.0)])
def test_scales_that_leave_equal_weights(form, dtype, scale, q_std):
    """Keys that are not seen stay out of a mean over the others."""
    s, heads, workspace, n = one(form, dtype)
    check_attention(s, heads, q_std=q_std if dtype != "fp16" else max(q_std, 1e-3), scale=scale, workspace=workspace, window=n - 7)


# ---- rows of the cache at the limit of fp32 -----------------------------------------------------------

def test_rows_whose_spread_just_fits():
    """hi - lo is finite, hi less the rounded lo is not."""
    import torch
    from oracle import kv as O
    x = np.random.default_rng(1).uniform(-1.69e38, 1.69e38, size=(40, 1, 64)).astype(np.float32)
    top, lo = np.float32(3.4028235e38), np.float32(-1.6955e38)
    x[:, 0, 3] = lo * np.linspace(1, 1.003, 40, dtype=np.float32)
    x[:, 0, 60] = top * np.float32(1 - 2.0 ** -13) + x[:, 0, 3]
    x[1::2, 0, 60] *= np.float32(0.99)
    with np.errstate(all="ignore"):
        lo16 = O.to_bf16(x.min(-1))
        assert np.isfinite(x.max(-1) - x.min(-1)).all() and (~np.isfinite(x.max(-1) - lo16)).sum() >= 5
    s = Setup("fp32", 1, 64, 32, [40], [3])
    t, x64 = put(x, "fp32")
    s.cache.append(s.batch(), t, t.clone(), None, stream())
    for j, place in enumerate(s.places(0)):
        with np.errstate(all="ignore"):
            c, sc, mn = O.chosen(x64[j].astype(np.float32), 32)
        for values in (0, 1):
            s.oracle.write(*s.slot(0, place), 0, values, c[0], sc[0], mn[0])
    assert torch.equal(s.pages.cpu(), torch.from_numpy(s.oracle.p))
    kb, vb = torch.zeros_like(t), torch.zeros_like(t)
    s.cache.read(s.batch(), kb, vb, stream())
    for got, ref in zip((kb, vb), s.rows(0)[:, 3:]):
        assert torch.equal(got.cpu(), torch.from_numpy(ref.astype(np.float32)))


# ---- rows beside rows that are NaN --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_growing_weights_beside_a_row_that_is_nan(dtype):
    """Tokens 0 to 15 see a key that is NaN, the others do not, and share their lanes: the others' weights grow by 2^28 while the values are 0,
    then the values are 1."""
    import torch
    from oracle import kv as O
    new, ctx, window = 64, 200, 150
    s = Setup(dtype, 1, 64, 64, [new], [ctx])
    n = new + ctx
    first = ctx + 15 - window + 1  # the last token's of the first 16 first key
    k, v = np.zeros((n, 1, 64)), np.zeros((n, 1, 64))
    k[first] = np.nan
    grown = (np.arange(n) >= first + 65) & (np.arange(n) % 16 < 4)  # keys of the lanes that have the one that is NaN
    k[grown] = 28 * np.log(2) / (64 * 0.125)  # a logit of 28 to base 2 with a q of ones
    v[ctx - 10:] = 1
    s.fill([k], [v])
    s.to_gpu()
    q, q64 = put(np.ones((new, 1, 64)), dtype)
    out = torch.zeros_like(q)
    s.cache.attend(s.batch(), q, out, 0.125, None, True, window, stream=stream())
    got = host(out)
    kk, vv = s.rows(0)
    ref, amp, size = O.attend(q64, np.nan_to_num(kk), vv, 0.125, s.places(0), window=window)
    assert np.isnan(got[:16]).all()
    bound = DT[dtype][0] * np.abs(ref) + (amp * (2.0 ** -10 + 2.0 ** -15 * size))[..., None]
    assert (np.abs(got - ref) <= bound)[16:].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("q_std,v_std", [(3e2, 1.0), (1e5, 1e9), (1e6, 1e-9), (1e6, 1.0)])
def test_large_logits(form, dtype, q_std, v_std):
    """Logits up to 1e7 leave one key's values, or a few, which are a mean of values all the same: no further out than the outermost one."""
    s, heads, workspace, n = one(form, dtype)
    out = host(check_attention(s, heads, q_std=q_std, v_std=v_std, workspace=workspace))
    low, high = s.rows(0)[1].min((0, 1)), s.rows(0)[1].max((0, 1))
    slack = (DT[dtype][0] + 2 * 2.0 ** (-22 if dtype == "fp32" else -11)) * np.maximum(np.abs(low), np.abs(high))  # the result's rounding, the weights' bits
    assert (out >= low - slack).all() and (out <= high + slack).all()
