"""What the calls on heads, rotary positions and the KV cache refuse.  Every check is ahead of the first launch, so these run
without a GPU; the pointers are never followed."""
import ctypes as C

import pytest
import torch  # noqa: F401  (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P

AT = 0x10000


def rows(data=AT, t=1024, h=128):
    return P.RowsStruct(data, t, h)


def rotary(table=AT, max_pos=16, rot=64, interleaved=0):
    return P.RotaryStruct(table, max_pos, rot, interleaved)


def cache(dtype=P.PLORA_BF16, heads=8, d=128, page=64, n=4, pages=AT):
    return P.KvCacheStruct(dtype, heads, d, page, n, pages)


def batch(n_seqs=2, n_tokens=3, max_new=2, max_len=100, stride=2, start=AT, length=AT, table=AT, positions=None):
    return P.KvBatchStruct(n_seqs, n_tokens, max_new, max_len, stride, start, length, table, positions)


def test_page_bytes():
    assert P.plora_kv_page_bytes(cache()) == 8 * 64 * 136
    for bad in (cache(d=80), cache(page=48), cache(page=512), cache(heads=0), cache(heads=1025), cache(dtype=3)):
        assert P.plora_kv_page_bytes(bad) == 0
    assert P.PagedKvCache.page_bytes(2, 64, 32) == 2 * 32 * 72


def test_nothing_to_do_is_fine():
    for b in (batch(n_tokens=0, start=None, length=None, table=None), batch(n_seqs=0, start=None, length=None, table=None)):
        assert P.plora_kv_append(cache(), b, rows(), rows()) == 0
        assert P.plora_kv_read(cache(), b, rows(), rows()) == 0
        assert P.plora_kv_attend(cache(), b, 8, rows(), rows(), 0.1) == 0
    assert P.plora_rotate(rotary(), P.PLORA_F16, 0, 8, 128, None, None, None) == 0


BAD_CACHE = [cache(d=96), cache(page=16), cache(heads=0), cache(dtype=7), cache(n=0), cache(pages=None), cache(pages=AT + 8)]
BAD_BATCH = [batch(n_seqs=-1), batch(n_tokens=-1), batch(max_new=0), batch(max_len=0), batch(stride=0), batch(start=None),
             batch(length=None), batch(table=None)]
BAD_ROWS = [None, rows(data=None), rows(data=AT + 2), rows(t=1028), rows(h=4), rows(t=-1024), rows(h=-128), rows(t=1 << 41)]
BAD_OUT = BAD_ROWS + [rows(t=0), rows(h=0), rows(t=1016), rows(h=120), rows(t=128, h=128)]
BAD_ROTARY = [rotary(table=None), rotary(table=AT + 4), rotary(max_pos=0), rotary(rot=0), rotary(rot=63), rotary(rot=130), rotary(interleaved=2)]


@pytest.mark.parametrize("c,b", [(c, batch()) for c in BAD_CACHE] + [(cache(), b) for b in BAD_BATCH] + [(None, batch()), (cache(), None)])
def test_bad_caches_and_batches(c, b):
    assert P.plora_kv_append(c, b, rows(), rows()) == P.PLORA_ERR_INVAL
    assert P.plora_kv_read(c, b, rows(), rows()) == P.PLORA_ERR_INVAL
    assert P.plora_kv_attend(c, b, 8, rows(), rows(), 0.1) == P.PLORA_ERR_INVAL


def test_bad_rows():
    for r in BAD_ROWS:
        assert P.plora_kv_append(cache(), batch(), r, rows()) == P.PLORA_ERR_INVAL
        assert P.plora_kv_append(cache(), batch(), rows(), r) == P.PLORA_ERR_INVAL
        assert P.plora_kv_attend(cache(), batch(), 8, r, rows(), 0.1) == P.PLORA_ERR_INVAL
        assert P.plora_rotate(rotary(), P.PLORA_BF16, 3, 8, 128, AT, r, rows(data=AT << 4)) == P.PLORA_ERR_INVAL
    for r in BAD_OUT:
        assert P.plora_kv_read(cache(), batch(), r, rows()) == P.PLORA_ERR_INVAL
        assert P.plora_kv_read(cache(), batch(), rows(), r) == P.PLORA_ERR_INVAL
        assert P.plora_kv_attend(cache(), batch(), 8, rows(), r, 0.1) == P.PLORA_ERR_INVAL
        assert P.plora_rotate(rotary(), P.PLORA_BF16, 3, 8, 128, AT, rows(data=AT << 4), r) == P.PLORA_ERR_INVAL


def test_bad_rotations():
    for r in BAD_ROTARY:
        assert P.plora_kv_append(cache(), batch(), rows(), rows(), r) == P.PLORA_ERR_INVAL
        assert P.plora_kv_attend(cache(), batch(), 8, rows(), rows(), 0.1, rotary=r) == P.PLORA_ERR_INVAL
        assert P.plora_rotate(r, P.PLORA_BF16, 3, 8, 128, AT, rows(), rows()) == P.PLORA_ERR_INVAL
    good = dict(rotary=rotary(), dtype=P.PLORA_BF16, n_tokens=3, n_heads=8, head_dim=128, positions_ptr=AT, x=rows(), y=rows())
    for bad in (dict(rotary=None), dict(dtype=4), dict(n_tokens=-1), dict(n_heads=0), dict(head_dim=132), dict(head_dim=1032), dict(head_dim=0),
                dict(positions_ptr=None), dict(x=rows(t=2048))):  # in place with other strides
        assert P.plora_rotate(**{**good, **bad}) == P.PLORA_ERR_INVAL


def test_bad_attention():
    for heads, scale, causal, window, ws, size in ((9, .1, 1, 0, None, 0), (0, .1, 1, 0, None, 0), (8, 0., 1, 0, None, 0), (8, -1., 1, 0, None, 0),
                                                   (8, float("nan"), 1, 0, None, 0), (8, float("inf"), 1, 0, None, 0), (8, .1, 1, -1, None, 0),
                                                   (8, .1, 0, 5, None, 0), (8, .1, 1, 0, AT + 8, 64), (8, .1, 1, 0, None, 64)):
        assert P.plora_kv_attend(cache(), batch(), heads, rows(), rows(), scale, causal, window, None, ws, size) == P.PLORA_ERR_INVAL


def test_bad_tables():
    ok = P.RotaryConfig()
    for cfg, rot, n, at in ((None, 8, 4, AT), (ok, 7, 4, AT), (ok, 0, 4, AT), (ok, 514, 4, AT), (ok, 8, 0, AT), (ok, 8, 4, None), (ok, 8, 4, AT + 8),
                            (P.RotaryConfig(base=0.), 8, 4, AT), (P.RotaryConfig(base=float("inf")), 8, 4, AT),
                            (P.RotaryConfig(magnitude=float("nan")), 8, 4, AT), (P.RotaryConfig(scaling=4), 8, 4, AT),
                            (P.RotaryConfig(scaling=P.PLORA_ROTARY_LINEAR, factor=.5), 8, 4, AT), (P.RotaryConfig(scaling=P.PLORA_ROTARY_NTK, factor=2.), 2, 4, AT),
                            (P.RotaryConfig(scaling=P.PLORA_ROTARY_TURNS, factor=2., low=1., high=1., original_len=8), 8, 4, AT),
                            (P.RotaryConfig(scaling=P.PLORA_ROTARY_TURNS, factor=2., low=1., high=4.), 8, 4, AT)):
        rc = P.lib.plora_rotary_table(None if cfg is None else C.byref(cfg), rot, n, at, None)
        assert rc == P.PLORA_ERR_INVAL


def test_wrapper_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    with pytest.raises(P.PloraError):  # not on the GPU
        P.Rotary(torch.zeros(4, 8, 2), 16)
    with pytest.raises(P.PloraError):
        P.PagedKvCache(P.PLORA_BF16, 1, 64, 32, torch.zeros(2, 32 * 72, dtype=torch.uint8))
