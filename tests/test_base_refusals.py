"""What the base layer's calls refuse.  Every check is ahead of the first launch, so these run without a GPU; the pointers are never
followed."""
import ctypes as C

import pytest
import torch  # noqa: F401  (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P

AT, FAR = 0x10000, 0x9000000
INVAL, LIMIT = P.PLORA_ERR_INVAL, P.PLORA_ERR_LIMIT


def matrix(data=AT, stride=256):
    return P.MatrixStruct(data, stride)


def rows8(codes=AT, scales=FAR, stride=256, scale_stride=64):
    return P.Fp8RowsStruct(codes, scales, stride, scale_stride)


def weights8(e=1, n=256, k=256, codes=AT, scales=FAR):
    return P.Fp8WeightsStruct(e, n, k, codes, scales)


def norm_of(weight=AT, bias=None, eps=1e-6, offset=0.0, center=0):
    return P.NormWeightsStruct(weight, bias, eps, offset, center)


def block(**kw):
    a = dict(dtype=P.PLORA_BF16, n_tokens=3, dim=256, scale=1.0, block=matrix(), places=None, place_weights=None, top_k=0, n_block_rows=0, post=None, pre=norm_of(),
             gate=None, residual=None, hidden=None, out=matrix(FAR), out8=None)
    a.update(kw)
    flat = []
    for name, v in a.items():
        if name in ("post", "pre"):
            flat.append(None if v is None else C.addressof(v))
            kept.append(v)
        elif name == "out8":
            flat += [None, None, 0, 0] if v is None else [getattr(v, f) for f, _ in v._fields_]
        elif name in ("block", "gate", "residual", "hidden", "out"):
            flat += [None, 0] if v is None else [v.data, v.stride]
        else:
            flat.append(v)
    return P.BlockNormStruct(*flat)


kept = []  # what the records point to
BAD_MATRIX = [matrix(None), matrix(AT + 8), matrix(stride=-256), matrix(stride=257), matrix(stride=1 << 41)]
BAD_OUT = BAD_MATRIX + [matrix(stride=0), matrix(stride=248)]
BAD_EIGHT = [rows8(None), rows8(AT + 8), rows8(scales=None), rows8(scales=FAR + 2), rows8(stride=252), rows8(stride=248), rows8(stride=-256), rows8(scale_stride=2),
             rows8(stride=1 << 41), rows8(scale_stride=1 << 41)]


def test_nothing_to_do_is_fine():
    assert P.plora_norm(block(n_tokens=0, block=None, out=matrix(None))) == 0
    assert P.plora_fp8_quantise(P.PLORA_F16, 0, 256, None, 0, None) == 0
    assert P.plora_fp8_matmul(None, weights8(), P.PLORA_F32, 0, None) == 0
    assert P.plora_fp8_grouped(None, 0, weights8(4), None, None, P.PLORA_F32, 0, None) == 0


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(n_tokens=-1), dict(dim=0), dict(dim=260), dict(dim=16392), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(block=None), dict(out=None), dict(out8=rows8()), dict(pre=norm_of(AT + 2)), dict(pre=norm_of(bias=AT + 4)), dict(pre=norm_of(eps=-1.)),
                                dict(pre=norm_of(eps=float("inf"))), dict(pre=norm_of(eps=float("nan"))), dict(post=norm_of(offset=float("nan"))),
                                dict(post=norm_of(center=2)), dict(places=AT), dict(place_weights=AT), dict(places=AT, place_weights=AT, top_k=0, n_block_rows=4),
                                dict(places=AT, place_weights=AT, top_k=33, n_block_rows=4), dict(places=AT, place_weights=AT, top_k=2, n_block_rows=-1),
                                # in place: not with places, not with another stride, and not two results in one
                                dict(places=AT, place_weights=AT, top_k=2, n_block_rows=4, out=matrix(AT)), dict(out=matrix(AT, 264)),
                                dict(hidden=matrix(FAR)), dict(residual=matrix(FAR, 0)), dict(gate=matrix(FAR, 0))])
def test_norms(kw):
    assert P.plora_norm(block(**kw)) == INVAL


def test_norm_matrices():
    for m in BAD_MATRIX:
        assert P.plora_norm(block(block=m)) == INVAL
        if m.data:  # (none is no gate)
            assert P.plora_norm(block(gate=m)) == P.plora_norm(block(residual=m)) == INVAL
    for m in BAD_OUT:
        assert P.plora_norm(block(out=m)) == INVAL
        assert not m.data or P.plora_norm(block(hidden=m)) == INVAL
    for r in BAD_EIGHT:
        assert P.plora_norm(block(out=None, out8=r)) == INVAL
    assert P.lib.plora_norm(None, None) == INVAL


def test_quantise():
    good = dict(dtype=P.PLORA_BF16, n_rows=3, k=256, x=matrix(), activation=0, out=rows8())
    for kw in [dict(dtype=5), dict(n_rows=-1), dict(k=0), dict(k=252), dict(k=(1 << 20) + 8), dict(activation=-1), dict(activation=3), dict(x=None), dict(out=None)] + \
            [dict(x=m) for m in BAD_MATRIX] + [dict(out=r) for r in BAD_EIGHT]:
        assert P.plora_fp8_quantise(**{**good, **kw}) == INVAL


BAD_WEIGHTS = [None, weights8(0), weights8(1025), weights8(n=0), weights8(n=252), weights8(n=(1 << 20) + 8), weights8(k=0), weights8(k=264), weights8(k=(1 << 20) + 16)]
BAD_POINTERS = [weights8(codes=None), weights8(codes=AT + 8), weights8(scales=None), weights8(scales=FAR + 1)]


def test_quantise_weights():
    for w in BAD_WEIGHTS + BAD_POINTERS:
        assert P.plora_fp8_quantise_weights(P.PLORA_F16, matrix(), w) == INVAL
    for m in BAD_MATRIX + [None]:
        assert P.plora_fp8_quantise_weights(P.PLORA_F16, m, weights8()) == INVAL
    assert P.plora_fp8_quantise_weights(3, matrix(), weights8()) == INVAL


def test_products():
    good = dict(x=rows8(), w=weights8(), dtype=P.PLORA_BF16, n_rows=3, out=matrix())
    more = dict(x=rows8(), n_x_rows=3, w=weights8(4), offsets_ptr=AT, rows_ptr=None, dtype=P.PLORA_BF16, n_rows=3, out=matrix())
    bad = [dict(w=w) for w in BAD_WEIGHTS + BAD_POINTERS] + [dict(dtype=-1), dict(n_rows=-1), dict(x=None), dict(out=None), dict(x=rows8(stride=264))] + \
        [dict(x=r) for r in BAD_EIGHT] + [dict(out=m) for m in BAD_OUT]
    for kw in bad + [dict(w=weights8(2)), dict(n_rows=65)]:  # (more rows than scales)
        assert P.plora_fp8_matmul(**{**good, **kw}) == INVAL
    for kw in bad + [dict(offsets_ptr=None), dict(n_x_rows=-1), dict(n_x_rows=2), dict(rows_ptr=AT, n_x_rows=0), dict(rows_ptr=AT, n_x_rows=65)]:
        assert P.plora_fp8_grouped(**{**more, **kw}) == INVAL


def test_routing():
    good = dict(dtype=P.PLORA_F32, n_tokens=3, n_experts=8, top_k=2, logits=matrix(), renormalise=1, scale=1.0, experts_ptr=AT, weights_ptr=AT, offsets_ptr=AT,
                rows_ptr=AT, places_ptr=AT, workspace_ptr=AT, workspace_bytes=1 << 20)
    for kw in [dict(dtype=4), dict(n_tokens=-1), dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=9), dict(n_experts=64, top_k=33), dict(logits=None),
               dict(logits=matrix(None)), dict(logits=matrix(AT + 2)), dict(logits=matrix(stride=-1)), dict(logits=matrix(stride=1 << 41)), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(experts_ptr=None), dict(weights_ptr=None), dict(offsets_ptr=None), dict(rows_ptr=None), dict(places_ptr=None),
               dict(workspace_ptr=AT + 8), dict(workspace_ptr=None), dict(n_tokens=65, workspace_bytes=8 * 6 * 4 - 1)]:
        assert P.plora_route(**{**good, **kw}) == INVAL
    assert P.plora_route(**{**good, "n_tokens": 1 << 30, "workspace_bytes": 1 << 40}) == LIMIT


def test_workspace_of_routing():
    assert P.plora_route_workspace_bytes(64, 512) == P.plora_route_workspace_bytes(0, 1024) == 0 and P.plora_route_workspace_bytes(1, 513) == 513 * 2 * 4 and P.plora_route_workspace_bytes(65, 8) == 8 * 6 * 4
    assert P.plora_route_workspace_bytes(300, 0) == P.plora_route_workspace_bytes(300, 1025) == P.plora_route_workspace_bytes(-5, 8) == 0


def test_wrappers_refuse_tensors_that_do_not_fit():
    t = torch
    u8, f32 = t.uint8, t.float32
    for make in (lambda: P.Fp8Rows(t.zeros(2, 64, dtype=u8), t.zeros(1, 2)), lambda: P.Fp8Weights(t.zeros(8, 64, dtype=u8), t.zeros(1, 1)),
                 lambda: P.Fp8Rows(t.zeros(64, dtype=u8), t.zeros(1, 2)), lambda: P.NormWeights(t.zeros(8)),
                 lambda: P.Routing(*(t.zeros(2, 2, dtype=t.int32),) * 5)):
        with pytest.raises(P.PloraError):  # not on the GPU, or of other dimensions
            make()
