"""Which kernels the 8-bit products choose (no GPU): the calls of base_tiles.py run each of them, in every type, over few blocks of K and over many."""
import re

import pytest
import torch  # noqa: F401  (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P
from base_tiles import EXPERTS, LARGEST, STAGES, calls

DTYPES = (P.PLORA_BF16, P.PLORA_F16, P.PLORA_F32)


def rows8(k, n):
    return P.Fp8RowsStruct(None, None, k, n)


def tile_of(t, n, k, dtype, grouped=False, gathered=False, experts=None, stride=None, x_rows=None):
    w = P.Fp8WeightsStruct(experts or (EXPERTS if grouped else 1), n, k, None, None)
    rc, tile = P.plora_fp8_tile_of(rows8(stride or k, t), x_rows or t, w, dtype, t, grouped, gathered)
    assert rc == P.PLORA_OK
    return tile


@pytest.mark.parametrize("gathered", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("grouped", [False, True])
def test_every_kernel_is_run(grouped, dtype, gathered):
    if gathered and not grouped:
        return
    blocks = {kernel: set() for kernel in STAGES}
    for kernel, t, n, k in calls(grouped):
        got = tile_of(t, n, k, dtype, grouped, gathered)
        assert got == kernel or (kernel == LARGEST and dtype == P.PLORA_F32 and got != LARGEST)
        blocks[got].add(-(-k // 128))
    for kernel, stages in STAGES.items():
        if kernel == LARGEST and dtype == P.PLORA_F32:
            assert not blocks[kernel]
            continue
        steps = {-(-b // kernel[2]) for b in blocks[kernel]}
        if stages is None:  # a wavefront's loop, two blocks a turn: entered with more than 3 blocks each; and calls that do not reach it
            assert max(steps) > 3 and min(steps) <= 3
        else:  # the stages go round more than twice
            assert max(steps) > 2 * stages
            if kernel in ((64, 64, 1), (64, 128, 1), (128, 256, 1), LARGEST):  # the others are not chosen for that few
                assert {1, 3, 4, 5} <= steps


def test_the_library_holds_the_kernels_that_calls_reach():
    names = open(P.LIB_PATH, "rb").read()
    few = set(re.findall(rb"k_fewILi(\d)ELi(\d+)ELi(\d)ELi(\d)ELi\dELb(\d)E", names))
    tiled = set(re.findall(rb"k_productILi(\d)ELi(\d+)ELi(\d+)ELi\dELi\dELi(\d)ELi(\d)ELb\dELb(\d)E", names))
    built = {((int(r), 16 * int(c), int(p)), int(d), int(g)) for d, r, c, p, g in few} | {((int(r), int(c), int(p)), int(d), int(g)) for d, r, c, p, s, g in tiled}
    assert built == {(kernel, d, g) for kernel in STAGES for d in DTYPES for g in (0, 1) if (kernel, d) != (LARGEST, P.PLORA_F32)}
    for d, r, c, p, s, g in tiled:
        assert STAGES[int(r), int(c), int(p)] == int(s)


def test_both_sides_of_a_border():
    for dtype in DTYPES:
        assert tile_of(1, 32776, 1408, dtype)[2] == 2 and tile_of(1, 32776, 1424, dtype)[2] == 4
        assert tile_of(16, 4096, 4096, dtype)[0] == 16 and tile_of(17, 4096, 4096, dtype)[0] > 16
        assert tile_of(64, 512, 1024, dtype, True, experts=8)[0] == 16 and tile_of(65, 512, 1024, dtype, True, experts=8)[0] > 16
        # rows further apart than 31 bits: of a tile of 256, or of all that may be gathered
        assert tile_of(600, 4096, 4096, dtype, stride=1 << 23)[0] == 16 and tile_of(600, 4096, 4096, dtype, stride=1 << 22)[0] > 16
        assert tile_of(5000, 4096, 4096, dtype, True, True, stride=1 << 20)[0] == 16 and tile_of(5000, 4096, 4096, dtype, True, False, stride=1 << 20)[0] > 16


def test_refusals():
    w = P.Fp8WeightsStruct(1, 256, 256, None, None)
    ok = (rows8(256, 8), 8, w, P.PLORA_BF16, 8, False, False)
    assert P.plora_fp8_tile_of(*ok)[0] == P.PLORA_OK
    for i, v in [(0, None), (0, rows8(-16, 8)), (0, rows8(1 << 41, 8)), (1, 0), (2, None), (2, P.Fp8WeightsStruct(2, 256, 256, None, None)), (2, P.Fp8WeightsStruct(1, 252, 256, None, None)),
                 (2, P.Fp8WeightsStruct(1, 256, 264, None, None)), (3, 5), (4, 0), (6, True)]:
        assert P.plora_fp8_tile_of(*ok[:i], v, *ok[i + 1:])[0] == P.PLORA_ERR_INVAL
    assert P.lib.plora_fp8_tile_of(*ok, None) == P.PLORA_ERR_INVAL
