"""Groups of rows that overlap (offsets that are not ascending): a row of one group alone is that group's product, a row of none stays as it was; what
groups share is undefined.  Bounds as in test_gpu_base.py."""
import numpy as np
import pytest

import test_gpu_base as B

pytestmark = pytest.mark.gpu


def overlapping(experts, total, high):
    """Every other group is rows 0 .. high - 1, the last one the rows behind them."""
    return np.array([high * (e % 2) for e in range(experts)] + [total])


# more tiles than a call with ascending offsets can have, for tiles and for few rows, with more experts than a wavefront has lanes, and rows that lie behind,
# ahead of and between the overlapping ones
CASES = [(overlapping(6, 1500, 1000), 1500, 72, 2064), (overlapping(6, 1500, 1000), 1500, 264, 144), (overlapping(6, 1500, 1000), 1500, 2056, 272),
         (overlapping(40, 300, 250), 300, 136, 528), (overlapping(130, 900, 820), 900, 72, 1424), (overlapping(130, 5000, 4600), 5000, 136, 272),
         (np.array([900, 1500, 100, 700, 100, 700, 100, 700, 0, 100]), 1500, 520, 1040), (np.array([500, 600, 0, 450, 0, 450, 0, 450, 700, 650]), 800, 1032, 144)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("offsets,total,n,k", CASES, ids=[str(i) for i in range(len(CASES))])
def test_rows_of_one_group_alone(dtype, offsets, total, n, k):
    import torch
    P = B.lib()
    rng = np.random.default_rng(total + n)
    experts = len(offsets) - 1
    xc, wc = B.random_codes(rng, total, k), B.random_codes(rng, experts, n, k)
    xs, ws = (np.exp(rng.normal(size=z)).astype(np.float32) for z in ((-(-k // 128), total), (experts, -(-n // 128), -(-k // 128))))
    xs /= 30 * k
    put = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    x, w = P.Fp8Rows(put(xc), put(xs)), P.Fp8Weights(put(wc), put(ws))
    out = torch.full((total, n), 7.0, device="cuda", dtype=getattr(torch, B.DT[dtype][1]))
    w.grouped(x, B.ints(offsets), out, stream=B.stream())
    got, xv = B.host(out), B.O.row_values(xc, xs)
    claims, of = np.zeros(total, int), np.full(total, -1)
    for e in range(experts):
        claims[offsets[e]:offsets[e + 1]] += 1
        of[offsets[e]:offsets[e + 1]] = e
    assert (got[claims == 0] == 7).all()
    alone = np.unique(of[claims == 1])
    assert len(alone)
    for e in alone:
        r = (of == e) & (claims == 1)
        B.check_product(got[r], xv[r], B.O.weight_values(wc[e], ws[e]), dtype)
