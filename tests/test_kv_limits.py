"""Limits of the calls on the KV cache and what the wrappers refuse, without a GPU: every check is ahead of the first launch and no pointer is followed."""
import torch  # noqa: F401  (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P
from test_kv_refusals import batch, cache, rows


def test_attention_over_more_than_two_to_the_30_keys():
    """What the page table covers counts, up to max_len: past 2^30 the kernels' places would not fit 32 bits."""
    most = 1 << 30
    for stride, max_len in ((most // 64 + 1, 2 ** 31 - 1), (most // 64 + 1, most + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        b = batch(stride=stride, max_len=max_len)
        assert P.plora_kv_attend(cache(page=64), b, 8, rows(), rows(), 0.1) == P.PLORA_ERR_LIMIT
        assert P.plora_kv_attend(cache(page=64), b, 8, rows(), rows(), 0.1, 0) == P.PLORA_ERR_LIMIT


def test_the_library_holds_the_attention_kernels_that_calls_reach():
    """k_attend_many<dtype, head_dim, tiles of a wavefront, halves of q>: fp16 with both numbers of halves (rotated, or not), bf16 with 1, fp32 with 2."""
    import re
    names = set(re.findall(rb"k_attend_manyILi(\d)ELi(\d+)ELi(\d)ELi(\d)E", open(P.LIB_PATH, "rb").read()))
    built = {(int(dt), int(d), int(h)) for dt, d, _, h in names}
    assert built == {(dt, d, h) for d in (64, 128, 256) for dt, h in ((P.PLORA_F16, 1), (P.PLORA_F16, 2), (P.PLORA_BF16, 1), (P.PLORA_F32, 2))}
    assert len(names) == len(built)
