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
