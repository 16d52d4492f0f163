"""What the attention's calls launch: counted as nodes of a captured graph."""
import ctypes as C

import numpy as np
import pytest

from test_gpu_kv import Setup, check_attention, ints, put, stream  # noqa: F401

pytestmark = pytest.mark.gpu


def kernels_of(call):
    import torch
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    path = next(l.split()[-1] for l in open("/proc/self/maps") if "libamdhip64" in l)
    n = C.c_size_t(0)
    assert C.CDLL(path).hipGraphGetNodes(C.c_void_p(graph.raw_cuda_graph()), None, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("heads,new,ctx,expected", [(32, [1, 1, 1, 2], [90, 7, 400, 0], 1),   # no sequence has 16 rows or fewer
                                                    (4, [1, 1, 1, 2], [90, 7, 400, 0], 1),    # all have
                                                    (4, [1, 1, 30, 1], [90, 7, 400, 0], 2)])  # some have
def test_a_call_launches_what_finds_rows(heads, new, ctx, expected):
    s = Setup("bf16", 1, 64, 64, new, ctx)
    q, _ = put(np.zeros((s.tokens, heads, 64)), "bf16")
    out = q.clone()
    batch = s.batch()
    assert kernels_of(lambda: s.cache.attend(batch, q, out, 0.125, None, stream=stream())) == expected


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("heads,kvh,new,ctx", [(32, 1, [1, 1, 4, 1], [90, 0, 400, 2500]), (34, 2, [1] * 6, [0, 1, 31, 32, 64, 700]), (24, 1, [2, 1, 17], [300, 5, 0])])
@pytest.mark.parametrize("workspace", [0, 1 << 22])
def test_more_than_16_query_heads_a_kv_head(dtype, heads, kvh, new, ctx, workspace):
    check_attention(Setup(dtype, kvh, 64, 64, new, ctx), heads, workspace=workspace)
    check_attention(Setup(dtype, kvh, 64, 64, new, ctx), heads, workspace=workspace, window=40, rot=64)
