"""Limits of the calls on the KV cache and what the wrappers refuse, without a GPU: every check is ahead of the first launch and no pointer is followed."""
import pytest
import torch  # (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P
from test_kv_refusals import AT, batch, cache, rows


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


class OnGpu:
    """Stands for a torch tensor of a GPU: what the wrappers look at."""

    def __init__(self, device, dtype, *shape):
        self.gpu, self.dtype, self.shape, self.is_cuda = device, dtype, torch.Size(shape), device >= 0

    def get_device(self):
        return self.gpu

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return AT

    nbytes = 1 << 20


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    """A call's tensors, batch, cache and table have to be on the current GPU.  (Batches without tokens: nothing is launched where all fits.)"""
    monkeypatch.setattr(P.binding, "_device", lambda: 0)

    def parts(device):
        i32 = [OnGpu(device, torch.int32, *s) for s in ((3,), (2,), (2, 4))]
        return (P.PagedKvCache(P.PLORA_BF16, 1, 64, 32, OnGpu(device, torch.uint8, 8, 32 * 72)), P.KvBatch(*i32, 0, 1, 100),
                P.Rotary(OnGpu(device, torch.float32, 16, 32, 2), 64), OnGpu(device, torch.bfloat16, 0, 1, 64), OnGpu(device, torch.int32, 0), OnGpu(device, torch.uint8, 1 << 20))

    here, there = parts(0), parts(1)
    mixtures = [here] + [tuple(there[k] if k == i else h for k, h in enumerate(here)) for i in range(len(here))] + [there]
    for n, (kv, b, rotary, rows_, at, ws) in enumerate(mixtures):
        calls = [(lambda: kv.append(b, rows_, rows_, rotary), {0, 5, 6}), (lambda: kv.read(b, rows_, rows_), {0, 3, 5, 6}),
                 (lambda: kv.attend(b, rows_, rows_, 0.1, ws, rotary=rotary), {0, 5}), (lambda: rotary.rotate(at, rows_, rows_), {0, 1, 2, 6})]
        for call, fine in calls:
            if n in fine:
                call()
            else:
                with pytest.raises(P.PloraError, match="INVAL"):
                    call()
    mixed = [OnGpu(d, torch.int32, *s) for d, s in ((0, (3,)), (1, (2,)), (0, (2, 4)))]
    with pytest.raises(P.PloraError, match="INVAL"):
        P.KvBatch(*mixed, 0, 1, 100)
    with pytest.raises(P.PloraError, match="INVAL"):
        P.KvBatch(*[OnGpu(-1, torch.int32, *t.shape) for t in mixed], 0, 1, 100)
    with pytest.raises(P.PloraError, match="INVAL"):
        P.Rotary.make(OnGpu(1, torch.float32, 16, 32, 2))


def test_tensors_with_other_dimensions_are_refused():
    for make in (lambda: P.Rotary.make(OnGpu(0, torch.float32, 64)), lambda: P.Rotary(OnGpu(0, torch.float32, 64), 64),
                 lambda: P.PagedKvCache(P.PLORA_BF16, 1, 64, 32, OnGpu(0, torch.uint8)), lambda: P.PagedKvCache(P.PLORA_BF16, 1, 64, 32, OnGpu(0, torch.uint8, 32 * 72))):
        with pytest.raises(P.PloraError, match="INVAL"):
            make()
