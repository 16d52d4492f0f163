"""What the base layer's wrappers refuse, without a GPU and without memory: the tensors have shapes alone."""
import pytest
import torch

import paper_2512_20210_amd as P

BIG = 1 << 32


class Shaped:
    """Stands for a contiguous torch tensor of GPU 0."""

    def __init__(self, dtype, *shape):
        self.t = torch.empty(shape, dtype=dtype, device="meta")
        self.dtype, self.shape, self.stride, self.dim, self.numel = dtype, self.t.shape, self.t.stride, self.t.dim, self.t.numel
        self.is_contiguous, self.nbytes = self.t.is_contiguous, self.t.nbytes

    def get_device(self):
        return 0

    def data_ptr(self):
        return 0x10008  # (no call takes it: none gets as far as a launch)


def rows(n, k):
    return P.Fp8Rows(Shaped(torch.uint8, n, k), Shaped(torch.float32, -(-k // 128), n))


def weights(*shape):
    return P.Fp8Weights(Shaped(torch.uint8, *shape), Shaped(torch.float32, *shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128)))


def routing(n, k, experts):
    i = lambda *z: Shaped(torch.int32, *z)  # noqa: E731
    return P.Routing(i(n, k), Shaped(torch.float32, n, k), i(experts + 1), i(n * k), i(n, k), Shaped(torch.uint8, 1 << 20))


def norm(n, dim, top_k=0, block_rows=None):
    f = lambda *z: Shaped(torch.bfloat16, *z)  # noqa: E731
    kw = dict(places=Shaped(torch.int32, n, top_k), place_weights=Shaped(torch.float32, n, top_k)) if top_k else {}
    return P.BlockNorm().run(f(n if block_rows is None else block_rows, dim), out=f(n, dim), **kw)


@pytest.mark.parametrize("call", [
    lambda: rows(BIG + 8, 64), lambda: rows(8, BIG + 64), lambda: rows(1 << 31, 64),
    lambda: weights(BIG + 8, 64), lambda: weights(8, BIG + 64), lambda: weights(BIG + 1, 8, 64), lambda: weights(2, BIG + 8, 64),
    lambda: routing(BIG + 3, 2, 8), lambda: routing(3, 2, BIG + 8), lambda: norm(BIG + 3, 64), lambda: norm(3, BIG + 64),
    lambda: norm(3, 64, 2, BIG + 5), lambda: norm(BIG + 3, 64, 2, 5),
    lambda: weights(2, 8, 64).grouped(rows(4, 64), Shaped(torch.int32, 3), Shaped(torch.bfloat16, BIG + 4, 8), Shaped(torch.int32, BIG + 4))])
def test_counts_past_32_bits(monkeypatch, call):
    """Refused, and not taken modulo 2^32."""
    monkeypatch.setattr(P.binding, "_device", lambda: 0)
    with pytest.raises(P.PloraError, match="LIMIT"):
        call()


def test_the_largest_counts_are_taken():
    """(Nothing is launched: these only hold what a call is given.)"""
    assert rows((1 << 31) - 1, 16).n == (1 << 31) - 1 and weights(8, 1 << 20).k == 1 << 20 and routing((1 << 31) - 1, 1, 8).n == (1 << 31) - 1


@pytest.mark.parametrize("width", [0, 1, 63, 128])
def test_a_gate_of_another_width(monkeypatch, width):
    monkeypatch.setattr(P.binding, "_device", lambda: 0)
    f = lambda *z: Shaped(torch.bfloat16, *z)  # noqa: E731
    gate = f(width)
    gate.expand = lambda *z: gate.t.expand(*z)
    with pytest.raises(P.PloraError, match="INVAL"):
        P.BlockNorm().run(f(3, 64), out=f(3, 64), gate=gate)
