"""Norms between blocks: every kernel of the norm (a width for each of its eight classes of channels, rows gathered or not, with a gate and a norm ahead or
without), in every type.  The test itself, with its bounds, is test_gpu_base.test_norm."""
import pytest

import test_gpu_base as B

pytestmark = pytest.mark.gpu

WIDTHS = [120, 392, 776, 1544, 3112, 5128, 7176, 12296]  # k_norm: up to 128, 512, 1024, 2048, 4096, 6144, 8192, 16384 channels
PARTS = [dict(pre=B.RMS), dict(pre=B.LAYER, gate="rows", post=B.RMS, scale=0.5), dict(pre=B.RMS, post=B.LAYER), dict(pre=B.RMS, gate="one")]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("places", [0, 3])
@pytest.mark.parametrize("parts", PARTS, ids=["plain", "gate-post", "post", "gate"])
@pytest.mark.parametrize("width", WIDTHS)
def test_every_kernel(dtype, places, parts, width):
    B.test_norm(dtype, 5, width, dict(parts, top_k=places))
