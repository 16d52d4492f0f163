"""Routing takes logits from any element on: the loads that the compiler makes of its source promise no more alignment than an element has (CPU only; the
kernels are compiled for the GPU, as far as the compiler's own form of them)."""
import os
import re
import subprocess

import pytest
import torch  # noqa: F401  (ahead of the package: both then share the HIP runtime that torch brings)

import paper_2512_20210_amd as P

CSRC = os.path.join(os.path.dirname(os.path.abspath(P.__file__)), "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_loads_of_logits_promise_an_elements_alignment(tmp_path):
    to = str(tmp_path / "base.ll")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-w", "--offload-device-only", "-S", "-emit-llvm", os.path.join(CSRC, "plora_base.hip"), "-o", to],
                   check=True, timeout=110)
    most = {P.PLORA_F16: 2, P.PLORA_BF16: 2, P.PLORA_F32: 4}
    seen = set()
    for dtype, body in re.findall(r"^define [^\n]*@\S*k_route_chooseILi(\d)E\S*\((.*?)^}", open(to).read(), re.S | re.M):
        loads = [int(a) for a in re.findall(r"= load [^\n]*ptr addrspace\(1\)[^\n]*align (\d+)", body)]
        assert loads and max(loads) <= most[int(dtype)]
        seen.add(int(dtype))
    assert seen == set(most)
