"""Registers that the kernels of adapters, adjusted logits and the distillation from top logits spill, read from the metadata of the built library: none, but
for those named here, and those no more."""
import os
import re

import pytest

from paper_2507_02659_amd import build
from test_kernel_resources import _kernels

pytestmark = pytest.mark.skipif(not os.path.exists(build.LIB_PATH), reason="not built")

# most spilled vector registers by the mangled name's part that tells a kernel from its kind: ranks 33 to 64 of bfloat16 matrices with bfloat16 and with
# float32 logits; rows of more than 524288 bfloat16 logits (a few: of more than 196608), with gradient
MOST = {"adapter_up_kernelIttLi2E": 4, "adapter_up_kernelItfLi2E": 12, "top_distill_kernelItLi1024ELi12ELb1ELb0E": 38}


def test_spills():
    seen = set()
    for k in _kernels():
        m = re.search(r"\d((?:adapter_(?:up|down)|adjust|top_distill)_kernelI\w+?E)E*v", k[".name"])
        if not m:
            continue
        seen.add(m[1].split("_kernel")[0])
        most = [n for key, n in MOST.items() if key in k[".name"]]
        assert k[".vgpr_spill_count"] <= (most[0] if most else 0), (k[".name"], k[".vgpr_spill_count"])
    assert seen == {"adapter_up", "adapter_down", "adjust", "top_distill"}
