"""The checks of test_isa_lds_waits.py on the cross-attention and rotary kernels."""
import os
import re

import pytest

from tests import test_isa_lds_waits as isa

CSRC = os.path.dirname(isa.SRC)


@pytest.mark.parametrize("src,reads,kernels", [("cross.hip", 1000, 19), ("rotary.hip", 0, 12)])
def test_lds_waits_and_no_scratch(src, reads, kernels):
    asm = isa.device_asm(os.path.join(CSRC, src))
    hazards, checked = isa.lds_wait_hazards(asm)
    assert checked >= reads and not hazards, hazards[:20]
    sizes = re.findall(r"^\s*\.private_segment_fixed_size:\s*(\d+)", asm, re.M)
    assert len(sizes) >= kernels and not any(int(x) for x in sizes)
