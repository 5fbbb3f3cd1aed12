"""CPU check of the kernels' inline assembly: an instruction that loads straight
into LDS takes its address from M0, and needs a wait state after the write of
M0 (the compiler inserts one between its own; it does not look into assembly)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_00079_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))), ids=os.path.basename)
def test_a_wait_state_between_m0_and_the_load(path):
    with open(path) as f:
        text = f.read()
    for asm in re.findall(r'asm\s+volatile\(\s*"([^;]*?)"\s*:', text):
        lines = [p.strip() for p in asm.replace('"', "").split("\\n\\t")]
        for before, after in zip(lines, lines[1:]):
            assert not ("m0," in before and "load_lds" in after), (before, after)
