"""CPU checks of the slot numbers that the weights' gradient forms
(csrc/slot_range.hpp, which its kernel is built from), up to the most slots that
a call takes, 2^31 - 257.  The program is built with the sanitizer for
arithmetic, which ends it at a sum past 31 bits."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_00079_amd", "csrc")
MOST = 2 ** 31 - 257


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("slots") / "check")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    f"-I{CSRC}", "-o", exe, os.path.join(HERE, "slot_range_check.cpp")], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return r.stdout.split()
    return run


@pytest.mark.parametrize("lo,hi", [(0, 0), (0, 1), (5, 5), (3, 70), (0, 4096), (1, 100001), (MOST, MOST),
                                   (MOST - 1, MOST), (MOST - 5000, MOST), (12345, MOST), (0, MOST),
                                   (0, MOST - 64), (0, 2 ** 31 - 16384), (0, 2 ** 31 - 16383)])
@pytest.mark.parametrize("parts", [1, 2, 3, 7, 32, 64, 100, 255, 256, 304])
def test_parts_cover_an_experts_slots(check, lo, hi, parts):
    assert check(lo, hi, parts, 64) == ["1"]


@pytest.mark.parametrize("lo,hi", [(0, 0), (0, 1), (7, 7), (3, 70), (1, 100001), (MOST, MOST), (MOST - 1, MOST),
                                   (MOST - 700, MOST - 254), (12345, MOST), (0, MOST)])
def test_slots_asked_for_ahead(check, lo, hi):
    """Eight stages of 64 slots at once, from every eighth stage that has a slot on: the first and last of them, and
    those around the expert's end."""
    last = max(0, hi - lo - 1) // 512 * 512
    for ahead in sorted({0, 1, 511, last, last + 1, last + 511, max(0, hi - lo - 1), hi - lo, min(hi - lo + 1, last + 511)}):
        assert check(lo, hi, ahead) == [str(lo + ahead if lo + ahead < hi else -1)], ahead
