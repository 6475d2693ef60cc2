"""CPU check of the narrow forward kernel's division of a piece's number by the pieces of a row (csrc/train_narrow.h).

A row too large and a piece of -1 would be 16 bytes read and written outside the row.  The host program under tests/host_checks
builds that same header, and only its host side runs; the launch must use the bound that the division is exact for.
"""
import os
import re
import subprocess

import test_kernel_hazards as hazards
from paper_2212_01185_amd import build as pcc_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@hazards.needs_hipcc
def test_rows_of_pieces_equal_integer_division(tmp_path):
    exe, src = str(tmp_path / "row_pieces_check"), os.path.join(ROOT, "tests", "host_checks", "row_pieces_check.cpp")
    flags = [f for f in pcc_build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([pcc_build.HIPCC, "-x", "hip"] + flags + ["-o", exe, src], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    res = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0 and res.stdout.split() == ["checked", str(32 * 50 * 51 // 2), "failures", "0"], res.stdout


def test_the_launch_keeps_to_that_bound():
    with open(pcc_build.TRAIN_SRC) as f:
        assert re.findall(r"narrow_row_pieces\([^()]*\) <= (\w+)", f.read()) == ["kMaxRowPieces"]
