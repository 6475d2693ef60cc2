"""The checks of the compiled kernels of test_kernel_hazards.py for the operators round the grouped products: no scalar result of the vector
ALU is read too soon on any path, no packed fp32 arithmetic, and nothing spills.  On the CPU."""
import functools
import os
import re
import subprocess
import tempfile

import test_kernel_hazards as hazards
from paper_2212_01185_amd import build as pcc_build


@functools.lru_cache(maxsize=None)
def _assembly():
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "routed.s")
        flags = [f for f in pcc_build.FLAGS if f not in ("-shared", "-fPIC")]
        subprocess.run([pcc_build.HIPCC] + flags + ["--cuda-device-only", "-S", "-o", out, pcc_build.ROUTED_SRC], check=True, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT)
        with open(out) as f:
            return f.read()


@hazards.needs_hipcc
def test_no_scalar_result_of_the_vector_alu_is_read_early_on_any_path():
    assert len([n for n, _, _ in hazards._functions(_assembly().split("\n"))]) >= 50
    found, _ = hazards.early_scalar_reads(_assembly())
    assert found == []


@hazards.needs_hipcc
def test_no_packed_fp32_arithmetic():
    assert re.search(r"v_pk_(add|mul|fma)_f32", _assembly()) is None


@hazards.needs_hipcc
def test_no_kernel_spills():
    sizes = [int(v) for v in re.findall(r"\.vgpr_spill_count:\s*(\d+)", _assembly())]
    assert sizes and max(sizes) == 0
