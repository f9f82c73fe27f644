"""The compiler's own check of constant array indexes (host logic, no GPU)."""
import os
import subprocess

import pytest

from paper_2410_09615_amd import build


@pytest.mark.parametrize("source", build.sources(), ids=os.path.basename)
def test_no_constant_index_leaves_its_array(source):
    """Kernels whose loops are unrolled by templates index register arrays with constants; the compiler sees one that is outside."""
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    run = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-Werror=array-bounds", "--cuda-device-only", "-fsyntax-only", "-I",
                          os.path.join(build.ROOT, "include"), "-I", build.CSRC, source], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-2000:]
