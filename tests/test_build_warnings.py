"""What the compiler can tell of the sources without running them."""
import os
import subprocess

import pytest

from paper_2011_09017_amd import build


@pytest.mark.parametrize("source", [s for s in build.SOURCES if "byte" in s or "norm" in s or "linear" in s])
def test_no_order_of_evaluation_is_taken_for_granted(source):
    """Host code of the plans: nothing modifies a value and reads it in one expression whose order the language leaves open."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no compiler here")
    run = subprocess.run([hipcc, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-fsyntax-only", "-Wunsequenced", "-Werror=unsequenced",
                          os.path.join(build.CSRC, source)], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
