"""The tensor-core kernels of the weight gradient keep their values in registers: a spill would lie next to registers that loads from tensor
memory write while other instructions run."""
import os
import re
import subprocess

from paper_2609_09821_b200 import build as lib_build


def test_no_kernel_of_the_weight_gradient_spills(tmp_path):
    source = os.path.join(lib_build.CSRC, "act8_gemm.cu")
    done = subprocess.run([lib_build._nvcc()] + lib_build.NVCC_FLAGS + ["-Xptxas", "-v", "-c", source, "-o", str(tmp_path / "o")], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    spills = re.findall(r"Function properties for (\S+)\n\s*(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", done.stderr)
    assert len(spills) >= 18
    assert not [s for s in spills if s[1:] != ("0", "0", "0")]
