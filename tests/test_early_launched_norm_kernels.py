"""The layer norm and 8-bit checkpoint kernels are launched with programmatic stream serialization: every one waits for its predecessor, and
none of its loads may claim that memory is read-only for the kernel's lifetime."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09821_b200", "csrc")


@pytest.mark.parametrize("name", ["norm.cu", "norm_backward.cu", "act8.cu", "act8_gemm.cu"])
def test_no_read_only_loads(name):
    text = open(os.path.join(CSRC, name)).read() + open(os.path.join(CSRC, "act8.cuh")).read()
    assert "launch_pdl(" in text and "__ldg(" not in text and "ld.global.nc" not in text and "<<<" not in text
    assert not re.search(r"const \w+ \*__restrict__", text)
    kernels = re.findall(r"__global__[^;{]*?\n?(\w+_kernel)\(.*?\n\{(.*?)\n\}\n", text, flags=re.S)
    assert kernels
    for kernel, body in kernels:
        assert "after_previous_kernel();" in body or "act8_tn_body<" in body, kernel
    assert name != "act8_gemm.cu" or text.count("after_previous_kernel();") >= 2
