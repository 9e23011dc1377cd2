"""The layer norm and 8-bit checkpoint kernels are launched while the kernel before them may still run: none touches global memory before it
has waited for that one."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09821_b200", "csrc")
WAIT = "after_previous_kernel();"
# what reads or writes global memory: the load and store helpers, PTX accesses, copies, an element of a pointer argument or of a pointer made from
# one, and what it points to
TOUCHES = re.compile(r"\b(load8|load_codes8|store8|store_codes8|full8|full_store8|keep8|keep_side8|store_as|load_scales|load_row|tma_load_\w+|atomic\w+|__ld\w+|__st\w+)\s*[<(]"
                     r"|\b(ld|st|red|atom)\.global|cp\.async|\bP\.(\w+\.)?\w+\[|\*\s*\(?P\.|\b(x|y|dx|dy|out|in|partial|gamma|beta|px|py|src|dst|row)\[|(?<![\w)>])\*(px|py|src|dst|out)\b|part_at")


def early_accesses(body):
    """What a kernel's body does to global memory before its wait (comments taken out)."""
    body = re.sub(r"//[^\n]*", "", body)
    assert body.count(WAIT) == 1
    return [m.group(0) for m in TOUCHES.finditer(body[:body.index(WAIT)])]


def bodies(name):
    text = open(os.path.join(CSRC, name)).read()
    found = re.findall(r"__global__[^;{]*?(\w+_kernel)\([^{]*?\)\n\{\n(.*?)\n\}\n", text, flags=re.S)
    return dict(found + re.findall(r"void (act8_tn_body)\([^{]*?\)\n\{\n(.*?)\n\}\n", text, flags=re.S))


KERNELS = {"norm.cu": ["norm_forward_kernel", "norm_finish_kernel"], "norm_backward.cu": ["norm_backward_kernel"], "act8.cu": ["pack_kernel", "unpack_kernel"],
           "act8_gemm.cu": ["act8_tn_body", "act8_tn_finish_kernel"]}


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_nothing_is_read_or_written_before_the_wait(name):
    found = bodies(name)
    callers = {k for k, b in found.items() if "act8_tn_body<" in b and b.count("\n") == 0}         # a call of the body and nothing else
    assert set(found) - callers == set(KERNELS[name])
    for kernel in KERNELS[name]:
        assert early_accesses(found[kernel]) == [], kernel


@pytest.mark.parametrize("name,kernel,line", [("norm.cu", "norm_forward_kernel", "load_row((long long)blockIdx.x * kGroups + g);"), ("act8.cu", "unpack_kernel", "const float g0 = gamma[0];"),
                                              ("norm.cu", "norm_finish_kernel", "double s0 = (double)__ldcg(partial);"), ("norm_backward.cu", "norm_backward_kernel", "const float m = P.mean[0];"),
                                              ("act8_gemm.cu", "act8_tn_body", "uint32_t w = load_scales(P.h.scale, 4, true);"), ("act8.cu", "pack_kernel", "Eight<T> e = load8<VEC>(x, col, 1, N);")])
def test_an_early_access_is_found(name, kernel, line):
    body = bodies(name)[kernel]
    assert early_accesses(body.replace(WAIT, line + "\n" + WAIT)) != []
