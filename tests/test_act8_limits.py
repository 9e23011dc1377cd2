"""Checkpoint calls at the ends of their ranges: arguments are checked without overflow, on the host."""
import ctypes as C

import pytest

from paper_2609_09821_b200 import binding as B
from paper_2609_09821_b200 import build as lib_build

P = 1 << 20                    # an address nothing is read from: every call below is refused
LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return B.load()


def act8(ld_code=LAST, ld_scale=2 ** 26, code=P, scale=P, form=0):
    return C.byref(B.Act8View(code, ld_code, scale, ld_scale, form))


@pytest.mark.parametrize("N", [LAST, LAST - 30, LAST - 31])
def test_scales_too_narrow_for_the_widest_rows(lib, N):
    short = act8(ld_scale=-(-N // 32) - 1)
    assert lib.im_act8_pack(1, N, P, N, 1, short, None) == -1
    assert lib.im_act8_unpack(1, N, short, None, None, 0, P, N, 1, None) == -1
    assert lib.im_layer_norm_forward(1, N, P, N, 1, None, None, 1e-5, 0, P, N, 1, None, None, short, None) == -1
    assert lib.im_gemm_act8_tn(P, 64, act8(ld_code=2 ** 31, ld_scale=-(-N // 32) - 1), P, N, 64, 64, N, None, None, 0, P, 1 << 40, P, None) == -1


@pytest.mark.parametrize("name", ["gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "status"])
@pytest.mark.parametrize("off", [1, 2])
def test_vectors_that_lie_on_no_word(lib, name, off):
    at = dict.fromkeys(("gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "status"), P)
    at[name] += off
    ga, be, mean, rstd = at["gamma"], at["beta"], at["mean"], at["rstd"]
    ck = act8(ld_code=64, ld_scale=2)
    if name in ("gamma", "beta", "mean", "rstd"):
        assert lib.im_layer_norm_forward(4, 64, P, 64, 1, ga, be, 1e-5, 0, P, 64, 1, mean, rstd, None, None) == -1
    if name != "status":
        assert lib.im_layer_norm_backward(4, 64, P, 64, 1, P, 64, 1, mean, rstd, None, ga, be, 1, P, 64, at["dgamma"], at["dbeta"], P, 1 << 20, None) == -1
    if name in ("gamma", "beta"):
        assert lib.im_act8_unpack(4, 64, ck, ga, be, 0, P, 64, 1, None) == -1
    if name in ("gamma", "beta", "status"):
        assert lib.im_gemm_act8_tn(P, 64, ck, P, 64, 4, 64, 64, ga, be, 0, None, 0, at["status"], None) == -1
