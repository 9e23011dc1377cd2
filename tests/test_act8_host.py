"""Refusals of the layer norm and 8-bit checkpoint calls, on the host: bad arguments are turned down before any device work."""
import ctypes as C

import pytest

from paper_2609_09821_b200 import binding as B
from paper_2609_09821_b200 import build as lib_build

P = 1 << 20                    # an address nothing is read from: every call below is refused


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return B.load()


def act8(code=P, ld_code=64, scale=P, ld_scale=2, form=0):
    return C.byref(B.Act8View(code, ld_code, scale, ld_scale, form))


BAD_ACT8 = [dict(code=None), dict(scale=None), dict(ld_code=63), dict(ld_scale=1), dict(form=2), dict(form=-1)]


def forward(lib, **kw):
    a = dict(M=4, N=64, x=P, ldx=64, xt=1, gamma=P, beta=P, eps=1e-5, relu=0, y=P, ldy=64, yt=1, mean=P, rstd=P, keep=None)
    a.update(kw)
    return lib.im_layer_norm_forward(a["M"], a["N"], a["x"], a["ldx"], a["xt"], a["gamma"], a["beta"], a["eps"], a["relu"], a["y"], a["ldy"], a["yt"],
                                     a["mean"], a["rstd"], a["keep"], None)


@pytest.mark.parametrize("kw", [dict(M=0), dict(M=-1), dict(N=0), dict(x=None), dict(y=None), dict(ldx=63), dict(ldy=63), dict(xt=2), dict(yt=-1), dict(eps=0.0),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=P + 1), dict(y=P + 2, yt=0)]
                         + [dict(keep=act8(**b)) for b in BAD_ACT8])
def test_forward_refuses(lib, kw):
    assert forward(lib, **kw) == -1


def backward(lib, **kw):
    a = dict(M=4, N=64, dy=P, ld_dy=64, dyt=1, x=P, ldx=64, xt=1, mean=P, rstd=P, kept=None, gamma=P, beta=P, relu=1, dx=P, ld_dx=64, dgamma=P, dbeta=P,
             ws=P, nws=1 << 20)
    a.update(kw)
    return lib.im_layer_norm_backward(a["M"], a["N"], a["dy"], a["ld_dy"], a["dyt"], a["x"], a["ldx"], a["xt"], a["mean"], a["rstd"], a["kept"], a["gamma"],
                                      a["beta"], a["relu"], a["dx"], a["ld_dx"], a["dgamma"], a["dbeta"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("kw", [dict(M=0), dict(N=-3), dict(dy=None), dict(rstd=None), dict(mean=None), dict(x=None), dict(kept=act8()), dict(ld_dy=63),
                                dict(ldx=63), dict(ld_dx=63), dict(xt=2), dict(dyt=7), dict(dx=None, dgamma=None, dbeta=None), dict(ws=None), dict(nws=100),
                                dict(ws=P + 8), dict(dy=P + 1), dict(dx=P + 1)] + [dict(x=None, kept=act8(**b)) for b in BAD_ACT8])
def test_backward_refuses(lib, kw):
    assert backward(lib, **kw) == -1


@pytest.mark.parametrize("kw", [dict(M=0), dict(N=0), dict(x=None), dict(ld=63), dict(dt=2), dict(x=P + 1)] + [dict(a=act8(**b)) for b in BAD_ACT8] + [dict(a=None)])
def test_pack_and_unpack_refuse(lib, kw):
    a = dict(M=4, N=64, x=P, ld=64, dt=1, a=act8())
    a.update(kw)
    assert lib.im_act8_pack(a["M"], a["N"], a["x"], a["ld"], a["dt"], a["a"], None) == -1
    assert lib.im_act8_unpack(a["M"], a["N"], a["a"], None, None, 0, a["x"], a["ld"], a["dt"], None) == -1


@pytest.mark.parametrize("kw", [dict(A=None), dict(Cp=None), dict(status=None), dict(R=0), dict(Mo=0), dict(No=0), dict(lda=60), dict(lda=65), dict(ldc=63),
                                dict(A=P + 8), dict(Cp=P + 2), dict(H=None), dict(H=act8(ld_code=72)), dict(H=act8(code=P + 8)), dict(R=100000, ws=None),
                                dict(R=100000, nws=64), dict(R=100000, ws=P + 8)] + [dict(H=act8(**b)) for b in BAD_ACT8])
def test_product_refuses(lib, kw):
    a = dict(A=P, lda=64, H=act8(), Cp=P, ldc=64, R=64, Mo=64, No=64, ws=P, nws=1 << 30, status=P)
    a.update(kw)
    assert lib.im_gemm_act8_tn(a["A"], a["lda"], a["H"], a["Cp"], a["ldc"], a["R"], a["Mo"], a["No"], None, None, 0, a["ws"], a["nws"], a["status"], None) == -1


def test_too_wide_is_unsupported(lib):
    wide = dict(N=8193, ldx=8200)
    assert forward(lib, ldy=8200, **wide) == -6
    assert backward(lib, ld_dy=8200, ld_dx=8200, nws=1 << 30, **wide) == -6
    h = act8(ld_code=70000 // 16 * 16 + 16, ld_scale=4000)
    assert lib.im_gemm_act8_tn(P, 64, h, P, 70000, 64, 64, 70000, None, None, 0, P, 1 << 40, P, None) == -6


def test_workspace_sizes(lib):
    assert lib.im_layer_norm_workspace_bytes(0, 5) == 0 and lib.im_layer_norm_workspace_bytes(3, 100) == 3 * 2 * 100 * 4
    assert lib.im_layer_norm_workspace_bytes(10 ** 6, 1024) == 592 * 2 * 1024 * 4
    assert lib.im_gemm_act8_tn_workspace_bytes(64, 64, 64) == 0                      # one k-block: one part per tile
    sizes = [lib.im_gemm_act8_tn_workspace_bytes(r, 512, 1024) for r in (64, 1000, 10000, 100000, 10 ** 6)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2] == (80 + 8) * 256 * 256 * 4      # 80 pairs, 8 tiles
    assert lib.im_gemm_act8_tn_workspace_bytes(-1, 1, 1) == 0


def test_form_names():
    assert B.ACT8_FORMS == {"int8": 0, "e4m3": 1}
