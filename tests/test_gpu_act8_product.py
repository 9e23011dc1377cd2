"""The weight gradient from 8 bits against 64 bits: sums over several chains on every tile width, leftover workers, every combination of
gamma, beta and ReLU, and scales at any address."""
import pytest

from tests import norm_reference as ref

pytestmark = pytest.mark.gpu

CHAIN_ROWS = 20 * 64                    # rows that tensor memory sums up before they are added in fp32
MAX_PARTS = 160                         # of a tile


@pytest.fixture(autouse=True)
def _torch():
    global torch, B
    import torch
    from paper_2609_09821_b200 import binding as B


def check(R, Mo, No, form, gamma=False, beta=False, relu=False, scale=None):
    """One product of dense normal data; scale(rows, blocks): where the scales lie."""
    g = torch.Generator("cuda").manual_seed(R + 7 * Mo + No)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    A = rand(R, (Mo + 7) // 8 * 8).bfloat16()[:, :Mo]
    ck = B.Act8.empty(R, No, form)
    if scale is not None:
        ck = B.Act8(ck.code, scale(R, -(-No // 32)), No, form)
    B.act8_pack(rand(R, No), ck)
    ga, be = rand(No) if gamma else None, rand(No) if beta else None
    C, status = torch.full((Mo, No), 5.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.gemm_act8_tn_workspace(R, Mo, No)
    ws.fill_(255)
    B.gemm_act8_tn(A, ck, C, ws, status, gamma=ga, beta=be, relu=relu)
    H = torch.empty(R, No, device="cuda", dtype=torch.bfloat16)
    B.act8_unpack(ck, H, gamma=ga, beta=be, relu=relu)
    assert int(status) == 0
    want, size = torch.zeros(Mo, No, device="cuda", dtype=torch.float64), torch.zeros(Mo, No, device="cuda", dtype=torch.float64)
    for r in range(0, R, 65536):
        a, h = A[r:r + 65536].double(), H[r:r + 65536].double()
        want += a.T @ h
        size += a.abs().T @ h.abs()
    # Products of two bf16 are exact.  Tensor memory adds sixteen rows at a time, each step off by a step (2 U) of the running sum at most,
    # CHAIN_ROWS / 16 steps to a chain; then one fp32 rounding for each chain and one for each part.
    bound = (CHAIN_ROWS / 16 + R / CHAIN_ROWS + 1 + MAX_PARTS) * 2 * ref.U * size
    assert bool(((C.double() - want).abs() <= bound).all())
    assert float((C.double() - want).norm() / want.norm()) <= 1e-5            # and far inside that for sums of random signs


# 64, 128 columns of A a tile and pairs; 148 SMs give 28 to 290 k-blocks a part: two chains and more, and with 9 tiles workers are left over
@pytest.mark.parametrize("R,Mo,No,form", [(65536, 28, 512, ref.INT8), (65536, 64, 512, ref.E4M3), (300000, 64, 1100, ref.INT8), (300000, 60, 1100, ref.E4M3),
                                          (200000, 100, 1100, ref.INT8), (131072, 65, 64, ref.E4M3), (100000, 300, 700, ref.INT8)])
def test_sums_of_several_chains(R, Mo, No, form):
    check(R, Mo, No, form)


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("gamma,beta,relu", [(1, 1, 0), (1, 0, 0), (0, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 1)])
@pytest.mark.parametrize("R,Mo,No", [(1000, 28, 361), (1500, 69, 200), (1201, 300, 700), (7001, 140, 130)])
def test_every_form_of_the_restored_operand(form, gamma, beta, relu, R, Mo, No):
    check(R, Mo, No, form, gamma=bool(gamma), beta=bool(beta), relu=bool(relu))


@pytest.mark.parametrize("R,Mo,No", [(1000, 28, 361), (1500, 69, 1000), (1201, 300, 700)])
@pytest.mark.parametrize("off,extra", [(0, 1), (1, 3), (2, 2), (3, 6)])             # of the first scale, and of a row's bytes behind the last
def test_scales_at_any_address(R, Mo, No, off, extra):
    def scale(rows, blocks):
        return torch.full((rows, off + blocks + extra), 77, dtype=torch.uint8, device="cuda")[:, off:]
    check(R, Mo, No, ref.INT8, gamma=True, beta=True, relu=True, scale=scale)
    check(R, Mo, No, ref.E4M3, scale=scale)


@pytest.mark.parametrize("R,Mo,No", [(300, 40, 200), (300, 100, 200), (300, 200, 200)])
def test_a_marked_block_under_gamma_and_beta(R, Mo, No):
    g = torch.Generator("cuda").manual_seed(R)
    A = torch.randn(R, (Mo + 7) // 8 * 8, device="cuda", generator=g).bfloat16()[:, :Mo]        # (strides of A are multiples of 8)
    x = torch.randn(R, No, device="cuda", generator=g)
    x[R - 1, 70] = float("inf")
    ck = B.Act8.empty(R, No)
    B.act8_pack(x, ck)
    ga, be = torch.randn(2, No, device="cuda", generator=g)
    C, status, ws = torch.empty(Mo, No, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), B.gemm_act8_tn_workspace(R, Mo, No)
    for kw in (dict(gamma=ga), dict(beta=be), dict(gamma=ga, beta=be), dict(gamma=ga, beta=be, relu=True)):
        B.gemm_act8_tn(A, ck, C, ws, status, **kw)
        assert bool(torch.isnan(C[:, 64:96]).all()) and bool(torch.isfinite(C[:, :64]).all()) and bool(torch.isfinite(C[:, 96:]).all()), kw
