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
