"""Checkpoints of the widest rows: columns up to 2^31 - 1."""
import pytest

from tests import norm_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [2 ** 31 - 1, 2 ** 31 - 200])
@pytest.mark.parametrize("shift", [0, 1])                 # rows that start on 16 bytes, and anywhere
def test_widest_rows(cols, shift):
    import torch
    from paper_2609_09821_b200 import binding as B
    blocks = -(-cols // 32)
    base = torch.empty(cols + 8, device="cuda", dtype=torch.bfloat16)
    x = base[shift:shift + cols].view(1, cols)
    g = torch.Generator("cuda").manual_seed(cols)
    noise = torch.randn(2 ** 20 + 7, device="cuda", generator=g).bfloat16()       # a length that shares no factor with a block's
    for c in range(0, cols, noise.numel()):
        x[0, c:c + noise.numel()] = noise[:cols - c]
    code, scale = torch.full((1, cols + 5), 77, dtype=torch.uint8, device="cuda"), torch.full((1, blocks + 5), 77, dtype=torch.uint8, device="cuda")
    ck = B.Act8(code, scale, cols)
    B.act8_pack(x, ck)
    # where values are wanted for comparison: the ends, and either side of 2^30 columns
    windows = [(0, 4096), (2 ** 30 - 4096, 2 ** 30 + 4096), (cols // 32 * 32 - 8192, cols)]
    kept = [x[:, a:b].clone() for a, b in windows]
    base.fill_(3.0)
    B.act8_unpack(ck, x)
    for (a, b), was in zip(windows, kept):
        assert torch.equal(x[:, a:b].double(), ref.kept(was, ref.INT8))
    assert bool((code[0, cols:] == 77).all()) and bool((scale[0, blocks:] == 77).all()) and bool((base[:shift] == 3).all()) and bool((base[shift + cols:] == 3).all())
    # every column in between was written: each block of the repeated noise restores to the block's own values
    for c in range(0, cols - 2 ** 24, 2 ** 24 * 7):
        want = ref.kept(noise.repeat(17)[c % noise.numel():][:2 ** 20].view(1, -1), ref.INT8)
        assert torch.equal(x[:, c:c + 2 ** 20].double(), want)


def test_product_of_rows_far_apart():
    # strides beyond 2^31 are addressed in 64 bits; what a tensor map cannot express is refused
    import ctypes
    import torch
    from paper_2609_09821_b200 import binding as B
    R, Mo, No, far = 3, 40, 200, 2 ** 31 + 32
    rand = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    A = torch.empty(R, far, device="cuda", dtype=torch.bfloat16)[:, :Mo]
    code = torch.empty(R, far, device="cuda", dtype=torch.uint8)[:, :No]
    scale = torch.empty(R, far + 1, device="cuda", dtype=torch.uint8)[:, 1:8]
    A.copy_(rand(R, Mo))
    ck = B.Act8(code, scale, No)
    B.act8_pack(rand(R, No), ck)
    H = torch.empty(R, No, device="cuda")
    B.act8_unpack(ck, H)
    C, status = torch.empty(Mo, No, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.gemm_act8_tn_workspace(R, Mo, No)
    B.gemm_act8_tn(A, ck, C, ws, status)
    want = A.double().T @ H.double()
    # products are exact, three of them are added: two roundings or truncations, each a step (2 U) of the sum of magnitudes at most
    assert bool(((C.double() - want).abs() <= 4 * ref.U * (A.double().abs().T @ H.double().abs())).all()) and int(status) == 0
    call = lambda lda, ld_code: B.load().im_gemm_act8_tn(A.data_ptr(), lda, ctypes.byref(B.Act8View(code.data_ptr(), ld_code, scale.data_ptr(), far + 1, 0)),  # noqa: E731
                                                         C.data_ptr(), No, 1, Mo, No, None, None, 0, None, 0, status.data_ptr(), None)
    assert call(2 ** 39, far) == -6 and call(far, 2 ** 40) == -6
    assert call(2 ** 39 - 8, far) == 0 and call(far, 2 ** 40 - 16) == 0
    torch.cuda.synchronize()
    assert int(status) == 0
