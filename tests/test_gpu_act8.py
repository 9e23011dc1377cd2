"""Activations in 8 bits: codes, scales and restored values against 64 bits, exactly; the weight gradient from them."""
import pytest

from tests import norm_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _torch():
    global torch, B
    import torch
    from paper_2609_09821_b200 import binding as B


def values(rows, cols, seed, spread=True):
    """Normal values; with `spread` each row at its own magnitude between 2^-140 and 2^120."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    if spread:
        e = torch.randint(-140, 121, (rows, 1), device="cuda", generator=g)
        x = torch.ldexp(x.double(), e).float()
    return x


def restored(ck, dtype, **kw):
    out = torch.empty(ck.rows, ck.cols, device="cuda", dtype=dtype)
    B.act8_unpack(ck, out, **kw)
    return out


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 31), (300, 32), (2, 33), (64, 64), (77, 100), (1000, 128), (9, 361), (515, 1024), (3, 5000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_round_trip(form, rows, cols, dtype):
    dt = getattr(torch, dtype)
    x = values(rows, cols, rows + cols).to(dt)
    ck = B.Act8.empty(rows, cols, form)
    ck.code.fill_(99)
    B.act8_pack(x, ck)
    want = ref.kept(x, form)
    assert torch.equal(restored(ck, torch.float32).double(), want)
    assert torch.equal(restored(ck, torch.bfloat16).double(), want)       # a code times a power of two is exact in bf16
    e, _ = ref.exponents(x, form)
    assert torch.equal(ck.scale[:, :e.shape[1]].int(), (e + 127).int())
    assert bool((ck.code[:, cols:] == 99).all())
    half = 0.5 * torch.exp2(e.double()).repeat_interleave(32, 1)[:, :cols] if form == ref.INT8 else None
    if half is not None:                                                    # half a step of the block's grid, by definition
        assert bool(((want - x.double()).abs() <= half).all())


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
def test_rows_that_start_anywhere(form):
    rows, cols = 67, 150
    x0 = torch.zeros(rows * 160 + 8, device="cuda")
    x = x0[3:3 + rows * 155].view(rows, 155)[:, :cols]
    x.copy_(values(rows, cols, 5))
    code = torch.full((rows, 163), 55, dtype=torch.uint8, device="cuda")[:, 1:]
    scale = torch.full((rows, 9), 55, dtype=torch.uint8, device="cuda")[:, 2:]
    ck = B.Act8(code, scale, cols, form)
    B.act8_pack(x, ck)
    want = ref.kept(x, form)
    out = torch.full((rows, 157), 7.0, device="cuda")
    B.act8_unpack(ck, out[:, 4:4 + cols])
    assert torch.equal(out[:, 4:4 + cols].double(), want) and bool((out[:, :4] == 7).all()) and bool((out[:, 154:] == 7).all())
    assert bool((code[:, cols:] == 55).all()) and bool((scale[:, 5:] == 55).all())


@pytest.mark.parametrize("form,top", [(ref.INT8, 127.0), (ref.E4M3, 448.0)])
def test_borders_of_the_scale(form, top):
    # the largest magnitude just on, below and above top 2^e, ties at half a step, zeros, the least and the largest numbers
    x = torch.zeros(10, 32, device="cuda")
    for i, k in enumerate((-20, 0, 1, 60)):
        x[i, 0] = top * 2.0 ** k
    x[4, 3] = torch.nextafter(torch.tensor(top), torch.tensor(1e9))
    x[5, 3] = -torch.nextafter(torch.tensor(top), torch.tensor(0.0))
    x[6, :] = torch.arange(32, device="cuda") + 0.5
    x[6, 31] = top
    x[7, 1] = 3.4028234663852886e38
    x[8, 1], x[8, 2] = 1e-45, 2.0 ** -101 * 1.5
    x[:7, 9] = -0.0
    ck = B.Act8.empty(10, 32, form)
    B.act8_pack(x, ck)
    want = ref.kept(x, form)
    assert float(want[7, 1]) == 2.0 ** 128           # the largest fp32 number rounds up to a code times a power of two that fp32 does not hold
    assert torch.equal(restored(ck, torch.float32), want.float())
    assert int(ck.scale[9, 0]) == 27 and bool((ck.code[9] == 0).all())


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_blocks_that_are_not_finite(form, bad):
    x = values(4, 100, 2, spread=False)
    x[1, 40] = bad
    x[3, 99] = bad
    ck = B.Act8.empty(4, 100, form)
    B.act8_pack(x, ck)
    out, want = restored(ck, torch.float32), ref.kept(x, form)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out.double().nan_to_num(7.0), want.nan_to_num(7.0))
    assert ck.scale[1].tolist()[1] == 255 and ck.scale[3].tolist()[3] == 255 and bool((ck.code[1, 32:64] == 0).all())
    relu = restored(ck, torch.bfloat16, relu=True)
    assert torch.equal(torch.isnan(relu), torch.isnan(want))


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("cols", [40, 361, 1024])
def test_restored_under_gamma_beta_and_relu(form, cols):
    rows = 130
    x = values(rows, cols, 9, spread=False)
    g = torch.Generator("cuda").manual_seed(1)
    gamma, beta = torch.randn(cols, device="cuda", generator=g), torch.randn(cols, device="cuda", generator=g)
    ck = B.Act8.empty(rows, cols, form)
    B.act8_pack(x, ck)
    v = ref.kept(x, form)
    for ga, be, relu in ((gamma, beta, True), (gamma, None, False), (None, beta, True), (None, None, True)):
        want = ref.affine(v, ga, be).float()          # gamma times a code is exact in 64 bits, the sum is rounded once
        want = torch.relu(want) if relu else want
        assert torch.equal(restored(ck, torch.float32, gamma=ga, beta=be, relu=relu), want)
        assert torch.equal(restored(ck, torch.bfloat16, gamma=ga, beta=be, relu=relu), want.bfloat16())


# ---------------------------------------------------------------------------------------------- products
def product(R, Mo, No, form, affine, seed=0, pad_a=0, pad_c=0):
    g = torch.Generator("cuda").manual_seed(seed)
    ld = (Mo + 7) // 8 * 8 + pad_a
    A = torch.randn(R, ld, device="cuda", generator=g).bfloat16()[:, :Mo]
    ck = B.Act8.empty(R, No, form)
    ck.code.random_(0, 127, generator=g)                                  # (the padding too: it must not matter)
    B.act8_pack(torch.randn(R, No, device="cuda", generator=g), ck)
    gamma, beta, relu = (torch.randn(No, device="cuda", generator=g), torch.randn(No, device="cuda", generator=g), True) if affine else (None, None, False)
    C = torch.full((Mo, No + pad_c), 5.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.gemm_act8_tn_workspace(R, Mo, No)
    ws.fill_(255)
    B.gemm_act8_tn(A, ck, C[:, :No], ws, status, gamma=gamma, beta=beta, relu=relu)
    return A, ck, gamma, beta, relu, C, status


def check_product(A, ck, gamma, beta, relu, C, status):
    No = ck.cols
    H = torch.empty(ck.rows, No, device="cuda", dtype=torch.bfloat16)
    B.act8_unpack(ck, H, gamma=gamma, beta=beta, relu=relu)
    want = A.double().T @ H.double()
    # products of two bf16 are exact; tensor memory adds sixteen rows at a time over at most 2048 rows (each step off by a step
    # of the running sum at most, 2 U), such chains are added in fp32, at most one for each of them and one for each of 160 parts
    bound = (128 + ck.rows / 2048 + 160) * 2 * ref.U * (A.double().abs().T @ H.double().abs())
    assert bool(((C[:, :No].double() - want).abs() <= bound).all())
    assert bool((C[:, No:] == 5.0).all()) and int(status) == 0
    # and far inside that for sums of random signs
    assert float((C[:, :No].double() - want).norm() / want.norm().clamp(min=1e-300)) <= 1e-5


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("R", [1, 15, 64, 65, 1000, 4133])
@pytest.mark.parametrize("Mo,No", [(1, 1), (28, 361), (64, 128), (69, 512), (129, 130), (256, 16), (300, 1000)])
def test_product_sizes(form, affine, R, Mo, No):
    check_product(*product(R, Mo, No, form, affine, seed=R + Mo, pad_a=8, pad_c=3))


@pytest.mark.parametrize("R,Mo,No", [(16000, 512, 1024), (70001, 1024, 1024), (40000, 69, 577), (300, 2048, 2048), (100, 4500, 5000), (131072, 28, 64)])
def test_product_large(R, Mo, No):
    check_product(*product(R, Mo, No, ref.INT8, True, seed=R))


def test_product_carries_nan_to_its_columns():
    R, Mo, No = 200, 64, 96
    g = torch.Generator("cuda").manual_seed(0)
    A = torch.randn(R, Mo, device="cuda", generator=g).bfloat16()
    x = torch.randn(R, No, device="cuda", generator=g)
    x[150, 40] = float("nan")
    ck = B.Act8.empty(R, No)
    B.act8_pack(x, ck)
    C, status = torch.empty(Mo, No, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for relu in (False, True):
        B.gemm_act8_tn(A, ck, C, B.gemm_act8_tn_workspace(R, Mo, No), status, relu=relu)
        assert bool(torch.isnan(C[:, 32:64]).all()) and bool(torch.isfinite(C[:, :32]).all()) and bool(torch.isfinite(C[:, 64:]).all())


def test_product_repeats_on_other_streams_and_in_graphs():
    R, Mo, No = 9001, 320, 512
    A, ck, gamma, beta, relu, C, status = product(R, Mo, No, ref.INT8, True, seed=3)
    outs, side = [torch.zeros(Mo, No, device="cuda") for _ in range(3)], [torch.cuda.Stream() for _ in range(2)]
    wss = [B.gemm_act8_tn_workspace(R, Mo, No) for _ in range(3)]
    torch.cuda.synchronize()
    for o, w, s in zip(outs, wss, side):
        with torch.cuda.stream(s):
            B.gemm_act8_tn(A, ck, o, w, status, gamma=gamma, beta=beta, relu=relu)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gemm_act8_tn(A, ck, outs[2], wss[2], status, gamma=gamma, beta=beta, relu=relu)
    outs[2].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(C, o) for o in outs) and int(status) == 0


@pytest.mark.parametrize("R,Mo,No,form", [(65536, 69, 512, ref.E4M3), (65536, 28, 512, ref.INT8), (16000, 512, 1024, ref.INT8)])
def test_product_many_in_a_row(R, Mo, No, form):
    # copies complete in another order each time; every launch gives the same bits
    sets = [product(R, Mo, No, form, False, seed=s) for s in (1, 2, 3)]
    wss = [B.gemm_act8_tn_workspace(R, Mo, No) for _ in sets]
    outs = [torch.zeros(Mo, No, device="cuda") for _ in sets]
    for i in range(600):
        A, ck, _, _, _, C, status = sets[i % 3]
        B.gemm_act8_tn(A, ck, outs[i % 3], wss[i % 3], status)
        if i % 60 >= 57:
            torch.cuda.synchronize()
            assert torch.equal(outs[i % 3], C)
            outs[i % 3].zero_()
    assert all(int(s[-1]) == 0 for s in sets)


def test_product_reports_a_wait_that_runs_out():
    R, Mo, No = 300, 64, 128
    A, ck, gamma, beta, relu, C, status = product(R, Mo, No, ref.INT8, False)
    ws = B.gemm_act8_tn_workspace(R, Mo, No)
    B.debug_set_wait(limit_ns=2_000_000, skip_loads=True)
    try:
        B.gemm_act8_tn(A, ck, torch.empty(Mo, No, device="cuda"), ws, status)
        torch.cuda.synchronize()
        assert int(status) == 2                                            # IM_DEV_WAIT_TIMEOUT
    finally:
        B.debug_set_wait()
    status.zero_()
    C2 = torch.empty(Mo, No, device="cuda")
    B.gemm_act8_tn(A, ck, C2, ws, status)
    assert torch.equal(C2, C[:, :No]) and int(status) == 0


def test_beyond_32_bits_of_elements():
    rows, cols, Mo = 2 ** 20 + 3, 4096 + 16, 64
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-1] = (torch.arange(cols, device="cuda") % 127).bfloat16()
    ck = B.Act8.empty(rows, cols)
    B.act8_pack(x, ck)
    want = ref.kept(x[-1:], ref.INT8)
    assert int(torch.count_nonzero(ck.code[:-1])) == 0
    x.fill_(1.0)
    B.act8_unpack(ck, x)
    assert torch.equal(x[-1:].double(), want) and bool((x[:-1].view(torch.int16) == 0).all())
    A = torch.zeros(rows, Mo, device="cuda", dtype=torch.bfloat16)
    A[-1] = torch.randn(Mo, device="cuda").bfloat16()
    C, status = torch.empty(Mo, cols, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.gemm_act8_tn(A, ck, C, B.gemm_act8_tn_workspace(rows, Mo, cols), status)
    assert torch.equal(C.double(), A[-1].double()[:, None] * want) and int(status) == 0      # one product a sum: exact
