"""Layer norm, forward and backward, against 64 bits: widths on both sides of every variant, rows that start anywhere, all type
pairs, the 8-bit checkpoint beside it, rows without spread, values that are not finite, other streams and captured graphs."""
import pytest

from tests import norm_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5
SENTINEL = 7.0


@pytest.fixture(autouse=True)
def _torch():
    global torch, B
    import torch
    from paper_2609_09821_b200 import binding as B


def matrix(rows, cols, dtype, pad, shift, g=None, fill=None):
    """[rows, cols] view with row stride cols + pad, `shift` elements into its storage; returns (view, storage)."""
    st = torch.full((rows * (cols + pad) + shift + 16,), SENTINEL, device="cuda", dtype=dtype)
    v = st[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if g is not None:
        v.copy_(torch.randn(rows, cols, device="cuda", generator=g) * 1.5 + 0.25)
    elif fill is not None:
        v.fill_(fill)
    return v, st


def untouched(view, storage):
    """Everything outside the view still holds the sentinel."""
    mask = torch.ones_like(storage, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((storage[mask] == SENTINEL).all())


def check_forward(x, gamma, beta, y, mean, rstd, relu):
    rmean, rrstd, xh, ry = ref.forward(x, gamma, beta, EPS, relu)
    big = x.double().abs().amax(1)
    # mean: 32 terms in a row and 5 + 8 levels, then a division; what it is off enters x - mean whole; the variance's sum the same way
    # again, halved by the root
    assert bool(((mean.double() - rmean).abs() <= 50 * ref.U * big).all())
    off = 50 * ref.U * big * rrstd
    assert bool(((rstd.double() - rrstd).abs() <= rrstd * (32 * ref.U + off * off + 2 * ref.U * off)).all())
    ga = torch.ones_like(xh) if gamma is None else gamma.double().abs()
    tol = ga * (xh.abs() * (36 * ref.U + off[:, None] ** 2) + off[:, None]) + 3 * ref.U * (ry.abs() + (0 if beta is None else beta.double().abs()))
    tol = tol + (ry.abs() + tol) * ref.HALF[y.dtype]
    assert bool(((y.double() - ry).abs() <= tol).all()), float(((y.double() - ry).abs() / tol.clamp(min=1e-300)).max())


WIDTHS = [1, 2, 8, 31, 33, 64, 65, 128, 136, 256, 257, 361, 512, 577, 1000, 1024, 1032, 2048, 2056, 4096, 5001, 8192]


@pytest.mark.parametrize("N", WIDTHS)
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("bfloat16", "float32")])
def test_forward_every_width(N, src, dst):
    g = torch.Generator("cuda").manual_seed(N)
    gamma, beta = torch.randn(N, device="cuda", generator=g), torch.randn(N, device="cuda", generator=g)
    for M, pad, shift in ((1, 0, 0), (37, 8 - N % 8, 0), (301, 3, 1)):
        x, _ = matrix(M, N, getattr(torch, src), pad, shift, g)
        y, sy = matrix(M, N, getattr(torch, dst), pad, shift)
        mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        for relu, ga, be in ((False, gamma, beta), (True, gamma, None), (True, None, beta)):
            B.layer_norm(x, ga, be, y, mean, rstd, eps=EPS, relu=relu)
            check_forward(x, ga, be, y, mean, rstd, relu)
            assert untouched(y, sy)


@pytest.mark.parametrize("form", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("N,pad,shift", [(31, 0, 0), (64, 0, 0), (72, 8, 0), (128, 0, 0), (361, 7, 0), (361, 0, 1), (1000, 24, 0), (1024, 0, 0), (2048, 0, 0), (2051, 0, 0), (5000, 0, 0)])
def test_forward_keeps_the_normalised_rows(form, N, pad, shift):
    M = 70
    g = torch.Generator("cuda").manual_seed(N)
    x, _ = matrix(M, N, torch.float32, pad, shift, g)
    y, _ = matrix(M, N, torch.float32, pad, shift)
    ck = B.Act8.empty(M, N, form)
    ck.code.fill_(77), ck.scale.fill_(77)
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.layer_norm(x, None, None, y, mean, rstd, eps=EPS, ckpt=ck)
    # with neither gamma nor beta y is xh, and the checkpoint is the 8-bit form of just that
    out = torch.empty(M, N, device="cuda")
    B.act8_unpack(ck, out)
    assert torch.equal(out.double(), ref.kept(y, form))
    assert bool((ck.code[:, N:] == 77).all())


@pytest.mark.parametrize("N", [28, 64, 128, 200, 361, 512, 1000, 1024, 2048, 2500, 4096, 8192])
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("form", [None, ref.INT8, ref.E4M3])
def test_backward_every_width(N, src, dst, form):
    g = torch.Generator("cuda").manual_seed(N + 1)
    gamma, beta = torch.randn(N, device="cuda", generator=g), torch.randn(N, device="cuda", generator=g)
    for M, pad, shift in ((1, 0, 0), (45, 8 - N % 8, 0), (1203, 0, 0), (130, 3, 1)):
        x, _ = matrix(M, N, getattr(torch, src), pad, shift, g)
        dy, _ = matrix(M, N, getattr(torch, dst), pad, shift, g)
        dx, sdx = matrix(M, N, getattr(torch, src), pad, shift)
        mean, rstd, _, _ = ref.forward(x, None, None, EPS, False)
        mean, rstd = mean.float(), rstd.float()
        xh32 = (x.float() - mean[:, None]) * rstd[:, None]
        xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        ck = None
        if form is not None:
            ck = B.Act8.empty(M, N, form)
            B.act8_pack(xh32, ck)
            xh = xh32 = ref.kept(xh32, form)
        dgamma, dbeta = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        ws = B.layer_norm_workspace(M, N)
        for relu, ga, be in ((False, gamma, None), (True, gamma, beta), (True, None, None)):
            ws.fill_(255)
            B.layer_norm_backward(dy, ga, be, rstd, dx, dgamma, dbeta, ws, relu=relu, **(dict(ckpt=ck) if ck else dict(x=x, mean=mean)))
            passed = ref.affine(xh32.double(), ga, be) > 0
            rdx, rg, rb, err, ag, ab = ref.backward(dy, xh, passed, rstd, ga, relu)
            tol = err + (rdx.abs() + err) * ref.HALF[dx.dtype]
            assert bool(((dx.double() - rdx).abs() <= tol).all()), (M, relu, float(((dx.double() - rdx).abs() / tol.clamp(min=1e-300)).max()))
            chain = 2 + 32 + M / 148 + 4             # a thread's rows, the row groups of a CTA, the products; the rest is fp64
            assert bool(((dgamma.double() - rg).abs() <= chain * ref.U * ag + 2 * ref.U * rg.abs()).all())
            assert bool(((dbeta.double() - rb).abs() <= chain * ref.U * ab + 2 * ref.U * rb.abs()).all())
            assert untouched(dx, sdx)


def test_backward_against_differences_of_the_forward():
    M, N = 6, 40
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(M, N, device="cuda", generator=g)
    w = torch.randn(M, N, device="cuda", generator=g)
    gamma, beta = 1 + 0.3 * torch.randn(N, device="cuda", generator=g), 0.3 * torch.randn(N, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    B.layer_norm(x, gamma, beta, y, mean, rstd, eps=EPS, relu=True)
    B.layer_norm_backward(w, gamma, beta, rstd, dx, dg, db, B.layer_norm_workspace(M, N), relu=True, x=x, mean=mean)
    loss = lambda x_, g_, b_: float((ref.forward(x_, g_, b_, EPS, True)[3] * w.double()).sum())  # noqa: E731
    h = 1e-6
    for grad, at in ((dx, 0), (dg, 1), (db, 2)):
        args = [x.double(), gamma.double(), beta.double()]
        d = torch.randn(args[at].shape, device="cuda", generator=g, dtype=torch.float64)
        plus, minus = list(args), list(args)
        plus[at], minus[at] = args[at] + h * d, args[at] - h * d
        want = (loss(*plus) - loss(*minus)) / (2 * h)
        # the difference is off by h^2 terms and 1e-16 / h; the gradient by a few fp32 roundings of its own size (and no kink
        # lies within h of these inputs' pre-activations, 240 values of unit size)
        assert abs(float((grad.double() * d).sum()) - want) <= 2e-6 * (1 + float((grad.double().abs() * d.abs()).sum()))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_backward_pass_opens_the_elements_that_the_forward_left_positive(dtype):
    # one row: dbeta is dy where y > 0; half of the pre-activations lie within a few roundings of 0
    N = 4096
    g = torch.Generator("cuda").manual_seed(11)
    for _ in range(20):
        x = torch.randn(1, N, device="cuda", generator=g).to(getattr(torch, dtype))
        gamma, beta = torch.rand(N, device="cuda", generator=g) + 0.5, torch.randn(N, device="cuda", generator=g)
        xh, mean, rstd = torch.empty(1, N, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        B.layer_norm(x, None, None, xh, mean, rstd)
        beta[::2] = -(gamma * xh[0])[::2]
        y, db, dy = torch.empty(1, N, device="cuda"), torch.empty(N, device="cuda"), torch.randn(1, N, device="cuda", generator=g)
        B.layer_norm(x, gamma, beta, y, relu=True)
        B.layer_norm_backward(dy, gamma, beta, rstd, None, None, db, B.layer_norm_workspace(1, N), relu=True, x=x, mean=mean)
        assert torch.equal(db, torch.where(y[0] > 0, dy[0], torch.zeros(N, device="cuda")))


def test_outputs_may_be_left_out_and_lie_on_inputs():
    M, N = 133, 1024
    g = torch.Generator("cuda").manual_seed(8)
    x, dy = torch.randn(M, N, device="cuda", generator=g), torch.randn(M, N, device="cuda", generator=g)
    gamma = torch.rand(N, device="cuda", generator=g) + 0.5
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.layer_norm(x, gamma, None, y, mean, rstd)
    for where in ("x", "dy"):
        dx, dg, db = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        ws = B.layer_norm_workspace(M, N)
        B.layer_norm_backward(dy, gamma, None, rstd, dx, dg, db, ws, x=x, mean=mean)
        x2, dy2, db2 = x.clone(), dy.clone(), torch.empty_like(db)
        B.layer_norm_backward(dy2, gamma, None, rstd, x2 if where == "x" else dy2, None, db2, ws, x=x2, mean=mean)
        assert torch.equal(dx, x2 if where == "x" else dy2) and torch.equal(db, db2)
        dg2 = torch.empty_like(dg)
        B.layer_norm_backward(dy, gamma, None, rstd, None, dg2, None, ws, x=x, mean=mean)
        assert torch.equal(dg, dg2)
        dx2 = torch.empty_like(dx)
        B.layer_norm_backward(dy, gamma, None, rstd, dx2, None, None, None, x=x, mean=mean)
        assert torch.equal(dx, dx2)
    x2 = x.clone()
    B.layer_norm(x2, gamma, None, x2)
    assert torch.equal(x2, y)


def test_rows_without_spread_and_rows_that_are_not_finite():
    M, N = 9, 200
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(M, N, device="cuda", generator=g)
    x[0] = 0.0
    x[1] = 3.0                                      # 200 threes add up exactly: no spread is left, xh is 0
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    x[4] += 4096.0                                  # an offset far above the spread
    x[5] *= 1e17
    x[6] *= 1e-30                                   # var + eps is eps
    beta = torch.randn(N, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ck = B.Act8.empty(M, N)
    B.layer_norm(x, None, beta, y, mean, rstd, eps=EPS, ckpt=ck)
    assert torch.equal(y[0], beta) and torch.equal(y[1], beta)
    assert bool(torch.isnan(y[2:4]).all()) and bool(torch.isfinite(y[:2]).all()) and bool(torch.isfinite(y[4:]).all())
    rows = [0, 1, 4, 5, 6, 7, 8]
    check_forward(x[rows], None, beta, y[rows], mean[rows], rstd[rows], False)
    out = torch.empty_like(x)
    B.act8_unpack(ck, out)
    assert bool(torch.isnan(out[2:4]).all()) and bool(torch.isfinite(out[rows]).all()) and bool((out[:2] == 0).all())
    B.layer_norm(x, None, beta, y, relu=True, eps=EPS)
    assert bool(torch.isnan(y[2:4]).all()) and bool((y[rows] >= 0).all())
    # a NaN in one row of dy stays in that row of dx, and reaches its columns' sums
    dy = torch.randn(M, N, device="cuda", generator=g)
    dy[7, 5] = float("nan")
    x[2, 7] = x[3, 9] = 0.0
    B.layer_norm(x, None, beta, y, mean, rstd, eps=EPS)
    dx, dg, db = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    B.layer_norm_backward(dy, None, beta, rstd, dx, dg, db, B.layer_norm_workspace(M, N), x=x, mean=mean)
    assert bool(torch.isnan(dx[7]).all()) and bool(torch.isfinite(dx[[0, 1, 2, 3, 4, 5, 6, 8]]).all())
    assert torch.isnan(dg).nonzero().tolist() == [[5]] and torch.isnan(db).nonzero().tolist() == [[5]]


def test_results_repeat_bit_for_bit_on_other_streams_and_in_graphs():
    M, N = 3001, 512
    g = torch.Generator("cuda").manual_seed(4)
    x = torch.randn(M, N, device="cuda", generator=g).bfloat16()
    dy = torch.randn(M, N, device="cuda", generator=g).bfloat16()
    gamma, beta = torch.rand(N, device="cuda", generator=g) + 0.5, torch.randn(N, device="cuda", generator=g)

    def buffers():
        e = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
        return dict(y=e(M, N, dtype=torch.bfloat16), mean=e(M), rstd=e(M), dx=e(M, N, dtype=torch.bfloat16), dg=e(N), db=e(N),
                    ws=B.layer_norm_workspace(M, N), ck=B.Act8.empty(M, N))

    def go(b):
        B.layer_norm(x, gamma, beta, b["y"], b["mean"], b["rstd"], relu=True, ckpt=b["ck"])
        B.layer_norm_backward(dy, gamma, beta, b["rstd"], b["dx"], b["dg"], b["db"], b["ws"], relu=True, ckpt=b["ck"])

    keys = ("y", "mean", "rstd", "dx", "dg", "db")
    first = buffers()
    go(first)
    torch.cuda.synchronize()
    others, side = [buffers() for _ in range(3)], [torch.cuda.Stream() for _ in range(2)]
    for b, s in zip(others, side):                  # two at once, each with its own workspace
        with torch.cuda.stream(s):
            go(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(others[2])
    for k in keys:
        others[2][k].zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for b in others:
        assert all(torch.equal(first[k], b[k]) for k in keys) and torch.equal(first["ck"].code, b["ck"].code)


def test_many_rows_of_few_columns():
    M, N = 200003, 28
    g = torch.Generator("cuda").manual_seed(6)
    x, dy = torch.randn(M, N, device="cuda", generator=g), torch.randn(M, N, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.layer_norm(x, None, None, y, mean, rstd, eps=EPS)
    check_forward(x, None, None, y, mean, rstd, False)
    dx, dg, db = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    B.layer_norm_backward(dy, None, None, rstd, dx, dg, db, B.layer_norm_workspace(M, N), x=x, mean=mean)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    rdx, rg, rb, err, ag, ab = ref.backward(dy, xh, None, rstd, None, False)
    assert bool(((dx.double() - rdx).abs() <= err + 2 * ref.U * rdx.abs()).all())
    chain = 38 + M / 148
    assert bool(((dg.double() - rg).abs() <= chain * ref.U * ag).all()) and bool(((db.double() - rb).abs() <= chain * ref.U * ab).all())


def test_rows_beyond_32_bits_of_elements():
    # the last rows of a matrix of more than 2^32 elements (8.6 GB of bf16): wrong offsets would land elsewhere
    M, N = 2 ** 20 + 3, 4096 + 8
    x = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    x[-1] = torch.arange(N, device="cuda") % 17
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    want = x[-1:].clone()
    B.layer_norm(x, None, None, x, mean, rstd, eps=EPS)
    torch.cuda.synchronize()
    check_forward(want, None, None, x[-1:], mean[-1:], rstd[-1:], False)
    assert bool((x[:-1].view(torch.int16) == 0).all())


def test_backward_beyond_32_bits_of_elements():
    M, N = 2 ** 20 + 3, 4096 + 8
    dy = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    dy[-1] = (torch.arange(N, device="cuda") % 13).bfloat16()
    ck = B.Act8.empty(M, N)
    ck.scale.fill_(120)
    ck.code[-1, :N] = torch.arange(N, device="cuda").remainder(251).to(torch.uint8)
    rstd = torch.ones(M, device="cuda")
    dg, db = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    h = dy[-1:].double()
    xh = ck.code[-1:, :N].view(torch.int8).double() * 2.0 ** (120 - 127)
    B.layer_norm_backward(dy, None, None, rstd, dy, dg, db, B.layer_norm_workspace(M, N), ckpt=ck)
    rdx, rg, rb, err, _, _ = ref.backward(h, xh, None, rstd[-1:], None, False)
    assert torch.equal(dg.double(), (h * xh)[0]) and torch.equal(db.double(), h[0])       # one row: exact products
    assert bool(((dy[-1:].double() - rdx).abs() <= err + (rdx.abs() + err) * ref.HALF[torch.bfloat16]).all())
    assert bool((dy[:-1].view(torch.int16) == 0).all())


def test_tensors_that_do_not_fit_are_refused():
    M, N = 8, 64
    x, y, v = torch.zeros(M, N, device="cuda"), torch.zeros(M, N, device="cuda"), torch.zeros(N, device="cuda")
    ck = B.Act8.empty(M, N)
    for bad in (x.cpu(), x.half(), x.double(), x.t(), x[:, :32], x[:4], x.view(-1)):
        with pytest.raises(ValueError):
            B.layer_norm(x, v, v, bad)
        with pytest.raises(ValueError):
            B.act8_unpack(B.Act8.empty(M, N), bad)
    for bad in (v.cpu(), v.bfloat16(), v[:32], torch.zeros(2 * N, device="cuda")[::2]):
        with pytest.raises(ValueError):
            B.layer_norm(x, bad, None, y)
        with pytest.raises(ValueError):
            B.layer_norm_backward(x, bad, None, torch.ones(M, device="cuda"), y, None, None, None, x=x, mean=torch.zeros(M, device="cuda"))
    with pytest.raises(ValueError):
        B.layer_norm(x, v, v, y, ckpt=B.Act8.empty(M, 32))
    with pytest.raises(ValueError):
        B.Act8(ck.code[:, :32], ck.scale, N)
    with pytest.raises(ValueError):
        B.Act8(ck.code, ck.scale[:4], N)
    with pytest.raises(KeyError):
        B.Act8(ck.code, ck.scale, N, "int4")
    with pytest.raises(ValueError):
        B.gemm_act8_tn(x, ck, torch.empty(N, N, device="cuda"), None, torch.zeros(1, dtype=torch.int32, device="cuda"))      # A not bf16
    with pytest.raises(B.ImError):
        B.layer_norm(torch.zeros(2, 8200, device="cuda"), None, None, torch.zeros(2, 8200, device="cuda"))
    with pytest.raises(B.ImError):
        B.layer_norm(torch.zeros(0, 8, device="cuda"), None, None, torch.zeros(0, 8, device="cuda"))


@pytest.mark.parametrize("N", [64, 360, 1024, 2052])
@pytest.mark.parametrize("pad,shift", [(0, 4), (4, 0), (4, 4), (12, 8)])
def test_fp32_rows_at_half_a_sector_hold_the_same_bits(N, pad, shift):
    """fp32 rows that start at a multiple of 16 bytes but not of 32 (all of them, or every other one) are written by other
    instructions: the values are the same, and so is all around them."""
    M = 77
    g = torch.Generator(device="cuda").manual_seed(N + pad)
    x, dy = (torch.randn(M, N, device="cuda", generator=g) for _ in range(2))
    gamma, beta = (torch.randn(N, device="cuda", generator=g) for _ in range(2))
    got = []
    for p, s in ((24, 0), (pad, shift)):
        p += -(N + p) % 4                                      # (rows of a multiple of 16 bytes in both)
        y, sy = matrix(M, N, torch.float32, p, s)
        dx, sdx = matrix(M, N, torch.float32, p, s)
        back, sback = matrix(M, N, torch.float32, p, s)
        mean, rstd = torch.empty(2, M, device="cuda")
        ck = B.Act8.empty(M, N, "int8")
        dgamma, dbeta = torch.empty(2, N, device="cuda")
        B.layer_norm(x, gamma, beta, y, mean, rstd, relu=True, ckpt=ck)
        B.layer_norm_backward(dy, gamma, beta, rstd, dx, dgamma, dbeta, B.layer_norm_workspace(M, N), relu=True, x=x, mean=mean)
        B.act8_unpack(ck, back, gamma, beta, relu=True)
        for view, storage in ((y, sy), (dx, sdx), (back, sback)):
            assert untouched(view, storage)
        got.append([t.clone() for t in (y, dx, back, dgamma, dbeta)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("N", [72, 40, 264, 520, 1032, 2056, 4104, 6000])
def test_an_infinite_gradient_spoils_its_row_as_the_formula_says(N, kept):
    """One infinity among the first columns of dy: dx of its row holds the infinities and NaNs that the formula gives (threads
    behind the last column add nothing to the row's sums), dgamma and dbeta of its column are infinite, all else is finite."""
    M, row, col = 13, 3, 2
    g = torch.Generator(device="cuda").manual_seed(N)
    x, dy = (torch.randn(M, N, device="cuda", generator=g) for _ in range(2))
    gamma = torch.rand(N, device="cuda", generator=g) + 0.5
    x[row, col] = 3.0
    dy[row, col] = float("inf")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(2, M, device="cuda")
    dgamma, dbeta = torch.empty(2, N, device="cuda")
    ck = B.Act8.empty(M, N, "int8")
    B.layer_norm(x, gamma, None, y, mean, rstd, ckpt=ck)
    B.layer_norm_backward(dy, gamma, None, rstd, dx, dgamma, dbeta, B.layer_norm_workspace(M, N), **(dict(ckpt=ck) if kept else dict(x=x, mean=mean)))
    xh = (x - mean[:, None]) * rstd[:, None]
    if kept:
        xh = torch.empty_like(x)
        B.act8_unpack(ck, xh)
    gh = dy.double() * gamma.double()
    c1, c2 = gh.mean(1, keepdim=True), (gh * xh.double()).mean(1, keepdim=True)
    want = rstd.double()[:, None] * (gh - c1 - xh.double() * c2)
    assert torch.equal(want.isnan(), dx.isnan())
    assert torch.equal(want.isneginf(), dx.isneginf()) and torch.equal(want.isposinf(), dx.isposinf())
    others = torch.arange(M, device="cuda") != row
    assert bool(dx[others].isfinite().all())
    for t in (dgamma, dbeta):
        assert float(t[col]) == float("inf")
        assert int((~t.isfinite()).sum()) == 1


@pytest.mark.parametrize("N", [8, 64, 200, 361, 512, 1000, 1024, 1032])
@pytest.mark.parametrize("M", [1, 2, 5, 8, 9, 32, 33, 64, 65])
def test_few_rows_column_sums(M, N):
    """Batches on both sides of the size up to which one launch does all: column sums against 64 bits, twice the same bits, no
    workspace beyond what was asked for, either of the two left out."""
    g = torch.Generator(device="cuda").manual_seed(M * N)
    x, dy = (torch.randn(M, N, device="cuda", generator=g) for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(2, M, device="cuda")
    B.layer_norm(x, None, None, y, mean, rstd)
    need = B.layer_norm_workspace(M, N).numel()
    store = torch.full((need + 256,), 170, dtype=torch.uint8, device="cuda")
    out = []
    for which in (3, 3, 1, 2):
        sums = torch.full((2, N), SENTINEL, device="cuda")
        B.layer_norm_backward(dy, None, None, rstd, dx, sums[0] if which & 1 else None, sums[1] if which & 2 else None, store[:need], x=x, mean=mean)
        out.append(sums)
    assert bool((store[need:] == 170).all())
    assert torch.equal(out[0], out[1])
    assert torch.equal(out[2][0], out[0][0]) and bool((out[2][1] == SENTINEL).all())
    assert torch.equal(out[3][1], out[0][1]) and bool((out[3][0] == SENTINEL).all())
    # products exact to U each (the same xh, in fp32), sums of at most M terms in fp32
    xh = ((x - mean[:, None]) * rstd[:, None]).double()
    terms = dy.double() * xh
    assert bool(((out[0][0].double() - terms.sum(0)).abs() <= (M + 2) * ref.U * terms.abs().sum(0) + 1e-30).all())
    assert bool(((out[0][1].double() - dy.double().sum(0)).abs() <= (M + 2) * ref.U * dy.double().abs().sum(0) + 1e-30).all())
