"""A policy with layer-normed hidden layers, one gradient through the building blocks: products, norms, activations kept in 8 bits,
and the weight gradients from them, against the same chain in 64 bits (rounded where the chain rounds)."""
import pytest

from tests import norm_reference as ref

pytestmark = pytest.mark.gpu


def bf(x):
    import torch
    return x.to(torch.float32).to(torch.bfloat16).double()


@pytest.mark.parametrize("M,widths,form", [(640, (361, 512, 256, 28), ref.INT8), (1088, (577, 256, 320, 69), ref.E4M3), (64, (100, 64, 64, 5), ref.INT8)])
@pytest.mark.parametrize("keep", [True, False])
def test_one_gradient(M, widths, form, keep):
    import torch
    from paper_2609_09821_b200 import binding as B
    g = torch.Generator("cuda").manual_seed(M)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    pad = lambda n: (n + 63) // 64 * 64  # noqa: E731
    D, N1, N2, A = widths
    EPS = 1e-5
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    W = [torch.zeros(rows, pad(cols), device="cuda", dtype=torch.bfloat16) for rows, cols in ((N1, D), (N2, N1), ((A + 15) // 16 * 16, N2))]
    for w, (rows, cols) in zip(W, ((N1, D), (N2, N1), (A, N2))):
        w[:rows, :cols] = rand(rows, cols) * cols ** -0.5
    gamma, beta = [1 + 0.2 * rand(n) for n in (N1, N2)], [0.3 * rand(n) for n in (N1, N2)]
    bias = [0.1 * rand(N1), 0.1 * rand(N2), torch.zeros(W[2].shape[0], device="cuda")]
    obs = torch.zeros(M, pad(D), device="cuda", dtype=torch.bfloat16)
    obs[:, :D] = rand(M, D)
    d_out = torch.zeros(M, pad(A), device="cuda", dtype=torch.bfloat16)
    d_out[:, :A] = rand(M, A)

    # forward: products, norms with the normalised rows kept in 8 bits (or pre-activations and statistics kept instead)
    e = lambda r, c, dt=torch.bfloat16: torch.empty(r, c, device="cuda", dtype=dt)  # noqa: E731
    x, Z, Y, mean, rstd, ck = obs, [], [], [], [], []
    for l, n in enumerate((N1, N2)):
        Z.append(e(M, n)), Y.append(e(M, n)), mean.append(torch.empty(M, device="cuda")), rstd.append(torch.empty(M, device="cuda"))
        ck.append(B.Act8.empty(M, n, form))
        B.gemm_bf16(x, W[l], Z[l], bias[l], False, status)
        B.layer_norm(Z[l], gamma[l], beta[l], Y[l], mean[l], rstd[l], eps=EPS, relu=True, ckpt=ck[l])
        x = Y[l]
    out = e(M, A, torch.float32)
    B.gemm_bf16_f32out(x, W[2], out, bias[2], status)

    # backward: weight gradients from the kept rows, the norm's backward pass from them too
    ws_n = B.layer_norm_workspace(M, max(N1, N2))
    held = ck if keep else [B.Act8.empty(M, n, form) for n in (N1, N2)]
    if not keep:                                                           # the layer outputs themselves in 8 bits
        for l in (0, 1):
            B.act8_pack(Y[l], held[l])
    how = lambda l: dict(gamma=gamma[l], beta=beta[l], relu=True) if keep else {}  # noqa: E731
    grad = lambda dz, rows, l: _product(B, torch, dz, held[l], rows, how(l), status)  # noqa: E731
    dW3 = grad(d_out[:, :A], A, 1)
    dZ, dgam, dbet = [None, None], [torch.empty(N1, device="cuda"), torch.empty(N2, device="cuda")], [torch.empty(N1, device="cuda"), torch.empty(N2, device="cuda")]
    up = d_out
    for l, n in ((1, N2), (0, N1)):
        Wt = e(n, up.shape[1])
        Wt.zero_()
        Wt[:, :W[l + 1].shape[0]] = W[l + 1][:, :n].T
        dH = e(M, n)
        B.gemm_bf16_dgrad(up, Wt, dH, None, None, status)
        dZ[l] = dH                                                         # in place
        src = dict(ckpt=ck[l]) if keep else dict(x=Z[l], mean=mean[l])
        B.layer_norm_backward(dH, gamma[l], beta[l], rstd[l], dZ[l], dgam[l], dbet[l], ws_n, relu=True, **src)
        up = dZ[l]
    dW2 = grad(dZ[1], N2, 0)
    obs8 = B.Act8.empty(M, D, form)
    B.act8_pack(obs[:, :D], obs8)
    dW1 = _product(B, torch, dZ[0], obs8, N1, {}, status)
    assert int(status) == 0

    # the same in 64 bits, rounded where the chain rounds
    x, zs, xhs, kept, rs, ys = obs.double(), [], [], [], [], []
    for l in (0, 1):
        z = bf(x @ W[l].double().T + bias[l].double())
        _, r, xh, y = ref.forward(z, gamma[l], beta[l], EPS, True)
        zs.append(z), xhs.append(xh), kept.append(ref.kept(xh.float(), form)), rs.append(r)
        x = bf(y)
        ys.append(x)
    want_out = x @ W[2].double().T[:, :A]
    hs = [bf(torch.relu(ref.affine(k, gamma[l], beta[l]))) for l, k in enumerate(kept)] if keep else [ref.kept(y, form) for y in ys]
    up, want = d_out.double(), {}
    want["dW3"] = up[:, :A].T @ hs[1]
    Wd = [w.double() for w in W]
    for l in (1, 0):
        rows = Wd[l + 1].shape[0]
        dH = bf(up[:, :rows] @ Wd[l + 1][:, :(N1, N2)[l]])
        xh = kept[l] if keep else xhs[l]
        dx, dg, db, _, _, _ = ref.backward(dH, xh, ref.affine(xh, gamma[l], beta[l]) > 0, rs[l], gamma[l], True)
        want["dgamma%d" % l], want["dbeta%d" % l] = dg, db
        up = bf(dx)
        want["dZ%d" % l] = up
    want["dW2"] = want["dZ1"].T @ hs[0]
    want["dW1"] = want["dZ0"].T @ ref.kept(obs[:, :D], form)
    got = dict(dW3=dW3, dW2=dW2, dW1=dW1, dgamma0=dgam[0], dgamma1=dgam[1], dbeta0=dbet[0], dbeta1=dbet[1], dZ0=dZ[0], dZ1=dZ[1])
    # a value passes four roundings to bf16 in a row at most; two sides that round next to a border differ by a step, half a
    # step (2^-8) each: 4 x 2^-8 if that happened to every value
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, want_out) <= 4 * 2.0 ** -8
    far = {k: rel(got[k], want[k]) for k in want}
    assert all(v <= 4 * 2.0 ** -8 for v in far.values()), far


def _product(B, torch, dz, ckpt, rows, how, status):
    out = torch.empty(rows, ckpt.cols, device="cuda")
    B.gemm_act8_tn(dz, ckpt, out, B.gemm_act8_tn_workspace(dz.shape[0], rows, ckpt.cols), status, **how)
    return out
