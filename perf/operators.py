"""Layer norm of the hidden layers and 8-bit activation checkpoints, as timed cases.

A case is a dict of plain values; `prepare` makes the inputs a training script holds, `run` makes one pass through an
operator, in its plain form or (own) through the library, `exact` states its result in 64 bits.  Five kinds of pass:

  norm       layer norm forward: y = act(gamma xh + beta), xh = (x - mean) rstd, with the row statistics
  keep       the same, keeping xh in 8 bits, and the values that the backward pass will read back
  grad       layer norm backward: dx, dgamma, dbeta, from the forward's input and statistics, or from the 8-bit xh
  round      a matrix stored in 8 bits and restored
  weight     the weight gradient of a linear layer, dZ^T H, with H restored from 8 bits as it is multiplied

The 8-bit form: 32 consecutive columns of a row share a power of two 2^e, the smallest (e >= -100) with which the
largest magnitude among them fits the code's range (127 for int8, 448 for e4m3); a code is the value over 2^e rounded to
nearest, ties to even.  In the backward pass an element counts as passed by the ReLU if gamma xh + beta > 0 for
the xh of the forward pass, fl32(fl32(x - mean) rstd), or the restored one.  A restored H under gamma, beta and ReLU is
rounded to fp32 and then to bf16, the values that a bf16 product reads.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32


def listed():
    return [
        # a debugging run or a handful of characters: one small minibatch, latency counts
        dict(name="norm_64x1024", kind="norm", rows=64, cols=1024, ld=1024, src="bf16", dst="bf16", relu=True),
        # observation rows of 24-body characters, an env count that is a multiple of nothing, normalised into bf16
        dict(name="norm_9001x577_f32", kind="norm", rows=9001, cols=577, ld=580, src="f32", dst="bf16", relu=False),
        # a hidden layer of the headline configuration's networks on one large minibatch
        dict(name="norm_131072x1024", kind="norm", rows=131072, cols=1024, ld=1024, src="bf16", dst="bf16", relu=True),
        # the wide layer of the reset-heavy configuration, kept in 8 bits for the backward pass
        dict(name="keep_32768x2048_int8", kind="keep", rows=32768, cols=2048, ld=2048, src="bf16", dst="bf16", relu=True, form="int8"),
        # backward, fp32 network on 64 rows
        dict(name="grad_64x512_f32", kind="grad", rows=64, cols=512, ld=512, src="f32", dst="f32", relu=True, form="none"),
        # backward on a minibatch of 16000 rows from the bf16 pre-activations
        dict(name="grad_16000x1024", kind="grad", rows=16000, cols=1024, ld=1024, src="bf16", dst="bf16", relu=True, form="none"),
        # backward of one large minibatch from the 8-bit checkpoint
        dict(name="grad_131072x1024_int8", kind="grad", rows=131072, cols=1024, ld=1024, src="bf16", dst="bf16", relu=True, form="int8"),
        # activations of a large minibatch stored in 8 bits between forward and backward
        dict(name="round_131072x1024_int8", kind="round", rows=131072, cols=1024, ld=1024, src="bf16", form="int8"),
        # observation rows of 15-body characters kept as e4m3
        dict(name="round_9001x361_e4m3", kind="round", rows=9001, cols=361, ld=364, src="f32", form="e4m3"),
        # second hidden layer's weights, a minibatch of 16000 rows
        dict(name="weight_16000x512x1024", kind="weight", rows=16000, outs=512, cols=1024, affine=True, form="int8"),
        # the largest product of the headline networks: 131072 rows, 1024 -> 1024
        dict(name="weight_131072x1024x1024", kind="weight", rows=131072, outs=1024, cols=1024, affine=True, form="int8"),
        # the action head of 24-body characters: a narrow product that reads far more than it multiplies
        dict(name="weight_65536x69x512_e4m3", kind="weight", rows=65536, outs=69, cols=512, affine=False, form="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "keep", "grad", "grad", "round", "weight", "weight"])
    form = rng.choice(["int8", "int8", "e4m3"])
    if kind == "weight":
        return dict(kind=kind, rows=_log_int(rng, 64, 131072), outs=rng.choice([28, 69, 64, 512, 1024, rng.randrange(1, 1025)]),
                    cols=rng.choice([512, 1024, rng.randrange(16, 1025)]), affine=rng.random() < 0.6, form=form)
    cols = rng.choice([64, 512, 1024, 2048, _log_int(rng, 16, 4096)])
    rows = _log_int(rng, 1, min(131072, (131072 * 1024) // cols))
    ld = rng.choice([cols, (cols + 7) // 8 * 8, (cols + 63) // 64 * 64])
    src = rng.choice(["bf16", "bf16", "f32"])
    if src == "f32":
        rows = max(1, rows // 2)
    if kind == "round":
        return dict(kind=kind, rows=rows, cols=cols, ld=ld, src=src, form=form)
    if kind == "grad":
        return dict(kind=kind, rows=rows, cols=cols, ld=ld, src=src, dst=src, relu=rng.random() < 0.7, form=rng.choice(["none", form]))
    case = dict(kind=kind, rows=rows, cols=cols, ld=ld, src=src, dst=rng.choice([src, "bf16"]), relu=rng.random() < 0.7)
    return dict(case, form=form) if kind == "keep" else case


_SIZE = {"f32": 4, "bf16": 2}
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def work(case):
    R, N, kind = case["rows"], case["cols"], case["kind"]
    held = R * N + R * ((N + BLOCK - 1) // BLOCK)                    # codes and one scale byte per block
    if kind == "norm":
        return {"bytes": R * N * (_SIZE[case["src"]] + _SIZE[case["dst"]]) + 8 * N + 8 * R, "flops": 8 * R * N}
    if kind == "keep":                                                # stored, and read back as bf16
        return {"bytes": R * N * (_SIZE[case["src"]] + _SIZE[case["dst"]] + 2) + 2 * held + 8 * N + 8 * R, "flops": 12 * R * N}
    if kind == "grad":
        x = held + 4 * R if case["form"] != "none" else R * N * _SIZE[case["src"]] + 8 * R
        return {"bytes": x + R * N * (_SIZE[case["dst"]] + _SIZE[case["src"]]) + 16 * N, "flops": 14 * R * N}
    if kind == "round":
        return {"bytes": 2 * R * N * _SIZE[case["src"]] + 2 * held, "flops": 4 * R * N}
    M = case["outs"]
    return {"bytes": 2 * R * M + held + 4 * M * N, "flops": 2 * R * M * N}


# ---------------------------------------------------------------------------------------------- inputs
def _matrix(g, rows, cols, ld, dtype, scale=None, shift=None):
    """[rows, cols] of normal values with a row stride of ld elements, columns of unlike spread and offset."""
    x = torch.zeros(rows, ld, device="cuda", dtype=dtype)
    v = torch.randn(rows, cols, device="cuda", generator=g)
    if scale is not None:
        v.mul_(scale).add_(shift)
    x[:, :cols] = v
    return x[:, :cols]


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    R, N, kind = case["rows"], case["cols"], case["kind"]
    st = dict(case=case, relu=case.get("relu", case.get("affine", False)))
    rand = lambda n: torch.randn(n, device="cuda", generator=g)  # noqa: E731
    st["gamma"], st["beta"] = 1 + 0.2 * rand(N), 0.3 * rand(N)
    spread, offset = torch.exp(0.5 * rand(N)), 0.5 * rand(N)      # pre-activations: some columns are wide, some are offset
    new = lambda *shape, **kw: torch.empty(*shape, device="cuda", **kw)  # noqa: E731
    if kind == "weight":
        ld_dz = (case["outs"] + 63) // 64 * 64                    # gradient rows are padded to the products' 64 columns
        st["dz"] = _matrix(g, R, case["outs"], ld_dz, torch.bfloat16)
        h = torch.randn(R, N, device="cuda", generator=g)
        st["code"], st["scale"] = _to_bytes(h if case["affine"] else h.relu_(), case["form"])
        st["out"], st["status"] = new(case["outs"], N), torch.zeros(1, dtype=torch.int32, device="cuda")
        if not case["affine"]:
            st["gamma"] = st["beta"] = None
        return st
    src = _TYPE[case["src"]]
    st["x"] = _matrix(g, R, N, case["ld"], src, spread, offset)
    if kind == "round":
        st["out"] = new(R, N, dtype=src)
        st["code"], st["scale"] = _empty_bytes(R, N)
        return st
    dst = _TYPE[case["dst"]]
    st["mean"], st["rstd"] = new(R), new(R)
    if kind == "grad":
        x = st["x"].double()
        mean = x.mean(1)
        rstd = 1 / torch.sqrt((x - mean[:, None]).square_().mean(1) + EPS)
        st["mean"], st["rstd"] = mean.float(), rstd.float()
        st["dy"] = _matrix(g, R, N, case["ld"], dst)
        st["dx"], st["dgamma"], st["dbeta"] = new(R, N, dtype=src), new(N), new(N)
        if case["form"] != "none":
            st["code"], st["scale"] = _to_bytes(((x - mean[:, None]) * rstd[:, None]).float(), case["form"])
            del st["x"]
        return st
    st["y"] = new(R, N, dtype=dst)
    if kind == "keep":
        st["out"] = new(R, N, dtype=torch.bfloat16)
        st["code"], st["scale"] = _empty_bytes(R, N)
    return st


def _empty_bytes(rows, cols):
    return (torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.uint8, device="cuda"),
            torch.zeros(rows, (cols + BLOCK - 1) // BLOCK, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------------------------------------- plain forms
def _blocks(x):
    """[rows, blocks, 32] view of x, the last block filled up with zeros."""
    pad = -x.shape[1] % BLOCK
    x = torch.cat([x, x.new_zeros(x.shape[0], pad)], 1) if pad else x
    return x.view(x.shape[0], -1, BLOCK)


def _exponents(b, form):
    """The blocks' exponents e (int32): the least >= -100 with max |b| <= top 2^e."""
    top = 127.0 if form == "int8" else 448.0
    amax = b.abs().amax(2)
    e = torch.floor(torch.log2(torch.clamp(amax, min=2.0 ** -110) / top)).int() - 1
    for _ in range(2):                                              # log2 may be off by one at a border
        e = torch.where(amax > top * torch.exp2(e.double()), e + 1, e)
    return torch.clamp(e, min=-100)


def _to_bytes(x, form):
    """(codes [rows, cols up to 16] uint8, scales [rows, blocks] uint8 = e + 127) of a float32 matrix."""
    code, scale = _empty_bytes(*x.shape)
    b = _blocks(x)
    e = _exponents(b, form)
    v = torch.ldexp(b, -e[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]]
    c = torch.round(v).to(torch.int8).view(torch.uint8) if form == "int8" else v.to(torch.float8_e4m3fn).view(torch.uint8)
    code[:, :x.shape[1]] = c
    scale[:] = (e + 127).to(torch.uint8)
    return code, scale


def _from_bytes(code, scale, cols, form):
    c = code[:, :cols]
    v = c.view(torch.int8).float() if form == "int8" else c.view(torch.float8_e4m3fn).float()
    s = torch.exp2(scale.float() - 127).repeat_interleave(BLOCK, 1)[:, :cols]
    return v * s


def _affine(v, st):
    """fl32(gamma v + beta), rounded once: the sum is formed in 64 bits."""
    v = (v.double() * st["gamma"].double()).add_(st["beta"].double()).float()
    return v.relu_() if st["relu"] else v


def _plain(st):
    case = st["case"]
    kind, N = case["kind"], case["cols"]
    if kind == "weight":
        h = _from_bytes(st["code"], st["scale"], N, case["form"])
        if case["affine"]:
            h = _affine(h, st).bfloat16().float()
        return st["dz"].float().T @ h
    if kind == "round":
        code, scale = _to_bytes(st["x"].float(), case["form"])
        return _from_bytes(code, scale, N, case["form"]).to(st["out"].dtype)
    if kind == "grad":
        if case["form"] != "none":
            xh = _from_bytes(st["code"], st["scale"], N, case["form"])
        else:
            xh = (st["x"].float() - st["mean"][:, None]) * st["rstd"][:, None]
        h = st["dy"].float()
        if st["relu"]:
            h = torch.where(xh.double() * st["gamma"].double() + st["beta"].double() > 0, h, torch.zeros_like(h))
        hx = h * xh
        dgamma, dbeta = hx.sum(0, dtype=torch.float64).float(), h.sum(0, dtype=torch.float64).float()
        g = h * st["gamma"]
        c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        dx = (g - c1 - xh * c2) * st["rstd"][:, None]
        return dict(dx=dx.to(st["dx"].dtype), dgamma=dgamma, dbeta=dbeta)
    x = st["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + EPS)
    xh = d * rstd[:, None]
    y = xh * st["gamma"] + st["beta"]
    y = (torch.clamp(y, min=0) if st["relu"] else y).to(st["y"].dtype)
    if kind == "norm":
        return dict(y=y, mean=mean, rstd=rstd)
    code, scale = _to_bytes(xh, case["form"])
    return dict(y=y, mean=mean, rstd=rstd, kept=_from_bytes(code, scale, N, case["form"]).bfloat16())


def run(state):
    if not own:
        return _plain(state)
    from paper_2609_09821_b200 import binding as B
    st, case = state, state["case"]
    kind, R, N = case["kind"], case["rows"], case["cols"]
    ckpt = B.Act8(st["code"], st["scale"], N, case["form"]) if case.get("form", "none") != "none" else None
    if kind == "norm":
        B.layer_norm(st["x"], st["gamma"], st["beta"], st["y"], st["mean"], st["rstd"], eps=EPS, relu=st["relu"])
        return dict(y=st["y"], mean=st["mean"], rstd=st["rstd"])
    if kind == "keep":
        B.layer_norm(st["x"], st["gamma"], st["beta"], st["y"], st["mean"], st["rstd"], eps=EPS, relu=st["relu"], ckpt=ckpt)
        B.act8_unpack(ckpt, st["out"])
        return dict(y=st["y"], mean=st["mean"], rstd=st["rstd"], kept=st["out"])
    if kind == "grad":
        if "ws" not in st:                                          # a script allocates its workspace once
            st["ws"] = B.layer_norm_workspace(R, N)
        B.layer_norm_backward(st["dy"], st["gamma"], st["beta"], st["rstd"], st["dx"], st["dgamma"], st["dbeta"], st["ws"],
                              relu=st["relu"], x=st.get("x"), mean=st["mean"] if ckpt is None else None, ckpt=ckpt)
        return dict(dx=st["dx"], dgamma=st["dgamma"], dbeta=st["dbeta"])
    if kind == "round":
        B.act8_pack(st["x"], ckpt)
        B.act8_unpack(ckpt, st["out"])
        return st["out"]
    if "ws" not in st:
        st["ws"] = B.gemm_act8_tn_workspace(R, case["outs"], N)
    B.gemm_act8_tn(st["dz"], ckpt, st["out"], st["ws"], st["status"], gamma=st["gamma"], beta=st["beta"], relu=st["relu"])
    return st["out"]


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_e4m3(v):
    """v (float64, |v| <= 448) rounded to four significant bits, or to multiples of 2^-9 below 2^-6, ties to even."""
    _, e = torch.frexp(v)                                          # |v| = m 2^e, m in [1/2, 1)
    q = torch.clamp(e - 1, min=-6) - 3
    return torch.ldexp(torch.round(torch.ldexp(v, -q)), q)


def _exact_round(x, form):
    """The values that the 8-bit form of x stands for."""
    R, N = x.shape
    out = torch.empty_like(x)
    top = 127.0 if form == "int8" else 448.0
    for c in range(0, N, BLOCK):
        b = x[:, c:c + BLOCK]
        m, e = torch.frexp(b.abs().amax(1) / top)                  # amax / top = m 2^e, m in [1/2, 1): the power above, or itself
        e = torch.where(m == 0.5, e - 1, e)
        e = torch.where(m == 0, torch.full_like(e, -100), e).clamp_(min=-100)[:, None]
        v = torch.ldexp(b, -e)
        out[:, c:c + BLOCK] = torch.ldexp(torch.round(v) if form == "int8" else _exact_e4m3(v), e)
    return out


def _exact_restore(st, cols):
    """Codes to values, from the bits of each code."""
    case = st["case"]
    c = st["code"][:, :cols].to(torch.int32)
    if case["form"] == "int8":
        v = torch.where(c > 127, c - 256, c).double()
    else:
        e, m = (c >> 3) & 15, (c & 7).double()
        v = torch.where(e > 0, torch.ldexp(8 + m, (e - 10)), torch.ldexp(m, torch.full_like(e, -9)))
        v = torch.where(c > 127, -v, v)
    block = torch.arange(cols, device="cuda") // BLOCK
    return torch.ldexp(v, st["scale"].to(torch.int32)[:, block] - 127)


def exact(case, seed):
    st = prepare(case, seed)
    kind, N = case["kind"], case["cols"]
    if kind == "weight":
        h = _exact_restore(st, N)
        if case["affine"]:                                          # the operand is defined as the bf16 value of the fp32 one
            h = torch.clamp(h * st["gamma"].double() + st["beta"].double(), min=0).to(torch.float32).to(torch.bfloat16).double()
        return torch.einsum("rn,rk->nk", st["dz"].double(), h)
    if kind == "round":
        return _exact_round(st["x"].double(), case["form"])
    gamma, beta = st["gamma"].double(), st["beta"].double()
    if kind == "grad":
        rstd = st["rstd"].double()[:, None]
        if case["form"] != "none":
            xh = _exact_restore(st, N)
            passed = xh
        else:
            xh = (st["x"].double() - st["mean"].double()[:, None]) * rstd
            passed = torch.mul(torch.sub(st["x"].float(), st["mean"][:, None]), st["rstd"][:, None]).double()   # the forward's fp32 value decides
        h = st["dy"].double()
        if st["relu"]:
            h = h * (passed * gamma + beta > 0)
        dgamma, dbeta = torch.einsum("rn,rn->n", h, xh), h.sum(0)
        g = h.mul_(gamma)
        dx = rstd * (g - g.sum(1, keepdim=True) / N - xh * ((g * xh).sum(1, keepdim=True) / N))
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    x = st["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    rstd = torch.rsqrt(var + EPS)
    xh = (x - mean[:, None]) * rstd[:, None]
    y = xh * gamma + beta
    y = torch.relu(y) if st["relu"] else y
    if kind == "norm":
        return dict(y=y, mean=mean, rstd=rstd)
    return dict(y=y, mean=mean, rstd=rstd, kept=_exact_round(xh, case["form"]))
