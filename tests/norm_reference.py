"""Layer norm, its gradients and the 8-bit form of activations in 64 bits (torch on whichever device the inputs are on)."""
import torch

BLOCK = 32
INT8, E4M3 = "int8", "e4m3"
TOP = {INT8: 127.0, E4M3: 448.0}
U = 2.0 ** -24                     # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def exponents(x, form):
    """[rows, blocks]: least e >= -100 with max |x| <= top 2^e over each block of 32 columns; None where a block is not finite."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    amax = x.abs().amax(2)
    bad = ~torch.isfinite(x).all(2)
    m, e = torch.frexp(torch.where(bad, torch.zeros_like(amax), amax) / TOP[form])      # the division is exact to 2^-53: a power of two stays one
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(m == 0, torch.full_like(e, -100), e).clamp(min=-100)
    return e, bad


def round_form(v, form):
    """v (already over 2^e) rounded to the codes' values."""
    if form == INT8:
        return torch.round(v)
    _, e = torch.frexp(v)
    q = torch.clamp(e - 1, min=-6) - 3
    return torch.ldexp(torch.round(torch.ldexp(v, -q)), q)


def kept(x, form):
    """The values that the 8-bit form of x stands for (float64)."""
    cols = x.shape[1]
    e, bad = exponents(x, form)
    e = e.repeat_interleave(BLOCK, 1)[:, :cols]
    v = torch.ldexp(round_form(torch.ldexp(x.double(), -e), form), e)
    return torch.where(bad.repeat_interleave(BLOCK, 1)[:, :cols], torch.full_like(v, float("nan")), v)


def forward(x, gamma, beta, eps, relu):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    y = affine(xh, gamma, beta)
    return mean, rstd, xh, (torch.where(y < 0, torch.zeros_like(y), y) if relu else y)


def affine(xh, gamma, beta):
    y = xh if gamma is None else xh * gamma.double()
    return y if beta is None else y + beta.double()


def backward(dy, xh, passed, rstd, gamma, relu):
    """dx, dgamma, dbeta (float64) and the absolute sums that bound their rounding errors; passed: the ReLU's decision."""
    h = dy.double()
    h = torch.where(passed, h, torch.zeros_like(h)) if relu else h
    g = h if gamma is None else h * gamma.double()
    gx = g * xh
    c1, c2 = g.mean(1, keepdim=True), gx.mean(1, keepdim=True)
    r = rstd.double()[:, None]
    dx = r * (g - c1 - xh * c2)
    # an fp32 sum of eight terms in a row and at most 5 + 32 pairwise levels: 45 roundings; xh itself is off by 2
    a1, a2 = g.abs().mean(1, keepdim=True), gx.abs().mean(1, keepdim=True)
    err = r * U * (46 * a1 + xh.abs() * 52 * a2 + 6 * (g.abs() + c1.abs() + (xh * c2).abs()))
    hx = h * xh
    return dx, hx.sum(0), h.sum(0), err, hx.abs().sum(0), h.abs().sum(0)
