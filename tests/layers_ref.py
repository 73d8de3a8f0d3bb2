"""The layer operators' formulas in 64 bits, and how far a result may be from them.

Bounds are derived, not fitted.  u(type) is half a spacing relative to the value
(2^-8 for bf16, 2^-11 for f16).  A sum of k products on the tensor cores takes
at most k/16 + 16 steps (32 bytes of depth each, and the joining of parts), each
off by at most 2^-22 of the sum of the magnitudes S.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
STEP = 2.0 ** -22
D = torch.float64
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
SLOPE = 1.13   # the largest |act'|
CURVE = 1.13   # the largest |act''|


def act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return z * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    """act' by its formula."""
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        g = torch.sigmoid(z)
        return g + z * g * (1 - g)
    return torch.ones_like(z)


def sum_error(p, q, depth):
    """Bound of the error of p·qᵀ's sums (p, q in 64 bits, depth their length)."""
    return (depth / 16 + 16) * STEP * (p.abs() @ q.abs().t())


def linear(x, w, bias=None, name="none", residual=None, x_scale=None, w_scale=None, out=None):
    """(y, z, bound of y's error, bound of z's error)."""
    out = out or (x.dtype if x.dtype in U else torch.bfloat16)
    X, W = x.to(D), w.to(D)
    if x_scale is not None:
        X, W = X * x_scale.to(D)[:, None], W * w_scale.to(D)[:, None]
    z = X @ W.t()
    err = sum_error(X, W, x.shape[1])
    if bias is not None:
        z = z + bias.to(D)
    err = err + 2 * STEP * z.abs()
    y = act(z, name)
    yerr = SLOPE * err + 2.0 ** -19 * (z.abs() + y.abs())  # exp, erf and a division in 32 bits
    if residual is not None:
        y = y + residual.to(D)
        yerr = yerr + STEP * y.abs()

    def rounded(v, e):
        return e + U[out] * (v.abs() + e) + TINY[out]

    return y, z, rounded(y, yerr), rounded(z, err)


def grad(dy, x, w, z, name):
    """((dx, dw, db), (bounds)): dz is rounded to its type before the products."""
    dt = dy.dtype
    dz = dy.to(D)
    ez = torch.zeros_like(dz)
    if name != "none":
        s = slope(z.to(D), name)
        ez = dy.to(D).abs() * 2.0 ** -20 * (1 + z.to(D).abs())  # the slope, in 32 bits
        dz = dz * s
    er = ez + U[dt] * (dz.abs() + ez) + TINY[dt] if name != "none" else ez
    X, W = x.to(D), w.to(D)
    m, n = dy.shape
    dx, dw, db = dz @ W, dz.t() @ X, dz.sum(0)

    def rounded(v, e, t=dt):
        return e + U[t] * (v.abs() + e) + TINY[t]

    a = dz.abs() + er
    bx = rounded(dx, er @ W.abs() + sum_error(a, W.t().contiguous(), n))
    ew = er.t() @ X.abs() + sum_error(a.t().contiguous(), X.t().contiguous(), m)
    bw = rounded(dw, ew)
    bb = ez.sum(0) + (m / 8 + 16) * 2.0 ** -23 * dz.abs().sum(0) + 2.0 ** -126
    return (dx, dw, db), (bx, bw, bb), ew


def close(got, want, bound, what=""):
    got = got.to(D)
    bad = ~((got - want).abs() <= bound)
    if bad.any():
        at = torch.nonzero(bad)[0].tolist()
        at = tuple(at)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} entries out of bounds, first at {at}: "
                             f"{got[at].item()} for {want[at].item()} ± {bound[at].item()}")


def e4m3_rows(t):
    scale = t.abs().amax(dim=1).clamp_min(1e-12) / 448
    return (t / scale[:, None]).to(torch.float8_e4m3fn), scale
