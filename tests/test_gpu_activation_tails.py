"""Activations and their slopes where they are small: errors relative to the value, in
64 bits, so that a tail that is lost or wrong shows."""
import math

import pytest

from helpers import ensure_built

pytestmark = pytest.mark.gpu

FLUSH = 2.0 ** -126  # a factor of z that is smaller may count as 0


@pytest.fixture(scope="module")
def env():
    ensure_built()
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_06510_gb300 as oz
    yield oz, torch
    torch.cuda.synchronize()
    assert oz.oz2_check_device_status() == 0


def two_u(z):
    return 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)


def factor(torch, z, name):
    """act(z)/z, without a difference of near values anywhere."""
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return torch.sigmoid(two_u(z) if name == "gelu_tanh" else z)


def exponent(z, name):
    """The size of the argument of exp in it."""
    return z * z / 2 if name == "gelu" else two_u(z).abs() if name == "gelu_tanh" else z.abs()


def slope_terms(torch, z, name):
    """The two terms that act' is the sum of."""
    f = factor(torch, z, name)
    if name == "gelu":
        return f, z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    g = f * torch.sigmoid(-two_u(z) if name == "gelu_tanh" else -z)
    inner = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z) if name == "gelu_tanh" else 1.0
    return f, z * g * inner


def relative(z, name):
    """Relative error of a factor: 2^-19 of the approximations, 2^-20 of a dozen
    roundings and of ex2 and rcp, and exp's argument, of up to eight roundings of 2^-24."""
    return 1.5 * 2.0 ** -19 + exponent(z, name) * 2.0 ** -21


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("m, k", [(1, 0), (24, 0), (300, 0), (3000, 0), (3, 13)])
def test_activation(env, name, kind, m, k):
    """z from a float32 bias: [-14, 0] densely, and out to where nothing is left.  The
    result is what some float32 within the error of the formula rounds to (rounding
    keeps order, so it lies between what the error's ends round to)."""
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[kind]
    bias = torch.cat([torch.linspace(-14, 0, 2501), torch.linspace(-130, -14, 501), torch.linspace(0, 14, 501),
                      -torch.logspace(-40, 30, 300, dtype=torch.float64).float()]).cuda()
    n = bias.numel()
    x, w = torch.zeros(m, k, dtype=dt, device="cuda"), torch.zeros(n, k, dtype=dt, device="cuda")
    y = oz.oz2_linear(x, w, bias=bias, act=name)
    assert (y == y[0]).all()
    z = bias.double()
    f = factor(torch, z, name)
    want = z * f
    off = want.abs() * relative(z, name) + z.abs() * FLUSH
    got, low, high = (t.to(dt).double() for t in (y[0], want - off, want + off))
    bad = ~((low <= got) & (got <= high))
    assert not bad.any(), (int(bad.sum()), z[bad][:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_slope(env, name, kind):
    """act'(z) at every finite 16-bit z, in float32: db of one token with dy = 1."""
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[kind]
    pre = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dt)
    pre = pre[torch.isfinite(pre.float())].cuda()[None]
    n = pre.shape[1]
    x, w = torch.zeros(1, 8, dtype=dt, device="cuda"), torch.zeros(n, 8, dtype=dt, device="cuda")
    db = oz.oz2_linear_grad(torch.ones(1, n, dtype=dt, device="cuda"), x, w, pre=pre, act=name, need=("db",))[2]
    z = pre[0].double().clamp(-1e4, 1e4)  # beyond, the slope is 0 or 1 to 300 digits
    a, b = slope_terms(torch, z, name)
    want = a + b
    # Of positive z, exp's argument shows in what the factor lacks to 1, and what is left
    # of 1 is a difference, off by up to 2^-22.
    at = z.clamp(-100, 100) if name == "silu" else z.clamp(-20, 20)
    rel, least = relative(at, name), relative(torch.zeros_like(z), name)
    bound = b.abs() * rel + torch.where(z > 0, a * least + (1 - a) * rel, a * rel)
    bound += torch.where((z > 0) & (z < 16), b.abs() + z * (1 + z * z / 4), torch.zeros_like(z)) * 2.0 ** -22
    bound += FLUSH * (1 + z.abs().clamp_max(200) ** (3 if name == "gelu_tanh" else 1))
    got = db.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), z[bad][:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())
