"""The layer operators' entry points: exported, and refusing what they should on
the host (no GPU work is issued)."""
import ctypes
import os
import re

import pytest
import torch

from helpers import ROOT, ensure_built


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    oz.lib()
    return oz


def test_header_and_binding_agree(oz):
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "oz2_layers.h")).read(), flags=re.S)
    names = set(re.findall(r"^int (oz2_\w+)\(", txt, flags=re.M))
    assert names == set(oz.layers.SIGS)
    raw = ctypes.CDLL(oz.LIB_PATH)
    assert all(hasattr(raw, n) for n in names)
    assert ctypes.sizeof(oz.layers.oz2_adamw_tensor) == 72 and ctypes.sizeof(oz.layers.oz2_adamw_step) == 64


BF16, F16, E4M3, F32 = 1, 2, 3, 0
N = None


def linear(oz, m=8, n=8, k=8, type=BF16, X=16, ldx=8, W=16, ldw=8, xs=N, ws=N, bias=N, bt=0, act=0, R=N, ldr=0, Z=N,
           ldz=0, Y=16, ldy=8, out=BF16):
    return oz.lib().oz2_linear(m, n, k, type, X, ldx, W, ldw, xs, ws, bias, bt, act, R, ldr, Z, ldz, Y, ldy, out, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=-1), dict(k=-1), dict(act=5), dict(act=-1), dict(type=F32), dict(type=7), dict(out=F32),
    dict(out=F16), dict(type=E4M3, out=E4M3), dict(ldx=7), dict(ldw=7), dict(ldy=7), dict(R=16, ldr=7),
    dict(Z=16, ldz=7), dict(X=N), dict(W=N), dict(Y=N), dict(X=17), dict(Y=17), dict(bias=16, bt=F16),
    dict(bias=18, bt=F32), dict(xs=16), dict(xs=16, ws=16), dict(type=E4M3, ws=16), dict(type=E4M3, xs=18, ws=16)])
def test_linear_refuses(oz, bad):
    assert linear(oz, **bad) == -1


def test_linear_limits_and_empty(oz):
    big = (1 << 31) - 256
    assert linear(oz, m=big) == -6
    assert linear(oz, k=big, ldx=big, ldw=big) == -6
    assert linear(oz, m=0, X=N, Y=N) == 0
    assert linear(oz, n=0, W=N, Y=N) == 0


def grad(oz, m=8, n=8, k=8, type=BF16, dY=16, lddy=8, Z=16, ldz=8, act=4, X=16, ldx=8, W=16, ldw=8, dX=16, lddx=8,
         dW=16, lddw=8, wt=BF16, db=16, flags=0):
    return oz.lib().oz2_linear_grad(m, n, k, type, dY, lddy, Z, ldz, act, X, ldx, W, ldw, dX, lddx, dW, lddw, wt, db,
                                    flags, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=-1), dict(k=-1), dict(type=E4M3), dict(type=F32), dict(act=9), dict(lddy=7), dict(ldz=7),
    dict(ldx=7), dict(ldw=7), dict(lddx=7), dict(lddw=7), dict(dY=N), dict(Z=N), dict(X=N), dict(W=N), dict(dY=17),
    dict(db=18), dict(wt=F16), dict(wt=E4M3), dict(flags=2), dict(flags=1), dict(wt=F32, dW=18)])
def test_grad_refuses(oz, bad):
    assert grad(oz, **bad) == -1


def test_grad_limits_and_nothing_wanted(oz):
    big = (1 << 31) - 256
    assert grad(oz, m=big) == -6
    assert grad(oz, dX=N, dW=N, db=N) == 0
    assert grad(oz, m=0, dW=N, db=N) == 0
    assert grad(oz, m=0, wt=F32, flags=1) == 0


def adamw(oz, change=None, count=1, param=BF16, grad=BF16, bits=32, args=None, step=1, beta1=0.9, beta2=0.9, gs=N):
    t = (oz.layers.oz2_adamw_tensor * 1)()
    for name in ("param", "grad", "master", "m", "v", "m_scale", "v_scale"):
        setattr(t[0], name, 64)
    t[0].numel = 4
    for name, value in (change or {}).items():
        setattr(t[0], name, value)
    a = oz.layers.oz2_adamw_step(step, 1e-3, beta1, beta2, 1e-8, 0.0, gs, 0)
    return oz.lib().oz2_adamw(t, count, param, grad, bits, ctypes.byref(a) if args is None else args, N)


@pytest.mark.parametrize("bad", [
    dict(count=-1), dict(param=E4M3), dict(param=9), dict(param=BF16, grad=F16), dict(bits=16), dict(step=0),
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(gs=66),
    dict(change=dict(numel=-1)), dict(change=dict(grad=N)), dict(change=dict(m=N)), dict(change=dict(v=N)),
    dict(change=dict(param=N, master=N)), dict(bits=8, change=dict(m_scale=N)), dict(change=dict(m=66)),
    dict(change=dict(param=65)), dict(param=F32, grad=F32), dict(bits=8, change=dict(v_scale=66))])
def test_adamw_refuses(oz, bad):
    assert adamw(oz, **bad) == -1


def test_adamw_nothing_to_do(oz):
    assert adamw(oz, count=0) == 0
    assert adamw(oz, change=dict(numel=0, param=N, grad=N, m=N, v=N)) == 0


def test_binding_refuses(oz):
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear(x, w)
    with pytest.raises(AssertionError, match="one dtype"):
        oz.oz2_linear(x, w.half())
    with pytest.raises(AssertionError, match="one dtype"):
        oz.oz2_linear(x, w[:, :7])
    with pytest.raises(AssertionError, match="out_dtype"):
        oz.oz2_linear(x, w, out_dtype=torch.float16)
    with pytest.raises(AssertionError, match="one dtype"):
        oz.oz2_linear_grad(x.float(), x, w)
    with pytest.raises(AssertionError, match="every parameter"):
        oz.oz2_adamw_plan([x], [], [x], [x])
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_adamw_plan([x], [x], [x.float()], [x.float()])


def test_rounding_hash_scatters():
    """The bits the 8-bit states are rounded by: over consecutive values, every bit
    is set half of the time and agrees with every other one, and with its
    neighbours', half of the time (N = 2^16 values: 6 deviations are 0.012)."""
    mask = 0xFFFFFFFF

    def scatter(x):
        x = x ^ (x >> 16)
        x = (x * 0x6A09E667) & mask
        x = x ^ (x >> 15)
        x = (x * 0xBB67AE85) & mask
        return x ^ (x >> 16)

    for seed in (0, 1, 12345, mask):
        for step in (1, 2, 1000):
            key = scatter((scatter(seed) + step) & mask)
            n = 1 << 16
            at = torch.arange(n, dtype=torch.int64)
            h = scatter((at * 0x9E3779B1 + key) & mask)
            bits = ((h[:, None] >> torch.arange(32)) & 1).double() * 2 - 1
            assert (bits.mean(0).abs() < 6 / n ** 0.5).all()
            for lag in (0, 1, 2, 4, 32, 128, 256):
                c = bits[:n - lag].t() @ bits[lag:] / (n - lag)
                if lag == 0:
                    c = c - torch.eye(32, dtype=torch.double)
                assert (c.abs() < 6 / (n - lag) ** 0.5).all(), (seed, step, lag)
