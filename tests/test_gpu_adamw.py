"""oz2_adamw against its formulas: 32-bit states in 64 bits, 8-bit states bit for
bit against the definition of their format and rounding in float32."""
import math

import pytest

from helpers import ensure_built

pytestmark = pytest.mark.gpu

BLOCK = 256


@pytest.fixture(scope="module")
def env():
    ensure_built()
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_06510_gb300 as oz
    yield oz, torch
    torch.cuda.synchronize()


HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8, weight_decay=0.1)


def step64(torch, p, g, m, v, t, lr, beta1, beta2, eps, weight_decay):
    d = torch.float64
    p, g, m, v = (a.to(d) for a in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    u = (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps)
    return p - lr * weight_decay * p - lr * u, m, v, u


def weight64(torch, p, m, v, t, lr, beta1, beta2, eps, weight_decay):
    """(w, the update's share of it) from the m and v of the same step."""
    p, m, v = (a.to(torch.float64) for a in (p, m, v))
    u = (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps)
    return p - lr * weight_decay * p - lr * u, u


def pow2(torch, e):
    """2^e exactly, in 64 bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def close(torch, got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:3].tolist(), want[bad][:3].tolist())


def tensors(torch, sizes, dtype, grad, seed, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(std, dt):
        return [(torch.randn(e + offset, generator=g, device="cuda") * std).to(dt)[offset:] for e in sizes]

    return normal(0.5, dtype), normal(0.02, grad), normal(0.01, torch.float32), \
        [t.square() for t in normal(0.02, torch.float32)]


SIZES = [1, 3, 255, 256, 257, 1024, 4097, 100003]
# Sums and products in 32 bits: a handful of roundings of what is added.
E = 2.0 ** -22


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "bf16 f32g", "master bf16", "master f16"])
def test_32_bit_states(env, kind, offset):
    oz, torch = env
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind.split()[-1].replace("f32g", "bf16")]
    gt = torch.float32 if "f32g" in kind else dt
    p, g, m, v = tensors(torch, SIZES, dt, gt, 1, offset)
    master = [torch.zeros(e + offset, device="cuda")[offset:].copy_(a) for e, a in zip(SIZES, p)] if "master" in kind else None
    plan = oz.oz2_adamw_plan(p, g, m, v, masters=master)
    for t in (1, 2, 7):
        old = [(master or p)[i].clone() for i in range(len(SIZES))]
        want = [step64(torch, old[i], g[i], m[i], v[i], t, **HYPER) for i in range(len(SIZES))]
        oz.oz2_adamw(plan, step=t, **HYPER)
        for i, (_, wm, wv, _) in enumerate(want):
            wp, u = weight64(torch, old[i], m[i], v[i], t, **HYPER)
            bound = 4 * E * (wp.abs() + HYPER["lr"] * u.abs()) + 1e-30
            if master:
                close(torch, master[i], wp, bound, "master")
                assert torch.equal(p[i], master[i].to(dt))
            else:
                r = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dt]
                close(torch, p[i], wp, bound + r * wp.abs() + (2.0 ** -25 if dt == torch.float16 else 0), "param")
            close(torch, m[i], wm, E * (wm.abs() + g[i].double().abs()) + 1e-38, "m")
            close(torch, v[i], wv, E * (wv.abs() + g[i].double() ** 2) + 1e-38, "v")


def test_factors_of_a_tensor_and_of_the_gradients(env):
    oz, torch = env
    p, g, m, v = tensors(torch, [300, 301, 302], torch.float32, torch.float32, 2)
    want = []
    c = 0.37
    old, hs = [a.clone() for a in p], []
    for i, (ls, ds) in enumerate(((1.0, 1.0), (0.5, 0.0), (2.0, 3.0))):
        h = dict(HYPER, lr=HYPER["lr"] * ls, weight_decay=HYPER["weight_decay"] * ds)
        want.append(step64(torch, p[i], g[i].double() * float(torch.tensor(c)), m[i], v[i], 4, **h))
        hs.append(h)
    plan = oz.oz2_adamw_plan(p, g, m, v, lr_scales=[1.0, 0.5, 2.0], decay_scales=[1.0, 0.0, 3.0])
    oz.oz2_adamw(plan, step=4, grad_scale=torch.tensor([c], device="cuda"), **HYPER)
    for i, (_, wm, wv, _) in enumerate(want):
        wp, u = weight64(torch, old[i], m[i], v[i], 4, **hs[i])
        close(torch, p[i], wp, 4 * E * (wp.abs() + 2 * HYPER["lr"] * u.abs()), "param")
        close(torch, m[i], wm, E * (wm.abs() + g[i].double().abs()), "m")


def test_more_tensors_than_a_launch_takes(env):
    """700 tensors, some empty; the 8-bit rounding goes by the place in the whole list."""
    oz, torch = env
    sizes = [(i * 37) % 513 for i in range(700)]
    p, g, m, v = tensors(torch, sizes, torch.float32, torch.float32, 3)
    old = [a.clone() for a in p]
    want = [step64(torch, p[i], g[i], m[i], v[i], 2, **HYPER) for i in range(700)]
    oz.oz2_adamw(oz.oz2_adamw_plan(p, g, m, v), step=2, **HYPER)
    for i, (_, wm, _, _) in enumerate(want):
        close(torch, m[i], wm, E * (wm.abs() + g[i].double().abs()), i)
        wp, u = weight64(torch, old[i], m[i], v[i], 2, **HYPER)
        close(torch, p[i], wp, 4 * E * (wp.abs() + HYPER["lr"] * u.abs()), i)
    check_8bit(oz, torch, sizes, torch.float32, torch.float32, seed=4, steps=2)


# ---------------------------------------------------------------- 8 bits
MASK = 0xFFFFFFFF


def scatter(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & MASK
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & MASK
    return x ^ (x >> 16)


def rounding_bits(torch, seed, t, first_block, count):
    key = scatter((scatter(seed) + t) & MASK)
    at = torch.arange(count, device="cuda", dtype=torch.int64) + first_block * BLOCK
    h = scatter((at * 0x9E3779B1 + (at >> 32) * 0x3C6EF372 + key) & MASK)
    return h & 0xFFFF, h >> 16


def encode(torch, x, u):
    """(E4M3 codes as float8, scales) of float32 values, from the definition: the
    neighbours below and above in magnitude, up where u/65536 is at least the
    lower one's share, all in exact 64-bit arithmetic."""
    e = x.numel()
    rows = (e + BLOCK - 1) // BLOCK
    b = torch.zeros(rows * BLOCK, dtype=torch.float64, device=x.device)
    b[:e] = x.double()
    fin = torch.where(torch.isfinite(b), b, torch.zeros_like(b)).view(rows, BLOCK)
    top = fin.abs().amax(1)
    mant, ex = torch.frexp(top)
    ex = torch.where(mant > 0.875, ex - 8, ex - 9).clamp_min(-126)
    scale = torch.where(top > 0, pow2(torch, ex), torch.ones_like(top))
    q = (b.view(rows, BLOCK) / scale[:, None]).view(-1)[:e]
    a = torch.where(torch.isfinite(q), q, torch.zeros_like(q)).abs()
    _, ex = torch.frexp(a.clamp_min(2.0 ** -6))
    spacing = pow2(torch, ex - 4)
    # Below 2^-6 the kernel adds 2^-6 in float32, which rounds at 2^-29.
    a = torch.where(a < 2.0 ** -6, ((a.float() + 2.0 ** -6).double() - 2.0 ** -6), a)
    units = a / spacing
    low = units.floor()
    cut = ((units - low) * 65536).floor()  # what is cut off, to 16 bits and below
    up = (cut + u) >= 65536
    val = (low + up) * spacing
    code = val.float().to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(code.view(torch.float8_e4m3fn).double(), val)
    code = torch.where(torch.isfinite(q), code, torch.full_like(code, 0x7F))
    sign = (x.view(torch.int32) < 0)
    code = torch.where(sign, code | 0x80, code)
    return code, scale.float()


def check_8bit(oz, torch, sizes, dt, gt, seed, steps, offset=0, master=False, poke=None):
    p, g, _, _ = tensors(torch, sizes, dt, gt, seed, offset)
    masters = [a.float() for a in p] if master else None
    st = oz.oz2_adamw_states(p, bits=8)
    plan = oz.oz2_adamw_plan(p, g, masters=masters, **st)
    h = HYPER
    f = lambda c: torch.tensor(c, dtype=torch.float32, device="cuda")  # noqa: E731
    for t in range(1, steps + 1):
        for i, a in enumerate(g):
            a.copy_(torch.randn(a.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(97 * t + i)) * 0.02)
            if poke:
                poke(i, a, t)
        old = [((masters[i] if master else p[i]).float().clone(), st["m"][i].float(), st["v"][i].float(),
                st["m_scales"][i].clone(), st["v_scales"][i].clone()) for i in range(len(sizes))]
        oz.oz2_adamw(plan, step=t, seed=12345, **h)
        block = 0
        for i, e in enumerate(sizes):
            if e == 0:
                continue
            w, m, s, ms, ss = old[i]
            rep = lambda a: a.repeat_interleave(BLOCK)[:e]  # noqa: E731
            m = m * rep(ms)
            v = (s * rep(ss)).square()
            gg = g[i].float()
            m = m * f(h["beta1"]) + gg * f(1 - h["beta1"])
            v = v * f(h["beta2"]) + gg.square() * f(1 - h["beta2"])
            root = v.sqrt()
            um, uv = rounding_bits(torch, 12345, t, block, e)
            for got, scales, x, u, what in ((st["m"][i], st["m_scales"][i], m, um, "m"),
                                            (st["v"][i], st["v_scales"][i], root, uv, "v")):
                code, scale = encode(torch, x, u)
                assert torch.equal(scales, scale), (what, i, t)
                assert torch.equal(got.view(torch.uint8), code), (what, i, t)
            wp, upd = weight64(torch, w, m, v, t, **h)
            now = masters[i] if master else p[i]
            r = 0.0 if now.dtype == torch.float32 else 2.0 ** -8
            bound = 8 * E * (wp.abs() + h["lr"] * upd.abs()) + r * wp.abs() + 1e-30
            fin = torch.isfinite(wp)
            close(torch, now[fin], wp[fin], bound[fin], "w")
            assert torch.equal(torch.isnan(now), torch.isnan(wp))
            if master:
                keep = torch.isfinite(masters[i])
                assert torch.equal(p[i][keep], masters[i].to(dt)[keep])
            block += (e + BLOCK - 1) // BLOCK


@pytest.mark.parametrize("offset", [0, 1, 2])
@pytest.mark.parametrize("kind", ["f32", "bf16", "master bf16"])
def test_8_bit_states(env, kind, offset):
    oz, torch = env
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    check_8bit(oz, torch, SIZES, dt, dt, seed=5, steps=4, offset=offset, master="master" in kind)


def test_8_bit_extremes(env):
    """Blocks of zeros, of one large value among tiny ones, of tiny ones only,
    and of values that are not finite."""
    oz, torch = env

    def poke(i, a, t):
        if i == 0:
            a.zero_()
        if i == 1:
            a.mul_(1e-6)
            a[::256] = 50.0
        if i == 2:
            a.mul_(1e-17)
        if i == 3 and t == 2:
            a[5] = float("inf")
            a[300] = float("nan")
            a[301] = -float("inf")

    check_8bit(oz, torch, [600, 600, 600, 600, 256], torch.float32, torch.float32, seed=6, steps=4, poke=poke)


def test_8_bit_rounding_is_unbiased(env):
    """The mean over seeds of a state is the unrounded one: within 5 deviations of
    a mean of N values that are each off by up to a spacing s (variance ≤ s²/4)."""
    oz, torch = env
    e, seeds = 256, 400
    g = torch.randn(e, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)) * 0.02
    total = torch.zeros(e, dtype=torch.float64, device="cuda")
    for s in range(seeds):
        p = [torch.zeros(e, device="cuda")]
        st = oz.oz2_adamw_states(p, bits=8)
        oz.oz2_adamw(oz.oz2_adamw_plan(p, [g], **st), step=1, seed=s, **HYPER)
        total += st["m"][0].double() * st["m_scales"][0].double()
    scale = st["m_scales"][0].double()
    want = 0.1 * g.double()
    spacing = pow2(torch, torch.frexp((want.abs() / scale).clamp_min(2.0 ** -6))[1] - 4) * scale
    dev = spacing / 2 / math.sqrt(seeds)
    assert ((total / seeds - want).abs() <= 5 * dev + spacing * 2.0 ** -15).all()


def test_repeats_bit_for_bit_and_on_another_stream(env):
    oz, torch = env
    outs = []
    for use in (None, torch.cuda.Stream()):
        p, g, _, _ = tensors(torch, SIZES, torch.bfloat16, torch.bfloat16, 8)
        st = oz.oz2_adamw_states(p, bits=8)
        plan = oz.oz2_adamw_plan(p, g, **st)
        torch.cuda.synchronize()
        with torch.cuda.stream(use or torch.cuda.current_stream()):
            for t in (1, 2, 3):
                oz.oz2_adamw(plan, step=t, seed=3, **HYPER)
        torch.cuda.synchronize()
        outs.append([a.clone() for a in p] + [a.view(torch.uint8).clone() for a in st["m"] + st["v"]])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_masters_for_some_of_the_tensors(env):
    """A list in which every other tensor has a master: two launches, one numbering."""
    oz, torch = env
    sizes = [700, 256, 513, 9]
    outs = []
    for mixed in (False, True):
        p, g, _, _ = tensors(torch, sizes, torch.bfloat16, torch.bfloat16, 11)
        st = oz.oz2_adamw_states(p, bits=8)
        plan = oz.oz2_adamw_plan(p, g, **st)
        masters = [a.float() for a in p]
        if mixed:
            for i in (1, 3):
                plan.tensors[i].master = masters[i].data_ptr()
        for t in (1, 2):
            oz.oz2_adamw(plan, step=t, seed=3, **HYPER)
        outs.append((p, masters, [a.view(torch.uint8) for a in st["m"] + st["v"]]))
    assert all(torch.equal(a, b) for a, b in zip(outs[0][2], outs[1][2]))
    assert torch.equal(outs[0][0][0], outs[1][0][0]) and torch.equal(outs[0][0][2], outs[1][0][2])
    for i in (1, 3):
        assert torch.equal(outs[1][0][i], outs[1][1][i].to(torch.bfloat16))
