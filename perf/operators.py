"""What the layer operators are measured on: a linear layer with its epilogue,
that layer's gradient, and the AdamW step that updates the weights.

A case is a dict of plain values.  `op` says which operator:

  "linear"  y = act(x·wᵀ + b) + r for m tokens: x (m, k), w (n, k); `type` of
            x and w ("bf16", "f16", or "e4m3" with a scale per token and per
            output; y is then bf16); `bias`, `residual`, `pre` (z = x·wᵀ + b
            is returned too, as training keeps it)
  "grad"    dx, dw and db of such a layer from dy, x, w and z
  "adamw"   one step over many tensors: the weights of `layers` blocks of
            width `width` (four width², two 4·width² matrices, six vectors
            each) and one tensor of `odd` elements; `param` and `grad` types,
            `master` (f32 weights beside 16-bit ones), `bits` of the states
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
BETA1, BETA2, EPS, LR, DECAY, STEP = 0.9, 0.999, 1e-8, 1e-3, 0.01, 10
BLOCK = 256  # values that share a scale in 8-bit states


# ---------------------------------------------------------------- cases
def _linear(m, n, k, type, act, bias=True, residual=False, pre=False, name=None):
    c = {"op": "linear", "m": m, "n": n, "k": k, "type": type, "act": act, "bias": bias, "residual": residual,
         "pre": pre}
    return {**c, "name": name} if name else c


def _grad(m, n, k, type, act, name=None):
    c = {"op": "grad", "m": m, "n": n, "k": k, "type": type, "act": act}
    return {**c, "name": name} if name else c


def _adamw(width, layers, odd, param, grad, master, bits, name=None):
    c = {"op": "adamw", "width": width, "layers": layers, "odd": odd, "param": param, "grad": grad, "master": master,
         "bits": bits}
    return {**c, "name": name} if name else c


def listed():
    return [
        # One token through a layer of a model being served: w's bytes, and latency.
        _linear(1, 4096, 4096, "bf16", "silu", residual=True, name="linear_token_4096"),
        # A batch of 16 requests decoding against a large matrix held in 8 bits.
        _linear(16, 16384, 16384, "e4m3", "none", bias=False, residual=True, name="linear_batch16_16384"),
        # A short prompt, sizes that no tile divides and rows that start off
        # the 16-byte grid.
        _linear(1000, 777, 1333, "f16", "gelu", residual=True, name="linear_ragged_1000x777x1333"),
        # The forward pass of a training step: z is kept for the gradient.
        _linear(4096, 4096, 4096, "bf16", "gelu_tanh", pre=True, name="linear_train_4096"),
        # A long prompt or a large training batch through a wide layer.
        _linear(16384, 16384, 4096, "bf16", "silu", residual=True, name="linear_wide_16384"),
        # The gradient of a small layer: launches and latency.
        _grad(256, 256, 256, "f16", "relu", name="grad_256"),
        # A gradient at odd sizes.
        _grad(2500, 3001, 2047, "bf16", "gelu", name="grad_ragged_2500x3001x2047"),
        # The gradient of the training step's layer.
        _grad(4096, 4096, 4096, "bf16", "gelu_tanh", name="grad_train_4096"),
        # Many tokens through a small projection: dw sums over a long axis.
        _grad(65536, 1024, 1024, "bf16", "none", name="grad_tallk_65536x1024"),
        # The step of a small model, f32 throughout: many small tensors.
        _adamw(64, 2, 1003, "f32", "f32", False, 32, name="adamw_small"),
        # A model trained in bf16 with f32 masters and states.
        _adamw(1024, 16, 50257, "bf16", "bf16", True, 32, name="adamw_master_32bit"),
        # The same with its states in 8 bits.
        _adamw(1024, 16, 50257, "bf16", "bf16", True, 8, name="adamw_master_8bit"),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]; a third of them as they
    fall (odd ones too), the others multiples of 8 or 64, as layers have."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice((1, 8, 64))
    v = max(lo, min(hi, int(round(v / step)) * step or step))
    return v + step if v == 3072 else v


def draw(rng):
    op = rng.choice(("linear", "linear", "grad", "adamw"))
    if op == "adamw":
        width = _size(rng, 64, 1024)
        width += 8 if width == 768 else 0
        layers = rng.randint(1, 16)
        param = rng.choice(("f32", "bf16", "f16"))
        grad = rng.choice(("f32", param))
        return _adamw(width, layers, _size(rng, 1, 50257), param, grad, param != "f32" and rng.random() < 0.7,
                      rng.choice((8, 32)))
    while True:
        m, n, k = _size(rng, 1, 16384), _size(rng, 64, 16384), _size(rng, 64, 16384)
        if m * n * k <= 16384 * 16384 * 4096 // (1 if op == "linear" else 2):
            break
    act = rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu"))
    if op == "grad":
        return _grad(m, n, k, rng.choice(("bf16", "f16")), act)
    return _linear(m, n, k, rng.choice(("bf16", "f16", "e4m3")), act, rng.random() < 0.7, rng.random() < 0.5,
                   rng.random() < 0.3)


def _places(case):
    """(start, size) of each tensor in flat buffers in which every tensor starts
    a block of BLOCK values, and the buffers' length."""
    w = case["width"]
    sizes = [w * w, w * w, w * w, w * w, 4 * w * w, 4 * w * w, w, w, w, w, w, 4 * w] * case["layers"] + [case["odd"]]
    places, at = [], 0
    for e in sizes:
        places.append((at, e))
        at += (e + BLOCK - 1) // BLOCK * BLOCK
    return places, at


# ---------------------------------------------------------------- inputs
def _normal(gen, shape, std, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _e4m3_rows(t):
    """Rows as E4M3 values and one scale each (the row's largest value at 448)."""
    scale = t.abs().amax(dim=1).clamp_min(1e-12) / 448
    return (t / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": dict(case)}
    if case["op"] == "adamw":
        places, total = _places(case)
        pt, gt = TYPES[case["param"]], TYPES[case["grad"]]
        used = torch.zeros(total, device="cuda")  # 0 between the tensors
        for at, e in places:
            used[at:at + e] = 1
        w = _normal(gen, (total,), 0.05, torch.float32) * used
        s["param"] = w.to(pt)
        s["master"] = w if case["master"] else None
        s["grad"] = _normal(gen, (total,), 0.01, torch.float32).mul_(used).to(gt)
        # States as some steps of such gradients leave them.
        m = _normal(gen, (total,), 0.004, torch.float32) * used
        v = (torch.randn(total, generator=gen, device="cuda") * 0.1 + 1).square() * 1e-6 * used
        s["m_scale"] = s["v_scale"] = None
        if case["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            s["m"], s["m_scale"] = _e4m3_blocks(m)
            s["v"], s["v_scale"] = _e4m3_blocks(v.sqrt())
        s["seed"] = int(seed) % (1 << 31)  # of the 8-bit states' rounding
        if own:  # the handle that a training program keeps: its tensors, as views of the buffers
            import paper_2606_06510_gb300 as oz

            def views(t, per=1):
                return None if t is None else [t[at // per:(at + e + per - 1) // per] for at, e in places]

            s["plan"] = oz.oz2_adamw_plan(views(s["param"]), views(s["grad"]), views(s["m"]), views(s["v"]),
                                          masters=views(s["master"]), m_scales=views(s["m_scale"], BLOCK),
                                          v_scales=views(s["v_scale"], BLOCK))
        return s
    m, n, k, dt = case["m"], case["n"], case["k"], TYPES[case["type"]]
    if case["type"] == "e4m3":
        s["x"], s["x_scale"] = _e4m3_rows(_normal(gen, (m, k), 1.0, torch.float32))
        s["w"], s["w_scale"] = _e4m3_rows(_normal(gen, (n, k), k ** -0.5, torch.float32))
        dt = torch.bfloat16
    else:
        s["x"], s["x_scale"] = _normal(gen, (m, k), 1.0, dt), None
        s["w"], s["w_scale"] = _normal(gen, (n, k), k ** -0.5, dt), None
    s["out"] = dt
    if case["op"] == "grad":
        s["dy"] = _normal(gen, (m, n), 1.0, dt)
        s["z"] = _normal(gen, (m, n), 1.0, dt) if case["act"] != "none" else None
        return s
    s["bias"] = _normal(gen, (n,), 0.5, dt) if case["bias"] else None
    s["residual"] = _normal(gen, (m, n), 1.0, dt) if case["residual"] else None
    return s


def _block_scales(t):
    """The power of two of each block (row) that brings its largest value to
    (224, 448]; 1 for a block of zeros."""
    top = t.abs().amax(dim=1)
    bits = top.view(torch.int32)
    e = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 254)
    return torch.where(top > 0, (e << 23).view(torch.float32), torch.ones_like(top))


def _e4m3_blocks(t):
    """f32 values as E4M3 ones, rounded to nearest, and their blocks' scales."""
    b = t.view(-1, BLOCK)
    scale = _block_scales(b)
    return (b / scale[:, None]).to(torch.float8_e4m3fn).view(-1), scale


# ---------------------------------------------------------------- the plain forms
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return g * (1 + z * (1 - g))
    return torch.ones_like(z)


def _plain_linear(s):
    c = s["case"]
    z = s["x"].float() @ s["w"].float().t()
    if s["x_scale"] is not None:
        z = z * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(s["out"])] + ([z.to(s["out"])] if c["pre"] else [])


def _plain_grad(s):
    c = s["case"]
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(s["z"].float(), c["act"])
    return [(dz @ s["w"].float()).to(s["out"]), (dz.t() @ s["x"].float()).to(s["out"]), dz.sum(dim=0)]


_MASK = 0xFFFFFFFF


def _mix(x):
    """32 bits scattered (of an int, or of an int64 tensor of values below 2^32)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & _MASK
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & _MASK
    return x ^ (x >> 16)


def _round_bits(seed, step, count, device):
    """Two 16-bit numbers for each value: what the roundings of its m and v go
    by.  Values are numbered through all tensors, each starting a block."""
    key = _mix((_mix(seed & _MASK) + step) & _MASK)
    at = torch.arange(count, device=device, dtype=torch.int64)
    h = _mix((at * 0x9E3779B1 + (at >> 32) * 0x3C6EF372 + key) & _MASK)
    return (h & 0xFFFF).int(), (h >> 16).int()


def _e4m3_stochastic(t, u):
    """f32 values of magnitude up to 448 as E4M3 ones: away from zero with the
    probability of what is cut off, which u (16 bits) is compared with."""
    a = t.abs()
    small = a < 2.0 ** -6
    b = torch.where(small, a + 2.0 ** -6, a).view(torch.int32)
    code = ((b + (u << 4)) >> 20) - (120 << 3) - 8 * small.int()
    code = code | torch.where(t < 0, 128, 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn)


def _plain_adamw(s):
    c = s["case"]
    p = (s["param"] if s["master"] is None else s["master"]).float()
    g, m, v = s["grad"].float(), s["m"].float(), s["v"].float()
    if c["bits"] == 8:  # v is kept as its square root
        m = (m.view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g.square() * (1 - BETA2)
    root = v.sqrt()
    p = p - (LR * DECAY) * p - (LR / (1 - BETA1 ** STEP)) * (m / (root / math.sqrt(1 - BETA2 ** STEP) + EPS))
    s["param"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    um, uv = _round_bits(s["seed"], STEP, m.numel(), m.device)
    for t, u, to, to_scale in ((m, um, s["m"], s["m_scale"]), (root, uv, s["v"], s["v_scale"])):
        scale = _block_scales(t.view(-1, BLOCK))
        to.copy_(_e4m3_stochastic((t.view(-1, BLOCK) / scale[:, None]).view(-1), u))
        to_scale.copy_(scale)


def _state(s):
    return [s[x] for x in ("param", "master", "m", "m_scale", "v", "v_scale") if s[x] is not None]


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2606_06510_gb300 as oz
        if c["op"] == "linear":
            y = oz.oz2_linear(s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["residual"],
                              x_scale=s["x_scale"], w_scale=s["w_scale"], save_pre=c["pre"])
            return list(y) if c["pre"] else [y]
        if c["op"] == "grad":
            return list(oz.oz2_linear_grad(s["dy"], s["x"], s["w"], pre=s["z"], act=c["act"]))
        oz.oz2_adamw(s["plan"], step=STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                     seed=s["seed"])
        return _state(s)
    if c["op"] == "linear":
        return _plain_linear(s)
    if c["op"] == "grad":
        return _plain_grad(s)
    _plain_adamw(s)
    return _state(s)


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _gauss_cdf(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _exact_act(z, act):
    """act(z) and its derivative."""
    one = torch.ones_like(z)
    if act == "none":
        return z, one
    if act == "relu":
        return torch.maximum(z, 0 * z), torch.where(z > 0, one, 0 * one)
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    if act == "gelu":
        return z * _gauss_cdf(z), _gauss_cdf(z) + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    # z·sigmoid(2u), the same as z·(1 + tanh u)/2
    u2 = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    q = torch.sigmoid(u2)
    return z * q, q + z * q * (1 - q) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z ** 2)


def _exact_linear(s):
    c, d = s["case"], torch.float64
    x, w = s["x"].to(d), s["w"].to(d)
    if c["type"] == "e4m3":
        x, w = x * s["x_scale"].to(d).unsqueeze(1), w * s["w_scale"].to(d).unsqueeze(1)
    z = torch.matmul(x, w.transpose(0, 1))
    z = z + s["bias"].to(d) if c["bias"] else z
    y = _exact_act(z, c["act"])[0]
    y = y + s["residual"].to(d) if c["residual"] else y
    return [y, z] if c["pre"] else [y]


def _exact_grad(s):
    d = torch.float64
    dz = s["dy"].to(d)
    if s["case"]["act"] != "none":
        dz = dz * _exact_act(s["z"].to(d), s["case"]["act"])[1]
    return [torch.matmul(dz, s["w"].to(d)), torch.matmul(dz.transpose(0, 1), s["x"].to(d)),
            torch.ones(dz.shape[0], dtype=d, device=dz.device) @ dz]


def _exact_states8(x, u):
    """The E4M3 code values (not scaled) and the scales of x: magnitudes cut to
    a multiple of their spacing, and one spacing more where u says so."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(dim=1, keepdim=True)
    top = torch.where(top > 0, top, torch.full_like(top, 448.0))
    scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp_min(-126))
    q = (b / scale).view(-1)
    # 8 values to a binade, never closer than 2^-9
    spacing = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
    units = q.abs() / spacing
    whole = torch.floor(units)
    up = (units - whole) + u.to(torch.float64) / 65536 >= 1
    return torch.sign(q) * (whole + up.to(torch.float64)) * spacing, scale.view(-1)


def _exact_adamw(s):
    c, d = s["case"], torch.float64
    p0 = (s["master"] if c["master"] else s["param"]).to(d)
    g, m, v = s["grad"].to(d), s["m"].to(d), s["v"].to(d)
    if c["bits"] == 8:
        m = m * s["m_scale"].to(d).repeat_interleave(BLOCK)
        v = (v * s["v_scale"].to(d).repeat_interleave(BLOCK)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    m_hat, v_hat = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
    p = p0 - LR * (m_hat / (torch.sqrt(v_hat) + EPS) + DECAY * p0)
    out = [p, p] if c["master"] else [p]
    if c["bits"] == 32:
        return out + [m, v]
    um, uv = _round_bits(s["seed"], STEP, m.numel(), m.device)
    return out + [*_exact_states8(m, um), *_exact_states8(torch.sqrt(v), uv)]


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "grad": _exact_grad, "adamw": _exact_adamw}[case["op"]](s)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "adamw":
        count = sum(e for _, e in _places(case)[0])
        p, g = BYTES[case["param"]], BYTES[case["grad"]]
        weights = 8 + p if case["master"] else 2 * p  # a master is read and written, its copy written
        states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": count * (g + weights + states), "flops": 15.0 * count}
    m, n, k, b = case["m"], case["n"], case["k"], BYTES[case["type"]]
    if case["op"] == "grad":
        z = b * m * n if case["act"] != "none" else 0
        return {"bytes": b * (m * n + 2 * m * k + 2 * n * k) + z + 4 * n, "flops": 4.0 * m * n * k}
    out = 1 + case["residual"] + case["pre"]
    extra = 4 * (m + n) if case["type"] == "e4m3" else 0
    return {"bytes": b * (m * k + n * k) + 2 * out * m * n + 2 * n * case["bias"] + extra, "flops": 2.0 * m * n * k}
