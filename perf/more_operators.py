"""What the operators at the two ends of a language model's training step, and
the norm between its layers, are measured on: embedding lookup, layer norm,
cross entropy over a vocabulary and distillation from a teacher's top logits
(both from the last layer's input and the head's weights, without keeping the
logits), each with its gradient.

A case is a dict of plain values.  `op` says which operator, `grad` whether its
gradient; m tokens, n rows of the vocabulary, k features, `type` of the matrices:

  "embedding"   y_t = scale·table[ids_t], zeros where ids_t < 0; the gradient of
                the table, or added to one that is there (`accumulate`)
  "norm"        y = (x - mean)·rstd·weight + bias, without the mean where not
                `center`; the gradient with that of a skip connection added to dx
                (`residual`)
  "xent"        z = scale·x·wᵀ; loss_t = lse_t - z_t,target + z_loss·lse_t², lse_t =
                log Σ_j exp z_tj; targets below 0 do not count (`masked`: some)
  "distill"     z = x·wᵀ / temperature; q = softmax(teacher / temperature) over a
                token's `top` listed rows (below 0: none there; `masked`: some);
                loss_t = Σ q·(log q - z_t,id) + lse_t
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5


# ---------------------------------------------------------------- cases
def _named(c, name):
    return {**c, "name": name} if name else c


def _embedding(m, n, k, type, grad, scale=1.0, masked=False, accumulate=False, name=None):
    return _named({"op": "embedding", "m": m, "n": n, "k": k, "type": type, "grad": grad, "scale": scale,
                   "masked": masked, "accumulate": accumulate}, name)


def _norm(m, k, type, grad, center=True, affine=True, residual=False, name=None):
    return _named({"op": "norm", "m": m, "k": k, "type": type, "grad": grad, "center": center, "affine": affine,
                   "residual": residual}, name)


def _xent(m, n, k, type, grad, scale=1.0, z_loss=0.0, masked=False, name=None):
    return _named({"op": "xent", "m": m, "n": n, "k": k, "type": type, "grad": grad, "scale": scale, "z_loss": z_loss,
                   "masked": masked}, name)


def _distill(m, n, k, top, type, grad, temperature=1.0, masked=False, name=None):
    return _named({"op": "distill", "m": m, "n": n, "k": k, "top": top, "type": type, "grad": grad,
                   "temperature": temperature, "masked": masked}, name)


def listed():
    return [
        # The tokens of 64 requests being decoded: latency.
        _embedding(64, 50257, 4096, "bf16", False, scale=64.0, name="embedding_decode_64"),
        # The table's gradient in a training step; a few padded places.
        _embedding(16384, 50257, 1024, "bf16", True, masked=True, name="embedding_grad_train"),
        # A table that is the head's weights too: its gradient is added to the
        # head's, in 32 bits, over many tokens.
        _embedding(65536, 131072, 2048, "f32", True, scale=0.5, accumulate=True, name="embedding_grad_tied"),
        # The same 64 requests' norm before a layer.
        _norm(64, 4096, "bf16", False, name="norm_decode_64"),
        # The gradient at odd sizes, rows off the 16-byte grid.
        _norm(1000, 777, "f16", True, name="norm_grad_ragged_1000x777"),
        # The gradient in a training step, with the skip connection's.
        _norm(16384, 4096, "bf16", True, residual=True, name="norm_grad_train"),
        # The loss of a small model, or of the last short batch: odd sizes.
        _xent(300, 1003, 256, "f16", False, masked=True, name="xent_small"),
        # The loss of a training step of a model of width 1024.
        _xent(4096, 50257, 1024, "bf16", False, z_loss=1e-4, masked=True, name="xent_train"),
        # Its gradient.
        _xent(4096, 50257, 1024, "bf16", True, z_loss=1e-4, masked=True, name="xent_grad_train"),
        # The gradient of a large batch over a large vocabulary: logits of 32
        # bits would be 4 GB.
        _xent(8192, 131072, 2048, "bf16", True, name="xent_grad_large"),
        # A small model that learns from a larger one's 64 top logits.
        _distill(4096, 50257, 1024, 64, "bf16", False, temperature=2.0, name="distill_train"),
        # The gradient with ragged lists, some of them empty, at odd sizes.
        _distill(1111, 32003, 1000, 33, "f16", True, temperature=1.5, masked=True, name="distill_grad_ragged"),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]; a third of them as they
    fall (odd ones too), the others multiples of 8 or 64, as layers have."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice((1, 8, 64))
    return max(lo, min(hi, int(round(v / step)) * step or step))


def draw(rng):
    op = rng.choice(("embedding", "norm", "xent", "distill"))
    grad = rng.random() < 0.6
    kind = rng.choice(("bf16", "f16"))
    masked = rng.random() < 0.5
    if op == "embedding":
        kind = rng.choice(("bf16", "f16", "f32"))
        while True:
            m, n, k = _size(rng, 1, 65536), _size(rng, 64, 131072), _size(rng, 16, 8192)
            if m * k <= 65536 * 2048 and n * k <= 131072 * 2048:
                break
        return _embedding(m, n, k, kind, grad, rng.choice((1.0, 0.5, 32.0)), masked, grad and rng.random() < 0.5)
    if op == "norm":
        kind = rng.choice(("bf16", "f16", "f32"))
        while True:
            m, k = _size(rng, 1, 65536), _size(rng, 16, 16384)
            if m * k <= 16384 * 4096:
                break
        return _norm(m, k, kind, grad, rng.random() < 0.7, rng.random() < 0.8, grad and rng.random() < 0.5)
    while True:
        m, n, k = _size(rng, 1, 16384), _size(rng, 64, 131072), _size(rng, 64, 4096)
        if m * n * k <= 8192 * 131072 * 2048 // (1 if op == "xent" else 4) and m * n <= 8192 * 131072:
            break
    if op == "xent":
        return _xent(m, n, k, kind, grad, rng.choice((1.0, 1.0, 0.25)), rng.choice((0.0, 1e-4)), masked)
    return _distill(m, n, k, min(n, _size(rng, 1, 128)), kind, grad, rng.choice((1.0, 1.5, 4.0)), masked)


# ---------------------------------------------------------------- inputs
def _ids(gen, m, n):
    """Rows of a vocabulary as text has them: the j-th as often as 1/j."""
    u = torch.rand(m, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(n + 1)).long() - 1).clamp(0, n - 1)


def _none_some(gen, ids, value, share=0.1):
    """The same with some of them not there."""
    gone = torch.rand(ids.shape, generator=gen, device="cuda") < share
    return torch.where(gone, torch.full_like(ids, value), ids)


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = TYPES[c["type"]]
    s = {"case": dict(c)}

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)

    if c["op"] == "embedding":
        m, n, k = c["m"], c["n"], c["k"]
        ids = _ids(gen, m, n)
        s["ids"] = _none_some(gen, ids, -1) if c["masked"] else ids
        if not c["grad"]:
            s["table"] = normal(n, k, std=0.02)
            return s
        s["dy"] = normal(m, k)
        s["table_grad"] = normal(n, k) if c["accumulate"] else None
        return s
    if c["op"] == "norm":
        m, k = c["m"], c["k"]
        s["x"] = (torch.randn((m, k), generator=gen, device="cuda") * 1.5 +
                  0.3 * torch.randn((m, 1), generator=gen, device="cuda")).to(dt)
        s["weight"] = (1 + 0.1 * torch.randn(k, generator=gen, device="cuda")).to(dt) if c["affine"] else None
        s["bias"] = normal(k, std=0.1) if c["affine"] and c["center"] else None
        if c["grad"]:
            x = s["x"].float()
            s["mean"] = x.mean(dim=1) if c["center"] else None
            if c["center"]:
                x = x - s["mean"][:, None]
            s["rstd"] = torch.rsqrt(x.square().mean(dim=1) + EPS)
            s["dy"] = normal(m, k)
            s["residual"] = normal(m, k) if c["residual"] else None
        return s
    # The head: tokens that a model is more or less sure of.
    m, n, k = c["m"], c["n"], c["k"]
    s["w"] = normal(n, k, std=2 * k ** -0.5)
    target = _ids(gen, m, n)
    sure = 4 * torch.rand((m, 1), generator=gen, device="cuda")
    s["x"] = (torch.randn((m, k), generator=gen, device="cuda") + sure * s["w"][target].float()).to(dt)
    if c["op"] == "xent":
        s["targets"] = _none_some(gen, target, -100) if c["masked"] else target
    else:  # the target and rows at even distances from it, the teacher's logits falling
        top = c["top"]
        step = torch.randint(1, n // top + 1, (m, 1), generator=gen, device="cuda")
        ids = (target[:, None] + step * torch.arange(top, device="cuda")) % n
        if c["masked"]:  # lists of 0 to `top` entries
            count = torch.randint(0, top + 1, (m, 1), generator=gen, device="cuda")
            ids = torch.where(torch.arange(top, device="cuda") < count, ids, torch.full_like(ids, -1))
        s["ids"] = ids
        s["teacher"] = (12 + 2 * torch.randn((m, top), generator=gen, device="cuda")).sort(dim=1, descending=True)[0]
    if c["grad"]:  # what the forward pass kept, and the mean's gradient (scaled, as 16-bit floats want it)
        z = _logits(s)
        s["lse"] = _lse(z)
        scale = 1024.0 if c["type"] == "f16" else 1.0
        s["dloss"] = scale / m * (0.5 + torch.rand(m, generator=gen, device="cuda"))
    return s


# ---------------------------------------------------------------- the plain forms
def _factor(c):
    return c["scale"] if c["op"] == "xent" else 1 / c["temperature"]


def _logits(s):
    return (s["x"].float() @ s["w"].float().t()) * _factor(s["case"])


def _lse(z):
    top = z.amax(dim=1)
    return top + torch.exp(z - top[:, None]).sum(dim=1).log()


def _picked(s, z):
    """The logits of the targets, or of the listed rows; 0 where there is none."""
    at = s["targets"][:, None] if s["case"]["op"] == "xent" else s["ids"]
    got = z.gather(1, at.clamp_min(0)) * (at >= 0)
    return got[:, 0] if s["case"]["op"] == "xent" else got


def _log_teacher(s):
    """(log q, q) with q = 0 where nothing is listed."""
    there = s["ids"] >= 0
    u = torch.where(there, s["teacher"] / s["case"]["temperature"], torch.full_like(s["teacher"], -1e30))
    top = u.amax(dim=1, keepdim=True)
    log_q = u - top - (torch.exp(u - top) * there).sum(dim=1, keepdim=True).clamp_min(1e-30).log()
    return torch.where(there, log_q, torch.zeros_like(log_q)), torch.exp(log_q) * there


def _plain_head(s):
    c = s["case"]
    z = _logits(s)
    lse = _lse(z)
    picked = _picked(s, z)
    if c["op"] == "xent":
        loss = (lse - picked + c["z_loss"] * lse.square()) * (s["targets"] >= 0)
    else:
        log_q, q = _log_teacher(s)
        loss = (q * (log_q - picked + lse[:, None])).sum(dim=1)
    return [loss, lse, picked]


def _plain_head_grad(s):
    c = s["case"]
    p = torch.exp(_logits(s) - s["lse"][:, None])
    g = s["dloss"] * _factor(c)
    if c["op"] == "xent":
        p = p * (1 + 2 * c["z_loss"] * s["lse"])[:, None]
        live = s["targets"] >= 0
        p.scatter_add_(1, s["targets"].clamp_min(0)[:, None], torch.full_like(p[:, :1], -1.0))
    else:
        live = (s["ids"] >= 0).any(dim=1)
        p.scatter_add_(1, s["ids"].clamp_min(0), -_log_teacher(s)[1])
    p = p * (g * live)[:, None]
    dt = s["x"].dtype
    return [(p @ s["w"].float()).to(dt), (p.t() @ s["x"].float()).to(dt)]


def _plain_embedding(s):
    c, ids = s["case"], s["ids"]
    there = (ids >= 0)[:, None]
    if not c["grad"]:
        y = s["table"][ids.clamp_min(0)].float() * c["scale"] * there
        return [y.to(s["table"].dtype)]
    dy = s["dy"].float() * c["scale"] * there
    if c["accumulate"]:
        total = s["table_grad"].float() if s["dy"].dtype != torch.float32 else s["table_grad"]
    else:
        total = torch.zeros((c["n"], c["k"]), device=dy.device)
    total.index_add_(0, ids.clamp_min(0), dy)
    if not c["accumulate"]:
        return [total.to(s["dy"].dtype)]
    s["table_grad"].copy_(total)
    return [s["table_grad"]]


def _plain_norm(s):
    c, x = s["case"], s["x"].float()
    mean = x.mean(dim=1) if c["center"] else None
    if c["center"]:
        x = x - mean[:, None]
    rstd = torch.rsqrt(x.square().mean(dim=1) + EPS)
    y = x * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return [y.to(s["x"].dtype), rstd] + ([mean] if c["center"] else [])


def _plain_norm_grad(s):
    c, dy, x = s["case"], s["dy"].float(), s["x"].float()
    if c["center"]:
        x = x - s["mean"][:, None]
    x = x * s["rstd"][:, None]
    out = [(dy * x).sum(dim=0), dy.sum(dim=0)]
    g = dy if s["weight"] is None else dy * s["weight"].float()
    dx = g - x * (g * x).mean(dim=1, keepdim=True)
    if c["center"]:
        dx = dx - g.mean(dim=1, keepdim=True)
    dx = dx * s["rstd"][:, None]
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return [dx.to(s["x"].dtype)] + (out[:1 + c["center"]] if c["affine"] else [])


# ---------------------------------------------------------------- one pass
def _own(s):
    import paper_2606_06510_gb300 as oz
    c = s["case"]
    if c["op"] == "embedding":
        if not c["grad"]:
            return [oz.oz2_embedding(s["ids"], s["table"], scale=c["scale"])]
        return [oz.oz2_embedding_grad(s["dy"], s["ids"], c["n"], scale=c["scale"], out=s["table_grad"],
                                      accumulate=c["accumulate"])]
    if c["op"] == "norm":
        if not c["grad"]:
            y, mean, rstd = oz.oz2_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, center=c["center"],
                                              save_stats=True)
            return [y, rstd] + ([mean] if c["center"] else [])
        need = ("dx", "dweight", "dbias")[:1 + c["affine"] * (1 + c["center"])]
        got = oz.oz2_layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], residual=s["residual"],
                                     need=need)
        return list(got[:len(need)])
    if c["op"] == "xent":
        if not c["grad"]:
            return list(oz.oz2_linear_xent(s["x"], s["w"], s["targets"], scale=c["scale"], z_loss=c["z_loss"]))
        return list(oz.oz2_linear_xent_grad(s["dloss"], s["x"], s["w"], s["targets"], s["lse"], scale=c["scale"],
                                            z_loss=c["z_loss"]))
    if not c["grad"]:
        return list(oz.oz2_linear_distill(s["x"], s["w"], s["ids"], s["teacher"], temperature=c["temperature"]))
    return list(oz.oz2_linear_distill_grad(s["dloss"], s["x"], s["w"], s["ids"], s["teacher"], s["lse"],
                                           temperature=c["temperature"]))


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "embedding":
        return _plain_embedding(state)
    if c["op"] == "norm":
        return _plain_norm_grad(state) if c["grad"] else _plain_norm(state)
    return _plain_head_grad(state) if c["grad"] else _plain_head(state)


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_embedding(s):
    c, d = s["case"], torch.float64
    used = s["ids"] >= 0
    if not c["grad"]:
        y = torch.zeros((c["m"], c["k"]), dtype=d, device="cuda")
        y[used] = c["scale"] * s["table"].to(d)[s["ids"][used]]
        return [y]
    # Sums of the rows that are there at all, then each to its place.
    out = s["table_grad"].to(d) if c["accumulate"] else torch.zeros((c["n"], c["k"]), dtype=d, device="cuda")
    rows, which = torch.unique(s["ids"][used], return_inverse=True)
    sums = torch.zeros((rows.numel(), c["k"]), dtype=d, device="cuda")
    sums.scatter_add_(0, which[:, None].expand(-1, c["k"]), s["dy"][used].to(d))
    out[rows] += c["scale"] * sums
    return [out]


def _exact_norm(s):
    c, d = s["case"], torch.float64
    x, k = s["x"].to(d), c["k"]
    one = torch.ones((k, 1), dtype=d, device="cuda")
    mu = x @ one / k if c["center"] else torch.zeros((c["m"], 1), dtype=d, device="cuda")
    var = ((x - mu) ** 2) @ one / k
    hat = (x - mu) / torch.sqrt(var + EPS)
    w = s["weight"].to(d) if s["weight"] is not None else one[:, 0]
    if not c["grad"]:
        y = hat * w
        if s["bias"] is not None:
            y = y + s["bias"].to(d)
        return [y, 1 / torch.sqrt(var[:, 0] + EPS)] + ([mu[:, 0]] if c["center"] else [])
    dy = s["dy"].to(d)
    ahead = dy * w
    along = (ahead * hat) @ one / k  # of the gradient, what lies along the row and along its mean
    level = ahead @ one / k if c["center"] else 0.0
    dx = (ahead - hat * along - level) / torch.sqrt(var + EPS)
    dx = dx + s["residual"].to(d) if c["residual"] else dx
    tokens = torch.ones((1, c["m"]), dtype=d, device="cuda")
    sums = [(tokens @ (dy * hat))[0], (tokens @ dy)[0]]
    return [dx] + (sums[:2 if c["center"] else 1] if c["affine"] else [])


def _exact_soft_targets(s):
    """The listed rows' weights as they are, and their logarithms."""
    u = s["teacher"].to(torch.float64) / s["case"]["temperature"]
    u = u.masked_fill(s["ids"] < 0, -math.inf)
    q = torch.nan_to_num(torch.softmax(u, dim=1), nan=0.0)  # an empty list has no weights
    return q, torch.xlogy(q, q)


def _exact_head(s):
    c, d = s["case"], torch.float64
    x, w = s["x"].to(d), s["w"].to(d)
    if c["op"] == "distill":
        x = x / c["temperature"]
    else:
        x = x * c["scale"]
    z = torch.matmul(x, w.transpose(0, 1))
    lse = torch.logsumexp(z, dim=1)
    if c["op"] == "xent":
        live = torch.nonzero(s["targets"] >= 0)[:, 0]
        y = s["targets"][live]
    else:
        q, q_log_q = _exact_soft_targets(s)
        live = torch.nonzero((s["ids"] >= 0).sum(dim=1) > 0)[:, 0]
    if not c["grad"]:
        loss = torch.zeros_like(lse)
        if c["op"] == "xent":
            picked = torch.zeros_like(lse)
            picked[live] = z[live, y]
            loss[live] = lse[live] - z[live, y] + c["z_loss"] * lse[live] ** 2
        else:
            picked = torch.where(s["ids"] >= 0, torch.gather(z, 1, s["ids"] * (s["ids"] >= 0)), 0.0 * q)
            loss[live] = (q_log_q.sum(dim=1) - (q * picked).sum(dim=1) + lse)[live]
        return [loss, lse, picked]
    z.sub_(lse[:, None]).exp_()
    if c["op"] == "xent":
        z.mul_(1 + 2 * c["z_loss"] * lse[:, None])
        z[live, y] -= 1
        factor = c["scale"]
    else:
        token = torch.arange(c["m"], device="cuda")[:, None].expand_as(s["ids"])
        listed_ = s["ids"] >= 0
        z.index_put_((token[listed_], s["ids"][listed_]), -q[listed_], accumulate=True)
        factor = 1 / c["temperature"]
    g = torch.zeros_like(lse)
    g[live] = s["dloss"].to(d)[live] * factor
    z.mul_(g[:, None])
    return [torch.matmul(z, w), torch.matmul(z.transpose(0, 1), s["x"].to(d))]


def exact(case, seed):
    if case["op"] in ("xent", "distill"):
        # At the measured rate of 64-bit products, some 1.2e12 operations a second.
        if (6.0 if case["grad"] else 2.0) * case["m"] * case["n"] * case["k"] > 1.5e13:
            return None
    s = prepare(case, seed)
    return {"embedding": _exact_embedding, "norm": _exact_norm, "xent": _exact_head, "distill": _exact_head}[case["op"]](s)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c, m, k, b = case, case["m"], case["k"], BYTES[case["type"]]
    if c["op"] == "embedding":
        if not c["grad"]:
            return {"bytes": 2.0 * b * m * k + 8 * m, "flops": 1.0 * m * k}
        # Added to: the rows that ids fall on (drawn as 1/j), read and written.
        n = c["n"]
        hit = n
        if c["accumulate"]:
            hit = sum(-math.expm1(m * math.log1p(-min(1 - 1e-12, math.log1p(1 / j) / math.log(n + 1))))
                      for j in range(1, n + 1))
        return {"bytes": b * k * (m + (2.0 * hit if c["accumulate"] else n)) + 8 * m, "flops": 1.0 * m * k}
    if c["op"] == "norm":
        if not c["grad"]:
            return {"bytes": 2.0 * b * m * k + 2 * b * k + 8 * m, "flops": 8.0 * m * k}
        return {"bytes": b * m * k * (3.0 + c["residual"]) + b * k + 8 * k + 8 * m, "flops": 15.0 * m * k}
    n = c["n"]
    beside = (8 + 12) * m if c["op"] == "xent" else (8 + 4 + 4) * m * c["top"] + 8 * m
    if not c["grad"]:
        return {"bytes": 2.0 * k * (m + n) + beside, "flops": 2.0 * m * n * k}
    return {"bytes": 4.0 * k * (m + n) + beside, "flops": 6.0 * m * n * k}
