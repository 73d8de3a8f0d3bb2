"""The formulas of the operators at a language model's ends in 64 bits, and how far a
result may be from them.

Bounds are derived, not fitted; u = 2^-24 is a rounding of FP32, U[type] of the result.
A sum of c terms in `steps` additions one after another is off by at most steps·u·Σ|terms|.
"""
import torch

from layers_ref import D, TINY, U, sum_error

u = 2.0 ** -24


def rounded(v, e, t):
    """Bound of a result of type t whose FP32 value is within e of v."""
    return e + U[t] * (v.abs() + e) + TINY[t]


# --- embedding -------------------------------------------------------------------------
def embedding(ids, table, scale):
    ids = ids.long()
    n = table.shape[0]
    y = table.to(D)[ids.clamp(0, n - 1)] * scale * (ids >= 0)[:, None]
    y[ids >= n] = float("nan")
    return y, rounded(y, u * y.abs(), table.dtype)


def embedding_grad(dy, ids, n, scale, out_dtype, old=None):
    ids = ids.long()
    there = (ids >= 0) & (ids < n)
    t = dy.to(D)[there]
    s = torch.zeros(n, dy.shape[1], dtype=D, device=dy.device).index_add_(0, ids[there], t)
    a = torch.zeros_like(s).index_add_(0, ids[there], t.abs())
    c = torch.zeros(n, dtype=D, device=dy.device).index_add_(0, ids[there], torch.ones_like(ids[there], dtype=D))
    e = abs(scale) * u * ((c[:, None] + 1) * a)
    s = s * scale
    if old is not None:
        hit = (c > 0)[:, None]
        s = s + old.to(D)
        return s, torch.where(hit, rounded(s, e + u * s.abs(), out_dtype), torch.zeros_like(s))
    return s, torch.where((c > 0)[:, None], rounded(s, e, out_dtype), torch.zeros_like(s))


# --- layer norm -------------------------------------------------------------------------
def row_steps(k):
    """Additions one after another in a row's sum: a thread's own 32 values (or its share of a
    long row among 512), 10 levels of joining them."""
    return max(32, k / 512 + 8) + 12


def layer_norm(x, weight, bias, eps, center):
    """(y, mean, rstd), (their bounds)"""
    X, k = x.to(D), x.shape[1]
    st = row_steps(k)
    mean = X.mean(1, keepdim=True) if center else torch.zeros(x.shape[0], 1, dtype=D, device=x.device)
    em = (st * u * X.abs().mean(1, keepdim=True) + 2 * u * mean.abs()) if center else mean
    d = X - mean
    ed = em + u * d.abs()
    var = (d * d).mean(1, keepdim=True)
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (st + 3) * u * var
    rstd = 1 / torch.sqrt(var + eps)
    low = (var - ev).clamp_min(0) + eps  # what its root is taken of lies between these
    er = (1 / torch.sqrt(low * (1 - 4 * u)) - 1 / torch.sqrt((var + ev + eps) * (1 + 4 * u))) + 4 * u * rstd
    h = d * rstd
    eh = ed * (rstd + er) + d.abs() * er + u * h.abs()
    W = weight.to(D) if weight is not None else torch.ones(k, dtype=D, device=x.device)
    B = bias.to(D) if bias is not None else torch.zeros(k, dtype=D, device=x.device)
    y = h * W + B
    ey = eh * W.abs() + 3 * u * ((h * W).abs() + B.abs())
    return (y, mean[:, 0], rstd[:, 0]), (rounded(y, ey, x.dtype), em[:, 0] + 2 ** -140, er[:, 0] + u * rstd[:, 0])


def layer_norm_grad(dy, x, mean, rstd, weight, residual):
    """((dx, dw, db), (bounds)) from the FP32 mean (or None) and rstd."""
    m, k = x.shape
    st = row_steps(k)
    X, G, r = x.to(D), dy.to(D), rstd.to(D)[:, None]
    d = X - mean.to(D)[:, None] if mean is not None else X
    h = d * r
    eh = 3 * u * h.abs()
    W = weight.to(D) if weight is not None else torch.ones(k, dtype=D, device=x.device)
    g = G * W
    along = (g * h).mean(1, keepdim=True)
    ea = ((st + 8) * u * (g * h).abs()).mean(1, keepdim=True)
    level = g.mean(1, keepdim=True) if mean is not None else torch.zeros_like(along)
    el = ((st + 4) * u * g.abs()).mean(1, keepdim=True) if mean is not None else level
    dx = r * (g - level - h * along)
    ex = r * (5 * u * (g.abs() + level.abs() + (h * along).abs()) + el + h.abs() * ea + eh * along.abs())
    if residual is not None:
        dx = dx + residual.to(D)
        ex = ex + u * dx.abs()
    steps = m / 152 + 110  # a group's rows, its block's groups, the blocks
    dw, db = (G * h).sum(0), G.sum(0)
    ew = (steps + 5) * u * (G * h).abs().sum(0)
    eb = steps * u * G.abs().sum(0)
    return (dx, dw, db), (rounded(dx, ex, x.dtype), ew + 2.0 ** -126, eb + 2.0 ** -126)


# --- losses over a vocabulary -------------------------------------------------------------
def logits(x, w, scale):
    """z and the bound of its error."""
    X, W = x.to(D), w.to(D)
    z = scale * (X @ W.t())
    return z, abs(scale) * sum_error(X, W, x.shape[1]) + 2 * u * z.abs()


def lse_of(z, ez):
    """lse and its bound.  Off by no more than the logits; by exp2 (2^-22 and half a step of its
    argument: Σ p·log2(1/p) ≤ log2 n ≤ 17 with what the maximum adds), by its sums and joins (a
    rescaling of 2^-21 each) and by the logarithm."""
    lse = torch.logsumexp(z, 1)
    n = z.shape[1]
    e = (ez + 3 * u * z.abs()).amax(1) + 2.0 ** -19 + (n / 2048 + 50) * 2.0 ** -21 + 2.0 ** -22 * (1 + lse.abs())
    return lse, e


def xent(x, w, targets, scale=1.0, z_loss=0.0):
    """(loss, lse, picked), (bounds)"""
    z, ez = logits(x, w, scale)
    n = w.shape[0]
    lse, el = lse_of(z, ez)
    t = targets.long()
    at = t.clamp(0, n - 1)[:, None]
    picked, ep = z.gather(1, at)[:, 0], ez.gather(1, at)[:, 0]
    loss = lse - picked + z_loss * lse * lse
    e = el * (1 + 2 * z_loss * lse.abs() + z_loss * el) + ep + 4 * u * (lse.abs() + picked.abs() + z_loss * lse * lse) + 2 ** -140
    for v in (loss, picked, e, ep):
        v[t < 0] = 0
    loss[t >= n] = picked[t >= n] = float("nan")
    return (loss, lse, picked), (e, el, ep + 2 ** -140)


def teacher(ids, logits_, temperature, n):
    """(q, its relative bound, listed)."""
    there = ids >= 0
    U_ = (logits_.to(D) / temperature).masked_fill(~there, -float("inf"))
    q = torch.nan_to_num(torch.softmax(U_, 1), nan=0.0)
    size = U_.masked_fill(~there, 0).abs().amax(1, keepdim=True)
    return q, 8 * u * size + 2.0 ** -20, there


def distill(x, w, ids, logits_, temperature):
    z, ez = logits(x, w, 1 / temperature)
    ez = ez + 2 * u * z.abs()  # 1/temperature in FP32
    n = w.shape[0]
    lse, el = lse_of(z, ez)
    ids = ids.long()
    q, rq, there = teacher(ids, logits_, temperature, n)
    at = ids.clamp(0, n - 1)
    picked, ep = z.gather(1, at) * there, ez.gather(1, at) * there
    log_q = torch.where(q > 0, q.clamp_min(1e-300).log(), torch.zeros_like(q))
    loss = (q * (log_q - picked)).sum(1) + lse
    top = ids.shape[1]
    e = (q * (rq * (1 + log_q.abs() + picked.abs()) * 2 + ep + (top / 32 + 10) * u * (log_q.abs() + picked.abs()))).sum(1) + \
        el + 2 * u * (lse.abs() + loss.abs())
    live = there.any(1)
    loss, e = loss * live, e * live
    over = ids >= n
    picked[over] = float("nan")
    loss[over.any(1)] = float("nan")
    return (loss, lse, picked), (e, el, ep + 2 ** -140)


def head_grad(dz, edz, x, w, dw_dtype, live, old=None):
    """dX and dW of dz (and what it may be off by), rounded to x's type before the products."""
    dt = x.dtype
    edz = edz * live[:, None]
    dz = dz * live[:, None]
    tiny = 2.0 ** -38 * dz.abs().max() if dt == torch.float16 else TINY[dt]
    er = edz + U[dt] * (dz.abs() + edz) + tiny
    X, W = torch.nan_to_num(x.to(D)) * live[:, None], w.to(D)
    dx, dw = dz @ W, dz.t() @ X
    a = dz.abs() + er
    # (Pieces of the vocabulary are added up in FP32, another step each.)
    bx = rounded(dx, er @ W.abs() + 2 * sum_error(a, W.t().contiguous(), w.shape[0]), dt)
    ew = er.t() @ X.abs() + 2 * sum_error(a.t().contiguous(), X.t().contiguous(), x.shape[0])
    if old is not None:
        dw = dw + old.to(D)
        ew = ew + u * dw.abs()
    return (dx, dw), (bx * live[:, None], rounded(dw, ew, dw_dtype))


def _probabilities(x, w, scale, lse):
    z, ez = logits(x, w, scale)
    L = lse.to(D)[:, None]
    p = torch.exp(z - L)
    return p, ez + 4 * u * (z.abs() + L.abs() + (z - L).abs()) + 2.0 ** -20


def xent_grad(dloss, x, w, targets, lse, scale=1.0, z_loss=0.0, dw_dtype=None, old=None):
    t = targets.long()
    live = t >= 0
    x = torch.where(live[:, None], x, torch.zeros_like(x))
    p, rp = _probabilities(x, w, scale, torch.where(live, lse, torch.zeros_like(lse)))
    a = torch.where(live, dloss.to(D) * scale, torch.zeros_like(dloss, dtype=D))[:, None]
    e = 2 * z_loss * torch.where(live, lse, torch.zeros_like(lse)).to(D)[:, None]
    hot = torch.zeros_like(p).scatter_(1, t.clamp_min(0)[:, None], 1.0) * live[:, None]
    dz = a * ((1 + e) * p - hot)
    err = a.abs() * (1 + e.abs()) * p * rp * 1.1 + 8 * u * (dz.abs() + a.abs() * e.abs())
    return head_grad(dz, err, x, w, dw_dtype or x.dtype, live, old)


def distill_grad(dloss, x, w, ids, logits_, lse, temperature, dw_dtype=None, old=None):
    n = w.shape[0]
    ids = ids.long()
    q, rq, there = teacher(ids, logits_, temperature, n)
    live = there.any(1)
    x = torch.where(live[:, None], x, torch.zeros_like(x))
    p, rp = _probabilities(x, w, 1 / temperature, torch.where(live, lse, torch.zeros_like(lse)))
    rp = rp + 4 * u * (p.clamp_min(1e-300).log().abs() + lse.to(D).abs()[:, None])
    a = torch.where(live, dloss.to(D) / temperature, torch.zeros_like(dloss, dtype=D))[:, None]
    hot = torch.zeros_like(p).scatter_add_(1, ids.clamp_min(0), q)
    dz = a * (p - hot)
    count = ids.shape[1]
    err = a.abs() * (p * rp * 1.1 + hot * (rq + count * u)) + 8 * u * (dz.abs() + a.abs() * (p + hot))
    return head_grad(dz, err, x, w, dw_dtype or x.dtype, live, old)
