"""The layer operators' binding (include/oz2_layers.h): a linear layer with its
epilogue, that layer's gradient, and AdamW over many tensors.

Arrays are those of a PyTorch program, row-major: x (tokens, k), w (n, k),
y (tokens, n), with stride(1) == 1 and any row stride.  They are the C ABI's
column-major matrices with tokens as columns.  Row strides (and starts) that are
multiples of 16 bytes, 8 elements of 16 bits, are what the tensor cores' loads
want: other operands are copied to such rows first, but for weights that up to 16
tokens go through, which are mostly read where they lie; of two operands with rows on
odd multiples of 16 bytes, long products copy one.  A call runs on the current
stream, or on `stream`, whose memory its new outputs then are.
"""
from __future__ import annotations

import ctypes

import torch

ACT = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
TYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float8_e4m3fn: 3}
GRAD_ACCUMULATE = 0x1
ADAMW_BLOCK = 256

_I64, _P, _I, _U = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_uint


class oz2_adamw_tensor(ctypes.Structure):
    _fields_ = [("numel", _I64), ("param", _P), ("grad", _P), ("master", _P), ("m", _P), ("v", _P),
                ("m_scale", _P), ("v_scale", _P), ("lr_scale", ctypes.c_float), ("decay_scale", ctypes.c_float)]


class oz2_adamw_step(ctypes.Structure):
    _fields_ = [("step", _I64), ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("d_grad_scale", _P),
                ("seed", ctypes.c_uint32)]


SIGS = {
    "oz2_linear": (_I, [_I64, _I64, _I64, _I, _P, _I64, _P, _I64, _P, _P, _P, _I, _I, _P, _I64, _P, _I64, _P, _I64,
                        _I, _P]),
    "oz2_linear_grad": (_I, [_I64, _I64, _I64, _I, _P, _I64, _P, _I64, _I, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _I,
                             _P, _U, _P]),
    "oz2_adamw": (_I, [ctypes.POINTER(oz2_adamw_tensor), _I, _I, _I, _I, ctypes.POINTER(oz2_adamw_step), _P]),
}


# The C entry points by name, looked up on first use (an import inside each call is
# some 2 µs of it).
_ENTRIES = {}


def _entry(name):
    from . import lib
    f = _ENTRIES[name] = getattr(lib(), name)
    return f


def _done(code, what):
    if code:
        from . import Oz2Error
        raise Oz2Error(code, what)


def _stream():
    """The current stream (there is a CUDA tensor, so CUDA is up)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


# An output of its own is a good part of a small call's time: torch.empty takes 1.5 µs
# and, by what it drives out of the caches, 4 of the call; the allocation that PyTorch's
# own generated code makes takes a third of that.
_EMPTY = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)


def _new(like, shape, dtype, stream):
    """A contiguous output beside `like`, of the memory of the stream that writes it."""
    if stream is None:
        if _EMPTY is not None and like.get_device() == torch._C._cuda_getDevice():
            return _EMPTY(shape, (shape[1] or 1, 1) if len(shape) == 2 else (1,), dtype)
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _ld(t, rows, cols, what):
    """The row stride of a CUDA matrix of this shape."""
    assert t.is_cuda, f"{what}: oz2 operates on CUDA tensors"
    ld, one = t.stride()
    assert (one == 1 or cols <= 1) and (ld >= cols or rows <= 1), f"{what}: rows must be contiguous (stride(1) == 1)"
    return ld if rows > 1 and ld > 0 else cols or 1


def _rows(t, rows, cols, dtype, what):
    """(address, row stride) of a CUDA matrix of this shape and dtype."""
    assert t.shape == (rows, cols) and t.dtype == dtype, \
        f"{what}: expected shape ({rows}, {cols}) and {dtype}, got {tuple(t.shape)} and {t.dtype}"
    return t.data_ptr(), _ld(t, rows, cols, what)


def _vector(t, count, dtype, other, what):
    """The address of a contiguous CUDA vector of one of two dtypes."""
    dt = t.dtype
    assert (dt == dtype or dt == other) and t.is_cuda and t.shape == (count,) and t.is_contiguous(), \
        f"{what}: expected {count} contiguous values of {dtype} or {other} on the GPU"
    return t.data_ptr()


def oz2_linear(x, w, bias=None, act="none", residual=None, x_scale=None, w_scale=None, save_pre=False, out=None,
               out_dtype=None, stream=None):
    """act(x·wᵀ + bias) + residual for tokens x (m, k) and weights w (n, k).

    x and w: bfloat16, float16, or float8_e4m3fn with optional float32 scales
    x_scale (m,) and w_scale (n,), which multiply the products.  The result
    (m, n) has x's dtype, or out_dtype (bfloat16 by default) for E4M3; bias has
    the result's dtype or float32, residual the result's.  act: "none", "relu",
    "gelu", "gelu_tanh" or "silu".  With save_pre, returns (y, z) with z the
    activation's argument, which oz2_linear_grad wants.  `out` may be the
    residual itself, and overlaps neither x nor w.  No graph of gradients is recorded: tensors that require them
    are refused unless that is off (torch.no_grad()).
    """
    if x.requires_grad or w.requires_grad or (bias is not None and bias.requires_grad) or \
            (residual is not None and residual.requires_grad) or (x_scale is not None and x_scale.requires_grad) or \
            (w_scale is not None and w_scale.requires_grad):
        assert not torch.is_grad_enabled(), "a tensor requires its gradient, which would be lost: call oz2_linear " \
            "under torch.no_grad(), and oz2_linear_grad for the gradients"
    m, k = x.shape
    n, k2 = w.shape
    xt = dt = x.dtype
    assert k == k2 and w.dtype == xt, "x and w: expected (m, k) and (n, k) of one dtype"
    if xt == torch.float8_e4m3fn:
        dt = out_dtype or torch.bfloat16
    assert out_dtype is None or out_dtype == dt, "out_dtype: a 16-bit product has its operands' dtype"
    ldx, ldw = _ld(x, m, k, "x"), _ld(w, n, k, "w")
    if out is None:
        y, ldy = _new(x, (m, n), dt, stream), n or 1
        yp = y.data_ptr()
    else:
        y = out
        yp, ldy = _rows(y, m, n, dt, "out")
    z = zp = rp = bp = None
    ldr = bt = 0
    if save_pre:
        z = _new(x, (m, n), dt, stream)
        zp = z.data_ptr()
    if residual is not None:
        rp, ldr = _rows(residual, m, n, dt, "residual")
    if bias is not None:
        bp, bt = _vector(bias, n, dt, torch.float32, "bias"), TYPE[bias.dtype]
    xs = _vector(x_scale, m, torch.float32, torch.float32, "x_scale") if x_scale is not None else None
    ws = _vector(w_scale, n, torch.float32, torch.float32, "w_scale") if w_scale is not None else None
    _done((_ENTRIES.get("oz2_linear") or _entry("oz2_linear"))(
        m, n, k, TYPE.get(xt, -1), x.data_ptr(), ldx, w.data_ptr(), ldw, xs, ws, bp, bt, ACT[act], rp, ldr, zp, n or 1,
        yp, ldy, TYPE.get(dt, -1), _stream() if stream is None else stream.cuda_stream), "oz2_linear")
    return (y, z) if save_pre else y


def oz2_linear_grad(dy, x, w, pre=None, act="none", need=("dx", "dw", "db"), dx=None, dw=None, db=None,
                    dw_dtype=None, accumulate=False, stream=None):
    """(dx, dw, db) of oz2_linear from dy, its x and w, and the z it kept (pre).

    `need` names the gradients wanted (the others are None).  dx (m, k) has x's
    dtype, dw (n, k) that or float32, db (n,) float32; each may be given as the
    tensor to write.  With accumulate, dw (float32) and db are added to, and
    must be given.  The residual's gradient is dy itself.  The results have no graph of
    gradients of their own, whatever the arguments require.
    """
    m, n = dy.shape
    k = x.shape[1]
    dt = dy.dtype
    assert x.dtype == w.dtype == dt and x.shape[0] == m and w.shape == (n, k), \
        "dy, x and w: expected (m, n), (m, k) and (n, k) of one dtype"
    ldy, ldx, ldw = _ld(dy, m, n, "dy"), _ld(x, m, k, "x"), _ld(w, n, k, "w")
    ldz, zp = 1, None
    if act != "none":
        assert pre is not None, "pre: the activation's gradient wants the z that was kept"
        zp, ldz = _rows(pre, m, n, dt, "pre")
    assert not accumulate or (("dw" not in need or dw is not None) and ("db" not in need or db is not None)), \
        "accumulate: dw and db have to be given"
    xp = wp = bp = None
    lddx = lddw = k or 1
    wt = 0
    if "dx" not in need:
        dx = None
    elif dx is None:
        dx = _new(dy, (m, k), dt, stream)
        xp = dx.data_ptr()
    else:
        xp, lddx = _rows(dx, m, k, dt, "dx")
    if "dw" not in need:
        dw = None
    elif dw is None:
        dw = _new(dy, (n, k), dw_dtype or dt, stream)
        wp, wt = dw.data_ptr(), TYPE.get(dw.dtype, -1)
    else:
        wp, lddw = _rows(dw, n, k, dw.dtype, "dw")
        wt = TYPE.get(dw.dtype, -1)
    if "db" not in need:
        db = None
    else:
        if db is None:
            db = _new(dy, (n,), torch.float32, stream)
        bp = _vector(db, n, torch.float32, torch.float32, "db")
    _done((_ENTRIES.get("oz2_linear_grad") or _entry("oz2_linear_grad"))(
        m, n, k, TYPE.get(dt, -1), dy.data_ptr(), ldy, zp, ldz, ACT[act], x.data_ptr(), ldx, w.data_ptr(), ldw, xp, lddx,
        wp, lddw, wt, bp, GRAD_ACCUMULATE if accumulate else 0, _stream() if stream is None else stream.cuda_stream), "oz2_linear_grad")
    return dx, dw, db


class AdamWPlan:
    """The tensors of an AdamW step, as the C ABI takes them (oz2_adamw_plan).

    It holds the tensors, so their memory stays; a tensor that is replaced
    wants a new plan (`set_grads` takes new gradients).
    """

    def __init__(self, params, grads, m, v, masters, m_scales, v_scales, lr_scales, decay_scales):
        count = len(params)
        assert count == len(grads) == len(m) == len(v) and count > 0, "one gradient and one m and v for every parameter"
        self.bits = 8 if m[0].dtype == torch.float8_e4m3fn else 32
        state = torch.float8_e4m3fn if self.bits == 8 else torch.float32
        assert self.bits == 32 or (m_scales is not None and v_scales is not None), "8-bit states have scales"
        self.device = params[0].device
        self.param_type = params[0].dtype
        self.args = oz2_adamw_step()
        self.tensors = (oz2_adamw_tensor * count)()
        # Its own tuples: where a caller's list gets another entry, the tensor whose
        # address is taken below stays.
        self.params, self.m, self.v = tuple(params), tuple(m), tuple(v)
        self.masters, self.m_scales, self.v_scales = (None if t is None else tuple(t)
                                                      for t in (masters, m_scales, v_scales))
        for i, t in enumerate(self.tensors):
            e = params[i].numel()
            blocks = (e + ADAMW_BLOCK - 1) // ADAMW_BLOCK
            t.numel = e
            t.param = self._flat(params[i], e, self.param_type, "params")
            t.m, t.v = self._flat(m[i], e, state, "m"), self._flat(v[i], e, state, "v")
            if masters is not None and masters[i] is not None:
                t.master = self._flat(masters[i], e, torch.float32, "masters")
            if self.bits == 8:
                t.m_scale = self._flat(m_scales[i], blocks, torch.float32, "m_scales")
                t.v_scale = self._flat(v_scales[i], blocks, torch.float32, "v_scales")
            t.lr_scale = 1.0 if lr_scales is None else lr_scales[i]
            t.decay_scale = 1.0 if decay_scales is None else decay_scales[i]
        self.set_grads(grads)

    def _flat(self, t, numel, dtype, what):
        assert t.device == self.device and t.is_cuda and t.dtype == dtype and t.numel() == numel and t.is_contiguous(), \
            f"{what}: expected a contiguous CUDA tensor of {numel} {dtype} values"
        return t.data_ptr() if numel else None

    def set_grads(self, grads):
        """Take other gradients, one for each parameter (0.7 µs each on the host).  Where
        one of them is refused, the plan keeps the ones that it had."""
        grads = tuple(grads)
        assert len(grads) == len(self.tensors), "one gradient for every parameter"
        kind = grads[0].dtype
        at = [self._flat(g, t.numel, kind, "grads") for t, g in zip(self.tensors, grads)]
        self.grads, self.grad_type = grads, kind
        for t, a in zip(self.tensors, at):
            t.grad = a


def oz2_adamw_states(params, bits=32):
    """Zeroed states for oz2_adamw_plan: a dict of the lists m and v, and with
    bits=8 (E4M3 values with a scale per 256 of them) m_scales and v_scales."""
    assert bits in (8, 32)
    if bits == 32:
        return {s: [torch.zeros_like(p, dtype=torch.float32) for p in params] for s in ("m", "v")}
    out = {s: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for p in params]
           for s in ("m", "v")}
    for s in ("m_scales", "v_scales"):
        out[s] = [torch.ones((p.numel() + ADAMW_BLOCK - 1) // ADAMW_BLOCK, device=p.device) for p in params]
    return out


def oz2_adamw_plan(params, grads, m, v, masters=None, m_scales=None, v_scales=None, lr_scales=None,
                   decay_scales=None) -> AdamWPlan:
    """The handle of a step over these tensors (lists, contiguous): params of one
    dtype (float32, bfloat16, float16), grads of that or float32, states m and v
    float32 or float8_e4m3fn with float32 scales (oz2_adamw_states); masters:
    float32 weights beside 16-bit params, None for a tensor that has none; lr_scales
    and decay_scales: factors of each tensor's own (0 for no weight decay)."""
    return AdamWPlan(params, grads, m, v, masters, m_scales, v_scales, lr_scales, decay_scales)


def oz2_adamw(plan: AdamWPlan, step: int, lr: float, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
              grad_scale=None, seed=0, stream=None):
    """One AdamW step, in place.  step counts from 1; grad_scale: a float32 CUDA
    scalar that multiplies the gradients; seed: of the 8-bit states' rounding.

    Captured into a CUDA graph, a replay is the same step again (step, lr and seed as
    they were; grad_scale is read anew): a training program calls it for each step."""
    a = plan.args
    a.step, a.lr, a.beta1, a.beta2, a.eps, a.weight_decay, a.seed = step, lr, beta1, beta2, eps, weight_decay, seed
    if grad_scale is not None:
        assert grad_scale.is_cuda and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1
        a.d_grad_scale = grad_scale.data_ptr()
    else:
        a.d_grad_scale = None
    _done((_ENTRIES.get("oz2_adamw") or _entry("oz2_adamw"))(
        plan.tensors, len(plan.tensors), TYPE.get(plan.param_type, -1), TYPE.get(plan.grad_type, -1), plan.bits,
        ctypes.byref(a), _stream() if stream is None else stream.cuda_stream), "oz2_adamw")
