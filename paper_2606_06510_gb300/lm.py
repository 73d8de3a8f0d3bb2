"""The binding of the operators at a language model's ends (include/oz2_lm.h):
embedding, layer norm, and the losses over a vocabulary that are taken from the last
layer's input and the head's weights, each with its gradient.

Arrays are as in `layers`: row-major (tokens, features) with stride(1) == 1 and any
row stride, all on the current device.  Tokens name rows by int64 or int32.  A call
runs on the current stream, or on `stream`, whose memory its new outputs then are.  The
forward passes record no graph of gradients: tensors that require them are refused
unless that is off (torch.no_grad()).  Nor do the gradients' functions, whose results are
plain numbers: their x, weights and so on may require gradients, but a dy, dloss or
residual that does, as on the way to second derivatives, is refused in the same way.
"""
from __future__ import annotations

import ctypes

import torch

from .layers import _EMPTY, GRAD_ACCUMULATE, TYPE, _ENTRIES, _done, _entry, _ld, _new

_I64, _P, _I, _U, _F = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_uint, ctypes.c_float
GRAD_ONE_DLOSS = 0x2
MAX_TOP = 1024
IDS = {torch.int64: 64, torch.int32: 32}

SIGS = {
    "oz2_embedding": (_I, [_I64, _I64, _I64, _I, _P, _I, _P, _I64, _F, _P, _I64, _P]),
    "oz2_embedding_grad": (_I, [_I64, _I64, _I64, _I, _P, _I64, _P, _I, _F, _P, _I64, _I, _U, _P]),
    "oz2_layer_norm": (_I, [_I64, _I64, _I, _P, _I64, _P, _P, _I, _F, _I, _P, _I64, _P, _P, _P]),
    "oz2_layer_norm_grad": (_I, [_I64, _I64, _I, _P, _I64, _P, _I64, _P, _P, _P, _I, _P, _I64, _P, _I64, _P, _P, _U, _P]),
    "oz2_linear_xent": (_I, [_I64, _I64, _I64, _I, _P, _I64, _P, _I64, _P, _I, _F, _F, _P, _P, _P, _P]),
    "oz2_linear_xent_grad": (_I, [_I64, _I64, _I64, _I, _P, _P, _I64, _P, _I64, _P, _I, _P, _F, _F, _P, _I64, _P, _I64,
                                  _I, _U, _P]),
    "oz2_linear_distill": (_I, [_I64, _I64, _I64, _I64, _I, _P, _I64, _P, _I64, _P, _I64, _I, _P, _I64, _I, _F, _P, _P,
                                _P, _P]),
    "oz2_linear_distill_grad": (_I, [_I64, _I64, _I64, _I64, _I, _P, _P, _I64, _P, _I64, _P, _I64, _I, _P, _I64, _I, _F,
                                     _P, _P, _I64, _P, _I64, _I, _U, _P]),
}


# The checks of a call cost more than its launch (5 µs of Python for 2 of CUDA), so each
# operator asks for all of a tensor's properties at once, and only where one is not as
# expected goes to the function that says which, or finds that it does not matter.
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


_F32, _FLOATS = torch.float32, (torch.float32, torch.bfloat16, torch.float16)


def _empty(shape, strides, dtype):
    return torch.empty_strided(shape, strides, dtype=dtype, device="cuda")


# A new output on the current device, of the current stream's memory.
_fresh = _EMPTY or _empty


def _lost(what):
    assert not torch.is_grad_enabled(), f"a tensor requires its gradient, which would be lost: call {what} " \
        f"under torch.no_grad(), and {what}_grad for the gradients"


def _lost_twice(what):
    assert not torch.is_grad_enabled(), f"a gradient requires its gradient, which would be lost: {what} records no " \
        "graph for second derivatives; call it under torch.no_grad()"


def _home(t, what):
    """The device of a call's first tensor: the current one."""
    dev = t.get_device()
    assert dev >= 0 and dev == _device(), f"{what}: oz2 operates on CUDA tensors of the current device"
    return dev


def _odd(t, rows, cols, dtype, dev, what):
    """The row stride of a matrix that is not of this shape, dtype and device with contiguous rows,
    or need not be."""
    assert t.shape == (rows, cols) and t.dtype == dtype, \
        f"{what}: expected shape ({rows}, {cols}) and {dtype}, got {tuple(t.shape)} and {t.dtype}"
    assert t.get_device() == dev, f"{what}: oz2 operates on CUDA tensors of the current device"
    return _ld(t, rows, cols, what)


def _matrix(t, rows, cols, dtype, dev, what):
    """(address, row stride) of a matrix of this shape and dtype."""
    ld, one = t.stride() if t.dim() == 2 else (0, 0)
    if t.dtype is not dtype or t.shape != (rows, cols) or t.get_device() != dev or one != 1 or ld < cols or ld < 1:
        ld = _odd(t, rows, cols, dtype, dev, what)
    return t.data_ptr(), ld


def _vector(t, count, dtype, other, dev, what):
    """The address of a contiguous vector of one of two dtypes."""
    dt = t.dtype
    if (dt is not dtype and dt is not other) or t.shape != (count,) or t.get_device() != dev or not t.is_contiguous():
        assert t.shape == (count,) and (dt == dtype or dt == other) and t.is_contiguous(), \
            f"{what}: expected {count} contiguous values of {dtype}{'' if other is dtype else f' or {other}'}, " \
            f"got {tuple(t.shape)} and {dt}"
        assert t.get_device() == dev, f"{what}: oz2 operates on CUDA tensors of the current device"
    return t.data_ptr()


def oz2_embedding(ids, table, scale=1.0, out=None, stream=None):
    """scale·table[ids] for tokens ids (m,) and a table (n, k) of float32, bfloat16 or
    float16: (m, k) of its dtype.  ids below 0 (padding) give zeros, ids of n or more NaN."""
    if table.requires_grad:
        _lost("oz2_embedding")
    n, k = table.shape
    m, = ids.shape
    dt = table.dtype
    assert dt in _FLOATS, "table: expected float32, bfloat16 or float16"
    assert ids.dtype in IDS, "ids: expected int64 or int32"
    dev = _home(table, "table")
    ip = _vector(ids, m, torch.int64, torch.int32, dev, "ids")
    ldt, one = table.stride()
    if one != 1 or ldt < k or ldt < 1:
        ldt = _odd(table, n, k, dt, dev, "table")
    tp = table.data_ptr()
    if out is None:
        out = _fresh((m, k), (k or 1, 1), dt) if stream is None else _new(table, (m, k), dt, stream)
        op, ldo = out.data_ptr(), k or 1
    else:
        op, ldo = _matrix(out, m, k, dt, dev, "out")
    code = (_ENTRIES.get("oz2_embedding") or _entry("oz2_embedding"))(
        m, n, k, TYPE[dt], ip, IDS[ids.dtype], tp, ldt, scale, op, ldo,
        _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_embedding")
    return out


def oz2_embedding_grad(dy, ids, n, scale=1.0, out=None, out_dtype=None, accumulate=False, stream=None):
    """The gradient (n, k) of oz2_embedding's table from dy (m, k): the sum of scale·dy_t over
    each row's tokens, in dy's dtype or float32 (out_dtype).  With accumulate it is added to
    `out`, whose other rows stay; else rows without tokens are zeros.  ids outside [0, n) count
    for nothing."""
    if dy.requires_grad:
        _lost_twice("oz2_embedding_grad")
    m, k = dy.shape
    dt = dy.dtype
    assert dt in _FLOATS, "dy: expected float32, bfloat16 or float16"
    assert out is not None or not accumulate, "accumulate: out has to be given"
    assert ids.dtype in IDS, "ids: expected int64 or int32"
    dev = _home(dy, "dy")
    dp, ldd = _matrix(dy, m, k, dt, dev, "dy")
    ip = _vector(ids, m, torch.int64, torch.int32, dev, "ids")
    if out is None:
        ot = out_dtype or dt
        out = _new(dy, (n, k), ot, stream)
        op, ldo = out.data_ptr(), k or 1
    else:
        ot = out.dtype
        assert out_dtype is None or out_dtype == ot, "out_dtype: out has another"
        op, ldo = _matrix(out, n, k, ot, dev, "out")
    code = (_ENTRIES.get("oz2_embedding_grad") or _entry("oz2_embedding_grad"))(
        m, n, k, TYPE[dt], dp, ldd, ip, IDS[ids.dtype], scale, op, ldo, TYPE.get(ot, -1),
        GRAD_ACCUMULATE if accumulate else 0, _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_embedding_grad")
    return out


def oz2_layer_norm(x, weight=None, bias=None, eps=1e-5, center=True, save_stats=False, out=None, stream=None):
    """(x - mean)·rstd·weight + bias over the features of each row of x (m, k), of float32,
    bfloat16 or float16; without the mean where not center (rstd is then that of the mean of
    squares).  weight and bias (k,) have x's dtype or float32, both the same.  With
    save_stats, returns (y, mean, rstd) with the float32 (m,) that oz2_layer_norm_grad wants
    (mean None where not center).  `out` may be x itself."""
    if x.requires_grad or (weight is not None and weight.requires_grad) or (bias is not None and bias.requires_grad):
        _lost("oz2_layer_norm")
    m, k = x.shape
    dt = x.dtype
    assert dt in _FLOATS, "x: expected float32, bfloat16 or float16"
    dev = _home(x, "x")
    ldx, one = x.stride()
    if one != 1 or ldx < k or ldx < 1:
        ldx = _odd(x, m, k, dt, dev, "x")
    xp = x.data_ptr()
    wp = bp = mp = sp = mean = rstd = None
    wt = 0
    if weight is not None:
        wp, wt = _vector(weight, k, dt, torch.float32, dev, "weight"), TYPE[weight.dtype]
    if bias is not None:
        bp = _vector(bias, k, dt, torch.float32, dev, "bias")
        assert weight is None or bias.dtype is weight.dtype, "weight and bias: expected one dtype"
        wt = TYPE[bias.dtype]
    if out is None:
        out = _fresh((m, k), (k or 1, 1), dt) if stream is None else _new(x, (m, k), dt, stream)
        op, ldo = out.data_ptr(), k or 1
    else:
        op, ldo = _matrix(out, m, k, dt, dev, "out")
    if save_stats:
        rstd = _fresh((m,), (1,), _F32) if stream is None else _new(x, (m,), _F32, stream)
        sp = rstd.data_ptr()
        if center:
            mean = _fresh((m,), (1,), _F32) if stream is None else _new(x, (m,), _F32, stream)
            mp = mean.data_ptr()
    code = (_ENTRIES.get("oz2_layer_norm") or _entry("oz2_layer_norm"))(
        m, k, TYPE[dt], xp, ldx, wp, bp, wt, eps, 1 if center else 0, op, ldo, mp, sp,
        _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_layer_norm")
    return (out, mean, rstd) if save_stats else out


def oz2_layer_norm_grad(dy, x, mean, rstd, weight=None, residual=None, need=("dx", "dweight", "dbias"), dx=None,
                        dweight=None, dbias=None, accumulate=False, stream=None):
    """(dx, dweight, dbias) of oz2_layer_norm from dy, its x, and the mean (None: not centred)
    and rstd that it kept.  residual (m, k), the gradient that comes by a skip connection, is
    added to dx (which may be given as the same tensor).  `need` names the gradients wanted (the
    others are None).  dx has x's dtype, dweight and dbias (k,) are float32; with accumulate those
    two are added to, and must be given."""
    if dy.requires_grad or (residual is not None and residual.requires_grad):
        _lost_twice("oz2_layer_norm_grad")
    m, k = x.shape
    dt = x.dtype
    f32 = _F32
    assert dt in _FLOATS, "x: expected float32, bfloat16 or float16"
    assert dy.dtype is dt, "dy: expected x's dtype"
    dev = _home(x, "x")
    dp, ldd = _matrix(dy, m, k, dt, dev, "dy")
    xp, ldx = _matrix(x, m, k, dt, dev, "x")
    mp = None if mean is None else _vector(mean, m, f32, f32, dev, "mean")
    sp = _vector(rstd, m, f32, f32, dev, "rstd")
    wp = rp = op = gp = bp = None
    wt, ldr, ldo = 0, 1, k or 1
    if weight is not None:
        wp, wt = _vector(weight, k, dt, f32, dev, "weight"), TYPE[weight.dtype]
    if residual is not None:
        rp, ldr = _matrix(residual, m, k, dt, dev, "residual")
    assert not accumulate or (("dweight" not in need or dweight is not None) and ("dbias" not in need or dbias is not None)), \
        "accumulate: dweight and dbias have to be given"
    if "dx" not in need:
        dx = None
    elif dx is None:
        dx = _fresh((m, k), (k or 1, 1), dt) if stream is None else _new(x, (m, k), dt, stream)
        op = dx.data_ptr()
    else:
        op, ldo = _matrix(dx, m, k, dt, dev, "dx")
    if "dweight" not in need:
        dweight = None
    elif dweight is None:
        dweight = _fresh((k,), (1,), f32) if stream is None else _new(x, (k,), f32, stream)
        gp = dweight.data_ptr()
    else:
        gp = _vector(dweight, k, f32, f32, dev, "dweight")
    if "dbias" not in need:
        dbias = None
    elif dbias is None:
        dbias = _fresh((k,), (1,), f32) if stream is None else _new(x, (k,), f32, stream)
        bp = dbias.data_ptr()
    else:
        bp = _vector(dbias, k, f32, f32, dev, "dbias")
    code = (_ENTRIES.get("oz2_layer_norm_grad") or _entry("oz2_layer_norm_grad"))(
        m, k, TYPE[dt], dp, ldd, xp, ldx, mp, sp, wp, wt, rp, ldr, op, ldo, gp, bp, GRAD_ACCUMULATE if accumulate else 0,
        _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_layer_norm_grad")
    return dx, dweight, dbias


def _head(x, w):
    """Sizes, device and addresses of a head's input and weights."""
    m, k = x.shape
    n, k2 = w.shape
    dt = x.dtype
    assert k == k2 and w.dtype is dt, "x and w: expected (m, k) and (n, k) of one dtype"
    assert dt is torch.bfloat16 or dt is torch.float16, "x and w: expected bfloat16 or float16"
    dev = _home(x, "x")
    ldx, one = x.stride()
    if one != 1 or ldx < k or ldx < 1:
        ldx = _odd(x, m, k, dt, dev, "x")
    ldw, one = w.stride()
    if one != 1 or ldw < k or ldw < 1 or w.get_device() != dev:
        ldw = _odd(w, n, k, dt, dev, "w")
    return m, n, k, dt, dev, x.data_ptr(), ldx, w.data_ptr(), ldw


def _entries(ids, teacher, m, dev):
    """(entries of a token, the arguments of a teacher's rows and logits)."""
    assert ids.dim() == 2 and ids.shape[0] == m and ids.dtype in IDS, \
        f"ids: expected shape ({m}, top) of int64 or int32, got {tuple(ids.shape)} and {ids.dtype}"
    top = ids.shape[1]
    assert 1 <= top <= MAX_TOP, f"ids: expected 1 to {MAX_TOP} entries a token"
    ip, ldi = _matrix(ids, m, top, ids.dtype, dev, "ids")
    assert teacher.dtype in _FLOATS, "teacher: expected float32, bfloat16 or float16"
    tp, ldt = _matrix(teacher, m, top, teacher.dtype, dev, "teacher")
    return top, (ip, ldi, IDS[ids.dtype], tp, ldt, TYPE[teacher.dtype])


def oz2_linear_xent(x, w, targets, scale=1.0, z_loss=0.0, stream=None):
    """Cross entropy over the rows of w (n, k) of tokens x (m, k), bfloat16 or float16, with
    logits z = scale·x·wᵀ that are not kept: (loss, lse, picked), float32 (m,) each, with
    loss = lse - picked + z_loss·lse², lse = log Σ exp z and picked the target's z.
    targets (m,) below 0 do not count (loss and picked 0); of n or more: NaN."""
    if x.requires_grad or w.requires_grad:
        _lost("oz2_linear_xent")
    m, n, k, dt, dev, xp, ldx, wp, ldw = _head(x, w)
    assert targets.dtype in IDS, "targets: expected int64 or int32"
    ip = _vector(targets, m, torch.int64, torch.int32, dev, "targets")
    if stream is None:
        loss, lse, picked = _fresh((m,), (1,), _F32), _fresh((m,), (1,), _F32), _fresh((m,), (1,), _F32)
    else:
        loss, lse, picked = (_new(x, (m,), _F32, stream) for _ in range(3))
    code = (_ENTRIES.get("oz2_linear_xent") or _entry("oz2_linear_xent"))(
        m, n, k, TYPE[dt], xp, ldx, wp, ldw, ip, IDS[targets.dtype], scale, z_loss, loss.data_ptr(), lse.data_ptr(),
        picked.data_ptr(), _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_linear_xent")
    return loss, lse, picked


def _outputs(x, m, n, k, dt, dev, need, dx, dw, dw_dtype, accumulate, stream):
    """(dx, dw, their arguments) of a head's gradient."""
    assert not accumulate or "dw" not in need or dw is not None, "accumulate: dw has to be given"
    xp = wp = None
    ldx = ldw = k or 1
    wt = TYPE[dt]
    if "dx" not in need:
        dx = None
    elif dx is None:
        dx = _fresh((m, k), (k or 1, 1), dt) if stream is None else _new(x, (m, k), dt, stream)
        xp = dx.data_ptr()
    else:
        xp, ldx = _matrix(dx, m, k, dt, dev, "dx")
    if "dw" not in need:
        dw = None
    elif dw is None:
        dw = _fresh((n, k), (k or 1, 1), dw_dtype or dt) if stream is None else _new(x, (n, k), dw_dtype or dt, stream)
        wp, wt = dw.data_ptr(), TYPE.get(dw.dtype, -1)
    else:
        wp, ldw = _matrix(dw, n, k, dw.dtype, dev, "dw")
        wt = TYPE.get(dw.dtype, -1)
    return dx, dw, (xp, ldx, wp, ldw, wt)


def _dloss(dloss, m, dev):
    """(address, flags) of the losses' gradient: float32, one a token or one for all."""
    if dloss.dim() == 0 or (dloss.dim() == 1 and dloss.shape[0] == m and m > 1 and dloss.stride(0) == 0):
        assert dloss.dtype is torch.float32, "dloss: expected float32"
        assert dloss.get_device() == dev, "dloss: oz2 operates on CUDA tensors of the current device"
        return dloss.data_ptr(), GRAD_ONE_DLOSS
    return _vector(dloss, m, torch.float32, torch.float32, dev, "dloss"), 0


def oz2_linear_xent_grad(dloss, x, w, targets, lse, scale=1.0, z_loss=0.0, need=("dx", "dw"), dx=None, dw=None,
                         dw_dtype=None, accumulate=False, stream=None):
    """(dx, dw) of oz2_linear_xent from dloss, float32 (m,) or a scalar that goes for every
    token, and the lse that it kept.  `need` names the gradients wanted (the others are None).
    dx (m, k) has x's dtype, dw (n, k) that or float32 (dw_dtype); each may be given as the tensor
    to write.  With accumulate, dw (float32) is added to, and must be given."""
    if dloss.requires_grad:
        _lost_twice("oz2_linear_xent_grad")
    m, n, k, dt, dev, xp, ldx, wp, ldw = _head(x, w)
    assert targets.dtype in IDS, "targets: expected int64 or int32"
    ip = _vector(targets, m, torch.int64, torch.int32, dev, "targets")
    lp = _vector(lse, m, torch.float32, torch.float32, dev, "lse")
    gp, flags = _dloss(dloss, m, dev)
    dx, dw, outs = _outputs(x, m, n, k, dt, dev, need, dx, dw, dw_dtype, accumulate, stream)
    code = (_ENTRIES.get("oz2_linear_xent_grad") or _entry("oz2_linear_xent_grad"))(
        m, n, k, TYPE[dt], gp, xp, ldx, wp, ldw, ip, IDS[targets.dtype], lp, scale, z_loss, *outs,
        flags | (GRAD_ACCUMULATE if accumulate else 0), _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_linear_xent_grad")
    return dx, dw


def oz2_linear_distill(x, w, ids, teacher, temperature=1.0, stream=None):
    """The loss against a teacher's logits of `top` listed rows of each token, ids and teacher
    (m, top), with logits z = x·wᵀ/temperature that are not kept: (loss, lse, picked) with
    loss = Σ q·(log q - z_id) + lse, q the softmax of teacher/temperature over the token's listed
    rows, lse = log Σ exp z, float32 (m,), and picked the listed rows' z, float32 (m, top).  ids
    below 0 list nothing (picked 0); a token without rows does not count (loss 0); an id of n or
    more gives NaN.  x and w as for oz2_linear_xent, teacher float32, bfloat16 or float16."""
    if x.requires_grad or w.requires_grad or teacher.requires_grad:
        _lost("oz2_linear_distill")
    m, n, k, dt, dev, xp, ldx, wp, ldw = _head(x, w)
    top, listed = _entries(ids, teacher, m, dev)
    loss = _new(x, (m,), torch.float32, stream)
    lse = _new(x, (m,), torch.float32, stream)
    picked = _new(x, (m, top), torch.float32, stream)
    code = (_ENTRIES.get("oz2_linear_distill") or _entry("oz2_linear_distill"))(
        m, n, k, top, TYPE[dt], xp, ldx, wp, ldw, *listed, temperature, loss.data_ptr(), lse.data_ptr(),
        picked.data_ptr(), _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_linear_distill")
    return loss, lse, picked


def oz2_linear_distill_grad(dloss, x, w, ids, teacher, lse, temperature=1.0, need=("dx", "dw"), dx=None, dw=None,
                            dw_dtype=None, accumulate=False, stream=None):
    """(dx, dw) of oz2_linear_distill, as oz2_linear_xent_grad's."""
    if dloss.requires_grad:
        _lost_twice("oz2_linear_distill_grad")
    m, n, k, dt, dev, xp, ldx, wp, ldw = _head(x, w)
    top, listed = _entries(ids, teacher, m, dev)
    lp = _vector(lse, m, torch.float32, torch.float32, dev, "lse")
    gp, flags = _dloss(dloss, m, dev)
    dx, dw, outs = _outputs(x, m, n, k, dt, dev, need, dx, dw, dw_dtype, accumulate, stream)
    code = (_ENTRIES.get("oz2_linear_distill_grad") or _entry("oz2_linear_distill_grad"))(
        m, n, k, top, TYPE[dt], gp, xp, ldx, wp, ldw, *listed, temperature, lp, *outs,
        flags | (GRAD_ACCUMULATE if accumulate else 0), _raw_stream(dev) if stream is None else stream.cuda_stream)
    if code:
        _done(code, "oz2_linear_distill_grad")
    return dx, dw
