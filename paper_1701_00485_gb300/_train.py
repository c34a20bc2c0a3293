"""Binding of the operators beside the two-bit layers: layer norm, the AdamW
step and low-rank adapters (``tbn.h``).  The names are exported by the package."""
from __future__ import annotations

import ctypes
import struct

import torch

from . import TBN_F32, _check, _dt, _raw_stream, lib

_OP_NORM_FWD, _OP_NORM_BWD, _OP_ADAPTER_FWD, _OP_ADAPTER_BWD = range(5, 9)
_pack_norm_fwd = struct.Struct("=8qd6q").pack
_pack_norm_bwd = struct.Struct("=21q").pack
_pack_adapter_fwd = struct.Struct("=22q").pack
_pack_adapter_bwd = struct.Struct("=26q").pack
_STATE_32BIT, _STATE_8BIT = 0, 1
_ADAMW_BLOCK = 256


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("weight_decay", ctypes.c_float), ("lr_scale", ctypes.c_float),
                ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("state", ctypes.c_int32)]


class AdamWHyper(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("grad_scale", ctypes.c_void_p), ("seed", ctypes.c_uint32)]


class Adapters(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("r", ctypes.c_int64), ("K_in", ctypes.c_int64), ("K_out", ctypes.c_int64),
                ("ids", ctypes.c_void_p), ("ranks", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


def _rows(t, name, shape=None):
    """The row stride of a CUDA tensor [rows, D] whose rows are contiguous."""
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError("%s must be a 2-D tensor%s" % (
            name, "" if shape is None else " of shape %s" % (tuple(shape),)))
    ld, unit = t.stride()
    if unit != 1 and t.shape[1] > 1:
        raise ValueError("%s must have contiguous rows" % name)
    # rows of one element, and single rows, may carry any stride
    return ld if t.shape[0] > 1 else t.shape[1]


def _flat(t, name, n, dtypes):
    """The pointer of a contiguous CUDA tensor of n elements, 0 for None."""
    if t is None:
        return 0
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor" % name)
    if t.numel() != n or t.dtype not in dtypes:
        raise ValueError("%s must have %d elements of %s" % (
            name, n, " or ".join(str(d) for d in dtypes)))
    return t.data_ptr()


_F32 = (torch.float32,)
_FLOATS = (torch.float32, torch.bfloat16)
_BF16 = (torch.bfloat16,)
_I32 = (torch.int32,)


def _weights(gamma, beta, D):
    if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
        raise ValueError("gamma and beta must have the same dtype")
    w = gamma if gamma is not None else beta
    return (_flat(gamma, "gamma", D, _FLOATS), _flat(beta, "beta", D, _FLOATS),
            TBN_F32 if w is None else _dt(w))


def _bytes(t, name):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor" % name)
    return t.numel() * t.element_size()


def _scratch(nbytes, device, stream):
    """A workspace for one call; on another stream than the current one its
    memory is not handed out again before that stream's work is done."""
    t = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    if stream is not None:
        t.record_stream(stream)
    return t


def tbn_layernorm_fwd(x, gamma=None, beta=None, eps: float = 1e-5, out_dtype=None, out=None,
                      mean=None, rstd=None, stream=None):
    """Layer norm of the rows of x [rows, D] (bf16 or fp32; rows contiguous, any
    stride between them): (x - mean) rstd gamma + beta.

    Returns (y, mean, rstd); y has x's dtype or, with out_dtype or out, bf16;
    mean and rstd [rows] fp32 are what tbn_layernorm_bwd needs."""
    ldx = _rows(x, "x")
    rows, D = x.shape
    g, b, wdt = _weights(gamma, beta, D)
    if out is None:
        out = torch.empty((rows, D), dtype=out_dtype or x.dtype, device=x.device)
    if mean is None:
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
    if rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    ldy = _rows(out, "out", x.shape)
    _call_packed(_OP_NORM_FWD, "tbn_layernorm_fwd", _pack_norm_fwd(
        x.data_ptr(), _dt(x), rows, D, ldx, g, b, wdt, eps, out.data_ptr(), _dt(out), ldy,
        _flat(mean, "mean", rows, _F32), _flat(rstd, "rstd", rows, _F32), _raw_stream(stream)))
    return out, mean, rstd


def tbn_layernorm_bwd_workspace_bytes(rows: int, D: int) -> int:
    return int(lib().tbn_layernorm_bwd_workspace_bytes(rows, D))


def tbn_layernorm_bwd(dy, x, mean, rstd, gamma=None, dres=None, dx=None, dgamma=None, dbeta=None,
                      workspace=None, weight_grads: bool = True, stream=None):
    """Gradients of tbn_layernorm_fwd for dy [rows, D] (x's dtype or bf16).

    dx has x's dtype and is added to dres, the gradient of a residual branch
    around the norm, where one is given.  Returns (dx, dgamma, dbeta), the last
    two fp32 [D], or None without weight_grads."""
    ldx, lddy = _rows(x, "x"), _rows(dy, "dy", x.shape)
    rows, D = x.shape
    g, _, wdt = _weights(gamma, None, D)
    if dx is None:
        dx = torch.empty((rows, D), dtype=x.dtype, device=x.device)
    if weight_grads:
        if dgamma is None:
            dgamma = torch.empty(D, dtype=torch.float32, device=x.device)
        if dbeta is None:
            dbeta = torch.empty(D, dtype=torch.float32, device=x.device)
        if workspace is None:
            workspace = _scratch(tbn_layernorm_bwd_workspace_bytes(rows, D), x.device, stream)
        nws = _bytes(workspace, "workspace")
    else:
        dgamma = dbeta = workspace = None
        nws = 0
    if dx.dtype != x.dtype or (dres is not None and dres.dtype != x.dtype):
        raise ValueError("dx and dres must have x's dtype")
    lddres = 0 if dres is None else _rows(dres, "dres", x.shape)
    _call_packed(_OP_NORM_BWD, "tbn_layernorm_bwd", _pack_norm_bwd(
        dy.data_ptr(), _dt(dy), lddy, x.data_ptr(), _dt(x), rows, D, ldx,
        _flat(mean, "mean", rows, _F32), _flat(rstd, "rstd", rows, _F32), g, wdt,
        0 if dres is None else dres.data_ptr(), lddres, dx.data_ptr(), _rows(dx, "dx", x.shape),
        _flat(dgamma, "dgamma", D, _F32), _flat(dbeta, "dbeta", D, _F32),
        0 if workspace is None else workspace.data_ptr(), nws, _raw_stream(stream)))
    return dx, dgamma, dbeta


class AdamWPlan:
    """The tensors of an AdamW step, as tbn_adamw_step takes them.

    Lists of equal length: params (fp32 or bf16, updated in place), grads (fp32
    or bf16) and the moments m and v, updated in place and each either fp32 of
    the parameter's size, or torch.float8_e4m3fn and torch.float8_e5m2 with
    m_scale and v_scale, fp32 of one element for each 256 of the parameter
    (AdamWPlan.state8 makes them).  copies: bf16 tensors or None, which receive
    the rounded new parameters.  weight_decay and lr_scale: a number, or one
    for each tensor.  The plan keeps the tensors; with gradients in other
    memory call set_grads."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None,
                 weight_decay=0.0, lr_scale=1.0):
        n = len(params)
        none = [None] * n
        m_scale, v_scale, copies = (none if t is None else t for t in (m_scale, v_scale, copies))
        per = lambda c: [float(c)] * n if isinstance(c, (int, float)) else [float(x) for x in c]  # noqa: E731
        decay, lrs = per(weight_decay), per(lr_scale)
        lists = (grads, m, v, m_scale, v_scale, copies, decay, lrs)
        if any(len(t) != n for t in lists):
            raise ValueError("lists of %d tensors are needed" % n)
        self.tensors = (list(params), list(m), list(v), list(m_scale), list(v_scale), list(copies))
        self._array = (AdamWTensor * max(n, 1))()
        self.count = n
        for i, t in enumerate(self._array[:n]):
            p, size = params[i], params[i].numel()
            eight = m[i].dtype == torch.float8_e4m3fn
            blocks = -(-size // _ADAMW_BLOCK)
            t.param = _flat(p, "params[%d]" % i, size, _FLOATS)
            t.m = _flat(m[i], "m[%d]" % i, size, (torch.float8_e4m3fn,) if eight else _F32)
            t.v = _flat(v[i], "v[%d]" % i, size, (torch.float8_e5m2,) if eight else _F32)
            if eight and (m_scale[i] is None or v_scale[i] is None):
                raise ValueError("8-bit moments need m_scale and v_scale")
            t.m_scale = _flat(m_scale[i], "m_scale[%d]" % i, blocks, _F32) if eight else 0
            t.v_scale = _flat(v_scale[i], "v_scale[%d]" % i, blocks, _F32) if eight else 0
            t.copy = _flat(copies[i], "copies[%d]" % i, size, (torch.bfloat16,))
            t.n, t.weight_decay, t.lr_scale = size, decay[i], lrs[i]
            t.param_dtype = _dt(p)
            t.state = _STATE_8BIT if eight else _STATE_32BIT
        self._hyper = AdamWHyper()
        self.set_grads(grads)

    @staticmethod
    def state8(param):
        """Zeroed 8-bit moments of a parameter: (m, v, m_scale, v_scale)."""
        n, blocks = param.numel(), -(-param.numel() // _ADAMW_BLOCK)
        z = lambda k, d: torch.zeros(k, dtype=d, device=param.device)  # noqa: E731
        return (z(n, torch.uint8).view(torch.float8_e4m3fn), z(n, torch.uint8).view(torch.float8_e5m2),
                z(blocks, torch.float32), z(blocks, torch.float32))

    def set_grads(self, grads):
        """Other gradient tensors of the same sizes from the next step on."""
        if len(grads) != self.count:
            raise ValueError("lists of %d tensors are needed" % self.count)
        for i, (t, g) in enumerate(zip(self._array, grads)):
            t.grad, t.grad_dtype = _flat(g, "grads[%d]" % i, t.n, _FLOATS), _dt(g)
        self.grads = list(grads)


def tbn_adamw_step(plan: AdamWPlan, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
                   grad_scale=None, seed: int = 0, stream=None):
    """One AdamW step (number `step`, from 1) of the plan's tensors, in place.

    grad_scale: None, or a CUDA fp32 scalar that all gradients are multiplied
    by (1 / loss scale, or the factor of a clipped norm).  seed: another number
    in every step; it decides how 8-bit moments are rounded."""
    h = plan._hyper
    h.lr, (h.beta1, h.beta2), h.eps, h.step = lr, betas, eps, step
    h.grad_scale = _flat(grad_scale, "grad_scale", 1, _F32)
    h.seed = seed & 0xFFFFFFFF
    _check(lib().tbn_adamw_step(plan._array, plan.count, ctypes.byref(h), _raw_stream(stream)),
           "tbn_adamw_step")


def tbn_adapter_workspace_bytes(T: int, K_in: int, K_out: int, n: int, r: int,
                                backward: bool = False) -> int:
    """Scratch bytes of tbn_adapter_fwd, or with backward of tbn_adapter_bwd."""
    return int(lib().tbn_adapter_workspace_bytes(T, K_in, K_out, n, r, 1 if backward else 0))


def _adapters(a, b, T, ids, scale, ranks):
    """The first nine arguments of a packed adapter call."""
    if a.dim() != 3 or b.dim() != 3 or a.shape[:2] != b.shape[:2]:
        raise ValueError("a must be [n, r, K_in] and b [n, r, K_out]")
    n, r, K_in = a.shape
    return (_flat(a, "a", n * r * K_in, _BF16), _flat(b, "b", b.numel(), _BF16), n, r, K_in,
            b.shape[2], _flat(ids, "ids", T, _I32), _flat(ranks, "ranks", n, _I32),
            _flat(scale, "scale", n, _F32))


def _base(base, like, name):
    if base is None:
        return 0, 0
    if base.dtype != like.dtype:
        raise ValueError("base must have %s's dtype" % name)
    return base.data_ptr(), _rows(base, "base", like.shape)


def tbn_adapter_fwd(x, a, b, ids=None, scale=None, ranks=None, base=None, out_dtype=None,
                    out=None, v=None, workspace=None, stream=None):
    """Low-rank adapters of many requests: y_t = base_t + scale_i (a_i x_t) b_i
    with i = ids[t].

    x [T, K_in] (bf16 or fp32; rows contiguous, any stride between them),
    a [n, r, K_in] and b [n, r, K_out] bf16, both rank by rank; ids [T] int32 in
    any order, values outside 0 .. n - 1 for tokens without an adapter, None for
    adapter 0 everywhere; scale [n] fp32; ranks [n] int32 (what a and b hold past
    them is not read); base [T, K_out] of y's dtype, the shared projection's
    output, which `out` may be.  v: None, or fp32 [T, r] that receives a_i x_t
    for tbn_adapter_bwd.  y has base's, out's, out_dtype's or x's dtype."""
    ldx = _rows(x, "x")
    T = x.shape[0]
    ad = _adapters(a, b, T, ids, scale, ranks)
    if x.shape[1] != ad[4]:
        raise ValueError("x has %d columns, a expects %d" % (x.shape[1], ad[4]))
    if out is None:
        dt = out_dtype or (x if base is None else base).dtype
        out = torch.empty((T, ad[5]), dtype=dt, device=x.device)
    if workspace is None:
        workspace = _scratch(tbn_adapter_workspace_bytes(T, ad[4], ad[5], ad[2], ad[3]), x.device,
                             stream)
    ldy = _rows(out, "out", (T, ad[5]))
    _call_packed(_OP_ADAPTER_FWD, "tbn_adapter_fwd", _pack_adapter_fwd(
        *ad, x.data_ptr(), _dt(x), T, ldx, *_base(base, out, "y"), out.data_ptr(), _dt(out), ldy,
        _flat(v, "v", T * ad[3], _F32), workspace.data_ptr(), _bytes(workspace, "workspace"),
        _raw_stream(stream)))
    return out


def tbn_adapter_bwd(dy, x, a, b, ids=None, scale=None, ranks=None, v=None, base=None, dx=None,
                    da=None, db=None, need=(True, True, True), workspace=None, stream=None):
    """Gradients of tbn_adapter_fwd for dy [T, K_out]: (dx, da, db).

    dx has x's dtype and is added to base, the gradient through the shared
    projection, where one is given (`dx` may be it); da and db are fp32 of a's and
    b's shape, zero past an adapter's rank and for adapters without tokens.  v:
    what tbn_adapter_fwd wrote, or None to compute it again.  need: which of the
    three are wanted; the others come back as None."""
    ldx, lddy = _rows(x, "x"), _rows(dy, "dy")
    T = x.shape[0]
    ad = _adapters(a, b, T, ids, scale, ranks)
    if x.shape[1] != ad[4] or tuple(dy.shape) != (T, ad[5]):
        raise ValueError("x must be [T, K_in] and dy [T, K_out] of a and b")
    if not need[0]:
        dx = None
    elif dx is None:
        dx = torch.empty((T, ad[4]), dtype=x.dtype, device=x.device)
    elif dx.dtype != x.dtype:
        raise ValueError("dx must have x's dtype")
    if not need[1]:
        da = None
    elif da is None:
        da = torch.empty(a.shape, dtype=torch.float32, device=x.device)
    if not need[2]:
        db = None
    elif db is None:
        db = torch.empty(b.shape, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = _scratch(tbn_adapter_workspace_bytes(T, ad[4], ad[5], ad[2], ad[3], True),
                             x.device, stream)
    _call_packed(_OP_ADAPTER_BWD, "tbn_adapter_bwd", _pack_adapter_bwd(
        *ad, dy.data_ptr(), _dt(dy), lddy, x.data_ptr(), _dt(x), T, ldx,
        _flat(v, "v", T * ad[3], _F32), *(_base(base, x, "x") if dx is not None else (0, 0)),
        0 if dx is None else dx.data_ptr(), 0 if dx is None else _rows(dx, "dx", x.shape),
        _flat(da, "da", a.numel(), _F32), _flat(db, "db", b.numel(), _F32), workspace.data_ptr(),
        _bytes(workspace, "workspace"), _raw_stream(stream)))
    return dx, da, db


def _call_packed(op, where, block):
    status = lib().tbn_packed_call(op, block)
    if status != 0:
        _check(status, where)
