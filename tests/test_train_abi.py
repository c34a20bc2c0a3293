"""Host-side checks of the operators beside the two-bit layers (no GPU needed):
invalid arguments are refused before anything is launched."""
import ctypes
import math

import pytest

import paper_1701_00485_gb300 as tbn
from paper_1701_00485_gb300 import build as tbn_build

OK, INVALID, UNSUPPORTED, MISALIGNED = range(4)
D = ctypes.c_void_p(1 << 20)


@pytest.fixture(scope="module")
def L():
    tbn_build.build()
    return tbn.lib()


def _norm_fwd(L, **kw):
    a = dict(x=D, xdt=1, rows=4, D=64, ldx=64, gamma=D, beta=D, wdt=0, eps=1e-5, y=D, ydt=1, ldy=64,
             mean=D, rstd=D)
    a.update(kw)
    return L.tbn_layernorm_fwd(*a.values(), None)


def test_layernorm_fwd_refusals(L):
    for kw in (dict(x=None), dict(y=None), dict(rows=-1), dict(D=0), dict(xdt=2), dict(ydt=7),
               dict(wdt=-1), dict(ldx=63), dict(ldy=10), dict(eps=-1.0), dict(eps=math.nan)):
        assert _norm_fwd(L, **kw) == INVALID, kw
    for kw in (dict(ydt=0), dict(rows=1 << 31), dict(D=(1 << 28) + 1, ldx=1 << 30, ldy=1 << 30),
               dict(rows=1 << 20, ldx=1 << 40)):
        assert _norm_fwd(L, **kw) == UNSUPPORTED, kw
    odd = ctypes.c_void_p((1 << 20) + 1)
    for kw in (dict(x=odd), dict(y=odd), dict(gamma=odd), dict(beta=odd), dict(mean=odd), dict(rstd=odd)):
        assert _norm_fwd(L, **kw) == MISALIGNED, kw
    assert b"layernorm_fwd" in L.tbn_last_error()
    assert _norm_fwd(L, rows=0, x=None, y=None) == OK      # nothing to do


def _norm_bwd(L, **kw):
    need = L.tbn_layernorm_bwd_workspace_bytes(4, 64)
    a = dict(dy=D, ydt=1, lddy=64, x=D, xdt=1, rows=4, D=64, ldx=64, mean=D, rstd=D, gamma=D, wdt=0,
             dres=D, lddres=64, dx=D, lddx=64, dgamma=D, dbeta=D, ws=D, nws=need)
    a.update(kw)
    return L.tbn_layernorm_bwd(*a.values(), None)


def test_layernorm_bwd_refusals(L):
    need = L.tbn_layernorm_bwd_workspace_bytes(4, 64)
    assert need >= 2 * 64 * 4
    assert L.tbn_layernorm_bwd_workspace_bytes(-1, 64) == 0
    assert L.tbn_layernorm_bwd_workspace_bytes(4, 0) == 0
    for kw in (dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(rows=-1),
               dict(D=0), dict(lddy=63), dict(lddx=63), dict(lddres=63), dict(ws=None), dict(nws=need - 1),
               dict(xdt=3)):
        assert _norm_bwd(L, **kw) == INVALID, kw
    assert _norm_bwd(L, ydt=0) == UNSUPPORTED
    odd = ctypes.c_void_p((1 << 20) + 1)
    for kw in (dict(dy=odd), dict(dres=odd), dict(dgamma=odd), dict(ws=ctypes.c_void_p((1 << 20) + 8))):
        assert _norm_bwd(L, **kw) == MISALIGNED, kw


def _adamw(L, hyper=None, count=1, **kw):
    t = (tbn.AdamWTensor * 1)()
    a = dict(param=1 << 20, grad=1 << 21, m=1 << 22, v=1 << 23, n=8, weight_decay=0.1, lr_scale=1.0)
    a.update(kw)
    for k, v in a.items():
        setattr(t[0], k, v)
    h = tbn.AdamWHyper(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    for k, v in (hyper or {}).items():
        setattr(h, k, v)
    return L.tbn_adamw_step(t, count, ctypes.byref(h), None)


def test_adamw_refusals(L):
    for h in (dict(lr=-0.1), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
              dict(beta2=math.nan), dict(eps=-1e-9), dict(step=0)):
        assert _adamw(L, h) == INVALID, h
    assert _adamw(L, dict(grad_scale=(1 << 20) + 2)) == MISALIGNED
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(param_dtype=2),
               dict(grad_dtype=-1), dict(state=2), dict(state=1), dict(state=1, m_scale=1 << 24),
               dict(weight_decay=-1.0), dict(lr_scale=math.nan)):
        assert _adamw(L, **kw) == INVALID, kw
    assert _adamw(L, n=(1 << 40) + 1) == UNSUPPORTED
    for kw in (dict(param=(1 << 20) + 2), dict(grad=(1 << 20) + 1, grad_dtype=1), dict(m=(1 << 20) + 2),
               dict(copy=(1 << 20) + 1), dict(state=1, m_scale=(1 << 20) + 1, v_scale=1 << 20)):
        assert _adamw(L, **kw) == MISALIGNED, kw
    assert L.tbn_adamw_step(None, 1, ctypes.byref(tbn.AdamWHyper()), None) == INVALID
    assert L.tbn_adamw_step(None, 0, None, None) == INVALID
    assert _adamw(L, count=-1) == INVALID
    # nothing to do: no tensor, or only empty ones
    assert _adamw(L, count=0) == OK
    assert _adamw(L, n=0, param=None, grad=None, m=None, v=None) == OK


def _adapter(L, backward=False, fields=None, **kw):
    ad = tbn.Adapters(a=1 << 20, b=1 << 21, n=2, r=8, K_in=64, K_out=128)
    for k, v in (fields or {}).items():
        setattr(ad, k, v)
    need = L.tbn_adapter_workspace_bytes(5, 64, 128, 2, 8, 1 if backward else 0)
    if backward:
        a = dict(dy=D, ydt=1, lddy=128, x=D, xdt=1, T=5, ldx=64, v=D, base=D, ldbase=64, dx=D, lddx=64,
                 da=D, db=D, ws=D, nws=need)
    else:
        a = dict(x=D, xdt=1, T=5, ldx=64, base=D, ldbase=128, y=D, ydt=1, ldy=128, v=D, ws=D, nws=need)
    a.update(kw)
    call = L.tbn_adapter_bwd if backward else L.tbn_adapter_fwd
    return call(ctypes.byref(ad), *a.values(), None)


@pytest.mark.parametrize("backward", [False, True])
def test_adapter_refusals(L, backward):
    run = lambda fields=None, **kw: _adapter(L, backward, fields, **kw)  # noqa: E731
    need = L.tbn_adapter_workspace_bytes(5, 64, 128, 2, 8, 1 if backward else 0)
    for f in (dict(a=None), dict(b=None), dict(n=0), dict(r=0), dict(K_in=0), dict(K_out=-1)):
        assert run(f) == INVALID, f
    for f in (dict(n=1024), dict(r=129), dict(K_in=(1 << 22) + 1), dict(K_out=1 << 40)):
        assert run(f) == UNSUPPORTED, f
    assert run(T=1 << 31) == UNSUPPORTED and run(T=-1) == INVALID
    for f in (dict(a=(1 << 20) + 1), dict(ids=(1 << 20) + 2), dict(ranks=(1 << 20) + 1), dict(scale=(1 << 20) + 2)):
        assert run(f) == MISALIGNED, f
    wrong = [dict(x=None), dict(xdt=5), dict(ydt=-1), dict(ldx=63), dict(ldbase=3), dict(ws=None),
             dict(nws=need - 1)]
    wrong += [dict(dy=None), dict(lddy=127), dict(lddx=1)] if backward else [dict(y=None), dict(ldy=127)]
    for kw in wrong:
        assert run(**kw) == INVALID, kw
    assert run(ldx=1 << 45) == UNSUPPORTED
    odd = ctypes.c_void_p((1 << 20) + 1)
    for kw in (dict(x=odd), dict(base=odd), dict(v=odd), dict(ws=ctypes.c_void_p((1 << 20) + 128))):
        assert run(**kw) == MISALIGNED, kw
    assert L.tbn_adapter_workspace_bytes(5, 64, 128, 0, 8, 0) == 0
    assert L.tbn_adapter_workspace_bytes(-1, 64, 128, 1, 8, 0) == 0
    assert L.tbn_adapter_workspace_bytes(5, 64, 128, 1, 129, 1) == 0
    if not backward:
        assert run(T=0, x=None, y=None) == OK
