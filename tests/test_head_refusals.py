"""Arguments that the entry points of the tower's head refuse on the host, before anything is launched (no GPU needed)."""
import math

import pytest
import torch

from paper_2305_01515_b200 import binding as mb
from paper_2305_01515_b200 import head as hd

P = 1 << 20                # an address that is never read: every call here is refused first


def refused(code, fn, **kw):
    with pytest.raises(mb.MtsError) as e:
        fn(**kw)
    assert e.value.code == code, (kw, e.value)


def each(code, fn, *cases):
    for kw in cases:
        refused(code, fn, **kw)


def test_rms_norm_forward():
    def call(x=P, xs=64, r=None, rs=0, w=P, wd=0, dt=0, N=10, D=64, eps=1e-6, s=None, ss=0, out=P, os=64, inv=None):
        mb.rms_norm_forward(x, xs, r, rs, w, wd, dt, N, D, eps, s, ss, out, os, inv)

    each(mb.ERR_INVALID_ARG, call, dict(x=None), dict(w=None), dict(out=None), dict(dt=3), dict(wd=-1), dict(N=-1), dict(D=0), dict(xs=63), dict(os=63),
         dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(r=P, rs=64), dict(s=P, ss=64), dict(r=P, rs=63, s=P, ss=64), dict(r=P, rs=64, s=P, ss=1))
    each(mb.ERR_UNSUPPORTED, call, dict(N=1 << 31), dict(D=mb.RMS_NORM_MAX_D + 1, xs=1 << 20, os=1 << 20))
    each(mb.ERR_ALIGNMENT, call, dict(x=P + 2), dict(out=P + 1), dict(w=P + 2), dict(inv=P + 2), dict(x=P + 1, dt=2), dict(r=P + 2, rs=64, s=P, ss=64),
         dict(r=P, rs=64, s=P + 2, ss=64))


def test_rms_norm_8bit():
    def call(x=P, w=P, N=10, D=64, codes=P, cs=64, scales=P, group=32, xs=64):
        mb.rms_norm_forward_8bit(x, xs, None, 0, w, 0, 0, N, D, 1e-6, None, 0, codes, cs, scales, group, None)

    each(mb.ERR_INVALID_ARG, call, dict(x=None), dict(codes=None), dict(scales=None), dict(cs=63), dict(group=-1), dict(group=1), dict(group=48), dict(group=512),
         dict(group=16), dict(N=-1), dict(D=0), dict(xs=1))
    each(mb.ERR_ALIGNMENT, call, dict(scales=P + 2), dict(x=P + 1))
    each(mb.ERR_UNSUPPORTED, call, dict(N=1 << 31))

    def back(codes=P, cs=64, scales=P, group=0, N=10, D=64, out=P, dt=2, os=64):
        mb.rows_from_8bit(codes, cs, scales, group, N, D, out, dt, os)

    each(mb.ERR_INVALID_ARG, back, dict(codes=None), dict(scales=None), dict(out=None), dict(group=33), dict(dt=3), dict(N=-1), dict(D=0), dict(cs=63), dict(os=63))
    each(mb.ERR_ALIGNMENT, back, dict(scales=P + 1), dict(out=P + 1))
    each(mb.ERR_UNSUPPORTED, back, dict(N=1 << 31), dict(D=mb.RMS_NORM_MAX_D + 1, cs=1 << 20, os=1 << 20))


def test_rms_norm_backward():
    need = mb.rms_norm_workspace_bytes(10, 64)
    assert need > 0 and mb.rms_norm_workspace_bytes(-1, 64) == 0 and mb.rms_norm_workspace_bytes(10, 0) == 0

    def call(x=P, xs=64, w=P, N=10, D=64, inv=P, go=P, gos=64, gs=None, gss=0, dx=P, dxs=64, dw=P, ws=P, wb=need, dt=0):
        mb.rms_norm_backward(x, xs, w, 0, dt, N, D, inv, go, gos, gs, gss, dx, dxs, dw, ws, wb)

    each(mb.ERR_INVALID_ARG, call, dict(x=None), dict(w=None), dict(inv=None), dict(go=None), dict(dx=None), dict(xs=0), dict(gos=63), dict(gs=P, gss=63), dict(dxs=63),
         dict(dt=9), dict(N=-1), dict(D=-1))
    each(mb.ERR_WORKSPACE, call, dict(ws=None), dict(wb=need - 1))
    each(mb.ERR_ALIGNMENT, call, dict(ws=P + 128), dict(dw=P + 2), dict(inv=P + 1), dict(go=P + 2), dict(gs=P + 2, gss=64), dict(dx=P + 1))
    each(mb.ERR_UNSUPPORTED, call, dict(N=1 << 31), dict(D=mb.RMS_NORM_MAX_D + 1, xs=1 << 20, gos=1 << 20, dxs=1 << 20))


def test_logprobs():
    def call(x=P, st=100, dt=0, N=4, V=100, scale=1.0, t=P, k=5, lp=P, en=P, stt=P, ti=P, tl=P):
        mb.logprobs_forward(x, st, dt, N, V, scale, t, k, lp, en, stt, ti, tl)

    each(mb.ERR_INVALID_ARG, call, dict(x=None), dict(st=99), dict(dt=3), dict(N=-1), dict(V=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
         dict(scale=math.inf), dict(scale=2e30), dict(t=None), dict(k=-1), dict(k=6, V=5))
    each(mb.ERR_UNSUPPORTED, call, dict(N=100_000_001), dict(V=1_000_000_001, st=1 << 40), dict(k=mb.LOGPROBS_MAX_TOP + 1))
    each(mb.ERR_ALIGNMENT, call, dict(x=P + 2), dict(t=P + 4), dict(ti=P + 4), dict(lp=P + 2), dict(en=P + 1), dict(stt=P + 2), dict(tl=P + 2))

    def back(x=P, st=100, N=4, V=100, scale=1.0, t=P, stt=P, en=P, gl=P, gh=P, dx=P, ds=100, dt=0):
        mb.logprobs_backward(x, st, dt, N, V, scale, t, stt, en, gl, gh, dx, ds)

    each(mb.ERR_INVALID_ARG, back, dict(x=None), dict(dx=None), dict(stt=None), dict(t=None), dict(en=None), dict(ds=99), dict(st=99), dict(scale=0.0), dict(V=0),
         dict(dt=-1))
    each(mb.ERR_ALIGNMENT, back, dict(x=P + 1), dict(dx=P + 2), dict(t=P + 4), dict(stt=P + 2), dict(gl=P + 2), dict(gh=P + 2), dict(en=P + 2))
    each(mb.ERR_UNSUPPORTED, back, dict(N=100_000_001), dict(V=1_000_000_001, st=1 << 40, ds=1 << 40))


def test_distill_loss():
    def call(x=P, st=100, dt=0, N=4, V=100, scale=1.0, i=P, t=P, td=0, K=8, r=None, w=None, loss=P, dx=P, ds=100):
        mb.distill_loss(x, st, dt, N, V, scale, i, t, td, K, r, w, loss, dx, ds)

    each(mb.ERR_INVALID_ARG, call, dict(x=None), dict(i=None), dict(t=None), dict(loss=None, dx=None), dict(dt=3), dict(td=5), dict(N=-1), dict(V=0), dict(K=0),
         dict(K=-1), dict(scale=0.0), dict(scale=math.nan), dict(scale=2e30), dict(st=99), dict(ds=99))
    each(mb.ERR_UNSUPPORTED, call, dict(K=mb.DISTILL_MAX_K + 1), dict(N=100_000_001), dict(V=1_000_000_001, st=1 << 40, ds=1 << 40))
    each(mb.ERR_ALIGNMENT, call, dict(x=P + 2), dict(dx=P + 2), dict(i=P + 4), dict(t=P + 1), dict(t=P + 2), dict(r=P + 2), dict(w=P + 1), dict(loss=P + 2))


def test_torch_functions_refuse_tensors_that_are_not_on_a_gpu():
    x, w, i = torch.zeros(3, 8), torch.ones(8), torch.zeros(3, 2, dtype=torch.int64)
    for fn in (lambda: hd.rms_norm(x, w), lambda: hd.rms_norm_8bit(x, w), lambda: hd.log_probs(x), lambda: hd.distill_loss(x, i, torch.zeros(3, 2)),
               lambda: hd.distill_loss_and_grad(x, i, torch.zeros(3, 2)), lambda: hd.rows_from_8bit(x, w)):
        with pytest.raises(ValueError):
            fn()
