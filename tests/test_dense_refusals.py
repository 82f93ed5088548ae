"""Arguments that the entry points of the sequence tower refuse on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_2305_01515_b200 import binding as mb

P = 1 << 20                # an address that is never read: every call here is refused first


def refused(code, fn, *args, **kw):
    with pytest.raises(mb.MtsError) as e:
        fn(*args, **kw)
    assert e.value.code == code, e.value


def test_recurrence_forward():
    def call(gate=P, gs=64, value=P, vs=64, dtype=0, N=10, D=64, off=P, S=2, out=P, os=64, ws=P, wb=1 << 30):
        mb.recurrence_forward(gate, gs, value, vs, dtype, N, D, off, S, None, out, os, None, None, ws, wb)

    for kw in (dict(gate=None), dict(value=None), dict(out=None), dict(off=None), dict(dtype=3), dict(dtype=-1), dict(N=-1), dict(S=-1),
               dict(D=0), dict(gs=63), dict(vs=63), dict(os=10), dict(S=0)):
        refused(mb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(N=1 << 31), dict(S=1 << 31), dict(D=(1 << 20) + 1, gs=1 << 21, vs=1 << 21, os=1 << 21)):
        refused(mb.ERR_UNSUPPORTED, call, **kw)
    for kw in (dict(gate=P + 2), dict(value=P + 1), dict(out=P + 3), dict(ws=P + 64), dict(gate=P + 1, dtype=2)):
        refused(mb.ERR_ALIGNMENT, call, **kw)
    for kw in (dict(ws=None), dict(wb=0), dict(wb=mb.recurrence_workspace_bytes(10, 2, 64, 0) - 1)):
        refused(mb.ERR_WORKSPACE, call, **kw)


def test_recurrence_backward():
    def call(entry=P, grad=P, gs=64, dg=P, dv=P, ws=P, wb=1 << 30, N=10, off=P):
        mb.recurrence_backward(P, 64, P, 64, 0, N, 64, off, 2, None, entry, grad, gs, None, dg, 64, dv, 64, None, ws, wb)

    for kw in (dict(entry=None), dict(grad=None), dict(dg=None), dict(dv=None), dict(gs=1), dict(off=None), dict(N=-1)):
        refused(mb.ERR_INVALID_ARG, call, **kw)
    refused(mb.ERR_ALIGNMENT, call, dg=P + 2)
    refused(mb.ERR_WORKSPACE, call, wb=16)
    assert mb.lib().mts_recurrence_status(None, None, None) == mb.ERR_INVALID_ARG
    assert mb.recurrence_chunks(-1, 4, 0) == 0 and mb.recurrence_workspace_bytes(4, 4, 0, 0) == 0 and mb.recurrence_chunks(5, 4, 9) == 0
    assert mb.recurrence_chunks(0, 4, 0) == 0 and mb.recurrence_chunks(1, 4, 0) == 1


def test_relpos_buckets():
    def call(starts=(0, 1), table=P, td=0, H=2, Lq=4, Lk=8, off=0, out=P, od=0, hs=32, rs=8):
        mb.relpos_bias_forward(mb.RelposBuckets(starts), table, td, H, Lq, Lk, off, out, od, hs, rs)

    for kw in (dict(starts=()), dict(starts=(1, 2)), dict(starts=(0, 5, 4)), dict(starts=(-1, 0)), dict(table=None), dict(out=None), dict(td=3),
               dict(od=-1), dict(H=0), dict(Lq=-1), dict(Lk=-1), dict(rs=7), dict(hs=31), dict(hs=-32), dict(rs=-8)):
        refused(mb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(starts=range(129)), dict(H=65536), dict(Lq=1 << 29), dict(Lk=1 << 29), dict(off=1 << 29), dict(off=-(1 << 29))):
        refused(mb.ERR_UNSUPPORTED, call, **kw)
    refused(mb.ERR_ALIGNMENT, call, out=P + 2)
    refused(mb.ERR_ALIGNMENT, call, table=P + 1, td=1)
    assert mb.lib().mts_relpos_bias_forward(None, P, 0, 1, 1, 1, 0, P, 0, 1, 1, None) == mb.ERR_INVALID_ARG
    call(Lq=0)             # nothing to write: nothing is launched
    call(Lk=0)


def test_relpos_bucket_starts_that_do_not_fit():
    for far in (1 << 31, (1 << 32) + 5, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            mb.RelposBuckets((0, far))
    assert list(mb.RelposBuckets((0, (1 << 31) - 1))._starts) == [0, (1 << 31) - 1]


def test_relpos_gradient():
    b = mb.RelposBuckets((0, 1, 2), two_sided=True)
    need = mb.relpos_bias_workspace_bytes(b, 2)
    assert need > 0 and mb.relpos_bias_workspace_bytes(b, 0) == 0

    def call(grad=P, dtype=0, B=2, bs=64, out=P, ws=P, wb=need, H=2):
        mb.relpos_bias_backward(b, grad, dtype, B, H, 4, 8, 0, bs, 32, 8, out, ws, wb)

    for kw in (dict(grad=None), dict(out=None), dict(dtype=7), dict(B=-1), dict(bs=-1), dict(H=0)):
        refused(mb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(ws=None), dict(wb=need - 1)):
        refused(mb.ERR_WORKSPACE, call, **kw)
    for kw in (dict(grad=P + 1), dict(out=P + 2), dict(ws=P + 8)):
        refused(mb.ERR_ALIGNMENT, call, **kw)


def test_adamw():
    def create(sizes=(4,), pd=0, gd=0, bits=32, params=(P,), grads=(P,), masters=None):
        mb.AdamW(sizes, pd, gd, bits, params, grads, masters)

    for kw in (dict(sizes=(), params=(), grads=()), dict(sizes=(-1,)), dict(pd=3), dict(gd=-1), dict(bits=16), dict(params=(None,)),
               dict(grads=(None,)), dict(masters=(None,))):
        refused(mb.ERR_INVALID_ARG, create, **kw)
    for kw in (dict(params=(P + 2,)), dict(grads=(P + 1,)), dict(grads=(P + 1,), gd=2), dict(masters=(P + 2,), pd=2)):
        refused(mb.ERR_ALIGNMENT, create, **kw)
    refused(mb.ERR_UNSUPPORTED, create, sizes=(1 << 40,))
    L = mb.lib()
    assert L.mts_adamw_create(None, None) == mb.ERR_INVALID_ARG
    assert L.mts_adamw_step(None, None, 0, 0.1, 0.9, 0.999, 1e-8, 0.0, 1, None, 0, None) == mb.ERR_INVALID_ARG
    assert L.mts_adamw_export_state(None, None, 0, None, None, None) == mb.ERR_INVALID_ARG
    assert L.mts_adamw_import_state(None, None, 0, None, None, None) == mb.ERR_INVALID_ARG
    assert L.mts_adamw_set_grads(None, None, None) == mb.ERR_INVALID_ARG
    assert L.mts_adamw_state_bytes(None) == 0 and L.mts_adamw_state_elements(None) == 0 and L.mts_adamw_destroy(None) == mb.OK
    with pytest.raises(AssertionError):
        mb.AdamW((4, 4), 0, 0, 32, (P,), (P, P))


@pytest.mark.gpu
def test_adamw_handle_refusals():
    import torch

    x = torch.zeros(1000, device="cuda:0")
    h = mb.AdamW((1000,), 0, 0, 8, (x,), (x.clone(),))
    state = torch.zeros(h.state_bytes + 512, dtype=torch.uint8, device="cuda:0")
    step = lambda st, lr=0.1, b1=0.9, b2=0.9, eps=1e-8, wd=0.0, n=1: mb.adamw_step(h, st, lr, b1, b2, eps, wd, n)  # noqa: E731
    refused(mb.ERR_WORKSPACE, step, state[:h.state_bytes - 1])
    refused(mb.ERR_ALIGNMENT, step, state[16:])
    nan = float("nan")
    for kw in (dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1.0), dict(eps=nan), dict(lr=nan), dict(lr=float("inf")), dict(wd=nan),
               dict(n=0), dict(n=-5)):
        refused(mb.ERR_INVALID_ARG, step, state, **kw)
    m = torch.zeros(h.elements + 8, device="cuda:0")
    refused(mb.ERR_ALIGNMENT, mb.adamw_export_state, h, state, m[1:], m)
    refused(mb.ERR_INVALID_ARG, mb.adamw_export_state, h, state, None, m)
    refused(mb.ERR_INVALID_ARG, mb.adamw_import_state, h, state, m, None)
    with pytest.raises(AssertionError):
        mb.adamw_set_grads(h, [])
    refused(mb.ERR_ALIGNMENT, mb.adamw_set_grads, h, [x.data_ptr() + 1])
    assert float(x.abs().sum()) == 0.0


def test_adamw_counts_the_last_tensor_too():
    half = 1 << 39
    for sizes in ((half, half), (half, half - 1), ((1 << 40) - 1,)):     # with the gaps up to whole blocks 2^40 elements each
        refused(mb.ERR_UNSUPPORTED, mb.AdamW, sizes, 0, 0, 32, (P,) * len(sizes), (P,) * len(sizes))


@pytest.mark.gpu
def test_adamw_refuses_null_gradients_of_tensors_that_have_elements():
    import torch

    x, g = torch.ones(300, device="cuda:0"), torch.ones(300, device="cuda:0")
    h = mb.AdamW((0, 300), 0, 0, 32, (None, x), (None, g))
    refused(mb.ERR_INVALID_ARG, mb.adamw_set_grads, h, [None, None])
    refused(mb.ERR_INVALID_ARG, mb.adamw_set_grads, h, [g, None])
    state = torch.zeros(h.state_bytes, dtype=torch.uint8, device="cuda:0")
    mb.adamw_set_grads(h, [None, g])                       # nothing is read of an empty tensor
    mb.adamw_step(h, state, 0.1, 0.9, 0.999, 1e-8, 0.0, 1)
    torch.cuda.synchronize()
    assert float((x - 0.9).abs().max()) < 1e-6             # the first step of equal gradients is lr


@pytest.mark.gpu
def test_adamw_refuses_new_gradients_on_a_stream_under_capture():
    """A captured copy would read the host array of pointers when the graph runs, after it is gone.  The step itself can be captured."""
    import torch

    x, g = torch.zeros(300, device="cuda:0"), torch.ones(300, device="cuda:0")
    h = mb.AdamW((300,), 0, 0, 32, (x,), (g.clone(),))
    state = torch.zeros(h.state_bytes, dtype=torch.uint8, device="cuda:0")
    mb.adamw_set_grads(h, [g], torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        refused(mb.ERR_UNSUPPORTED, mb.adamw_set_grads, h, [g.data_ptr()], torch.cuda.current_stream())
        mb.adamw_step(h, state, 0.1, 0.9, 0.999, 1e-8, 0.0, 1, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert float(x.abs().max()) == 0.0
    graph.replay()
    torch.cuda.synchronize()
    assert float((x + 0.1).abs().max()) < 1e-6
