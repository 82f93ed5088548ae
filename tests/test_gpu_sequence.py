"""The tower's functions inside torch's autograd, against the same formulas in torch (64 bits), and the example that trains a table and a
tower together."""
import os
import sys

import pytest
import torch

from paper_2305_01515_b200 import binding as mb
from paper_2305_01515_b200 import sequence as sq

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def recurrence_64(gate, value, offsets, h0):
    h, out, final = None, [], []
    for s in range(len(offsets) - 1):
        h = h0[s]
        for t in range(offsets[s], offsets[s + 1]):
            h = h + torch.sigmoid(gate[t]) * (value[t] - h)
            out.append(h)
        final.append(h)
    return torch.stack(out), torch.stack(final)


def test_gated_recurrence_in_autograd():
    g = torch.Generator(device="cuda").manual_seed(0)
    off = [0, 5, 5, 30, 31]
    both = torch.randn(31, 2 * 24, generator=g, device="cuda").requires_grad_()
    h0 = torch.randn(4, 24, generator=g, device="cuda").requires_grad_()
    w, wf = torch.randn(31, 24, generator=g, device="cuda"), torch.randn(4, 24, generator=g, device="cuda")
    out, final = sq.gated_recurrence(*both.chunk(2, dim=1), torch.tensor(off, device="cuda"), h0)
    got = torch.autograd.grad((out * w).sum() + (final * wf).sum(), (both, h0))
    b64, h64 = both.detach().double().requires_grad_(), h0.detach().double().requires_grad_()
    o64, f64 = recurrence_64(*b64.chunk(2, dim=1), off, h64)
    want = torch.autograd.grad((o64 * w.double()).sum() + (f64 * wf.double()).sum(), (b64, h64))
    # 25 steps of values around 4 at most: a few hundred units of 2^-24 of sums of 25 terms
    assert float((out.double() - o64).abs().max()) < 1e-4 and float((final.double() - f64).abs().max()) < 1e-4
    for x, y in zip(got, want):
        assert float((x.double() - y).abs().max()) < 2e-3 * float(y.abs().max())


def test_relpos_bias_in_autograd():
    g = torch.Generator(device="cuda").manual_seed(1)
    buckets = mb.RelposBuckets(sq.log_bucket_starts(8, 20), two_sided=True)
    table = torch.randn(buckets.rows, 3, generator=g, device="cuda").requires_grad_()
    scores = torch.randn(5, 3, 33, 40, generator=g, device="cuda").requires_grad_()
    w = torch.randn(5, 3, 33, 40, generator=g, device="cuda")
    bias = sq.relpos_bias(table, buckets, 33, 40, q_offset=7)
    (a,) = torch.autograd.grad(((scores.detach() + bias) * w).sum(), table)
    d_scores, b = torch.autograd.grad((sq.add_relpos_bias(scores, table, buckets, q_offset=7) * w).sum(), (scores, table))
    assert torch.equal(d_scores, w)
    one = torch.zeros(buckets.rows, 3, dtype=torch.float64, device="cuda")
    for k in range(buckets.rows):            # every bucket on its own: the bias is linear in the table
        t = torch.zeros(buckets.rows, 3, device="cuda")
        t[k] = 1.0
        one[k] = (sq.relpos_bias(t, buckets, 33, 40, q_offset=7).double() * w.double().sum(0)).sum((1, 2))
    for x in (a, b):                         # sums of up to 6600 terms of size 4 at most, rounded in fp32 along the way
        assert float((x.double() - one).abs().max()) < 6600 * 4 * 1e-6


def test_log_bucket_starts():
    assert sq.log_bucket_starts(32, 128)[:17] == list(range(17)) and sq.log_bucket_starts(32, 128)[-1] == 128
    for n, far in ((1, 5), (2, 1), (8, 20), (16, 64), (33, 1000)):
        s = sq.log_bucket_starts(n, far)
        assert len(s) == n and s[0] == 0 and s == sorted(s) and (n < 3 or s[-1] == far)
    with pytest.raises(ValueError):
        sq.log_bucket_starts(32, 8)


@pytest.mark.parametrize("bits,masters,dtype", [(32, False, torch.float32), (8, False, torch.float32), (32, True, torch.bfloat16)])
def test_adamw_against_torch(bits, masters, dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    params = [torch.randn(*s, generator=g, device="cuda").to(dtype).requires_grad_() for s in ((300, 7), (11,), (64, 64))]
    other = [p.detach().double().requires_grad_() for p in params]
    mine = sq.AdamW(params, lr=1e-2, weight_decay=0.1, state_bits=bits, masters=masters)
    theirs = torch.optim.AdamW([dict(params=[p for p in other if p.dim() > 1]), dict(params=[p for p in other if p.dim() == 1], weight_decay=0.0)],
                               lr=1e-2, weight_decay=0.1)
    for k in range(5):
        for p, o in zip(params, other):
            p.grad = torch.randn(p.shape, generator=g, device="cuda").to(dtype)          # new gradient tensors every step
            o.grad = p.grad.double()
        mine.step()
        theirs.step()
    for k, (p, o) in enumerate(zip(params, other)):
        got = mine.masters[k].double() if masters else p.double()
        # 8 bits: an update of at most lr is off by half a code of m and of the root of v a step, about an eighth of it
        assert float((got.detach() - o.detach()).abs().max()) < (5 * 1e-2 * 0.2 if bits == 8 else 1e-5)


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    off = torch.tensor([0, 4], device="cuda")
    for args in ((x, x[:, :4], off), (x, x.half(), off), (x, x, off.int()), (x, x, off.cpu()), (x, x, off, torch.zeros(2, 8, device="cuda"))):
        with pytest.raises(ValueError):
            sq.gated_recurrence(*args)
    with pytest.raises(TypeError):
        sq.gated_recurrence(x.double(), x.double(), off)
    with pytest.raises(ValueError):
        sq.relpos_bias(x, mb.RelposBuckets([0, 1]), 3, 3)
    with pytest.raises(ValueError):
        sq.AdamW([x.requires_grad_(), torch.zeros(3, device="cuda").half()])


def test_example_trains_a_table_and_a_tower():
    import history_tower

    tower = history_tower.HistoryTower(rows=3000, S=16, L=40, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    indices = torch.randint(3000, (16 * 40,), generator=g, device="cuda")
    target = torch.randn(16, tower.D, generator=g, device="cuda")
    before = tower.table.weights_numpy()
    losses = [float(tower.step(indices, target)) for _ in range(25)]
    after = tower.table.weights_numpy()
    assert losses[-1] < 0.5 * losses[0], losses
    assert (before != after).any() and tower.table.tables.status() == 0
    touched = set(indices.cpu().tolist())
    rows = (before.reshape(3000, -1) != after.reshape(3000, -1)).any(1)
    assert all(not rows[r] for r in range(3000) if r not in touched)
    tower.close()


def test_recurrence_refuses_arguments_on_another_device():
    x, off = torch.zeros(4, 8, device="cuda"), torch.tensor([0, 4], device="cuda")
    for args in ((x, x.cpu(), off), (x.cpu(), x, off), (x, x, off, torch.zeros(1, 8)), (x.cpu(), x.cpu(), off)):
        with pytest.raises(ValueError):
            sq.gated_recurrence(*args)
    sq.gated_recurrence(x, x, off, torch.zeros(1, 8, device="cuda"))


def test_adamw_refuses_arguments_that_the_kernel_cannot_read():
    w = torch.ones(5, 8, device="cuda").requires_grad_()
    with pytest.raises(ValueError):
        sq.AdamW([w, torch.zeros(3)])
    with pytest.raises(ValueError):
        sq.AdamW([torch.zeros(3), w])
    opt = sq.AdamW([w], lr=0.1, weight_decay=0.0)
    w.grad = torch.ones_like(w)
    for bad in (torch.tensor(0.5), torch.tensor(0.5, dtype=torch.float64, device="cuda"), torch.tensor(0.5, dtype=torch.float16, device="cuda"),
                torch.ones(2, device="cuda"), torch.ones(0, device="cuda")):
        with pytest.raises(ValueError):
            opt.step(grad_scale=bad)
    assert opt.steps == 0 and torch.equal(w.detach(), torch.ones_like(w))
    opt.step(grad_scale=torch.tensor(0.5, device="cuda"))
    opt.step(grad_scale=torch.tensor([0.25], device="cuda"))
    assert opt.steps == 2 and float((w.detach() - 0.8).abs().max()) < 0.05


def test_bias_refuses_scores_that_do_not_fit():
    b = mb.RelposBuckets([0, 1, 2])
    table = torch.zeros(3, 2, device="cuda")
    with pytest.raises(TypeError):
        sq.relpos_bias(table, b, 4, 4, dtype=torch.float64)
    with pytest.raises(TypeError):
        sq.add_relpos_bias(torch.zeros(1, 2, 4, 4, device="cuda", dtype=torch.float64), table, b)
    for scores in (torch.zeros(2, 4, 4, device="cuda"), torch.zeros(1, 2, 4, 4)):
        with pytest.raises(ValueError):
            sq.add_relpos_bias(scores, table, b)


def test_gradients_of_broadcast_heads():
    """One head's table for all heads, and one head's scores for all tables: the gradients are summed over what was broadcast."""
    g = torch.Generator(device="cuda").manual_seed(7)
    b = mb.RelposBuckets([0, 1, 3], two_sided=True)
    w = torch.randn(2, 3, 9, 10, generator=g, device="cuda")
    for hs, ht in ((3, 1), (1, 3)):
        scores = torch.randn(2, hs, 9, 10, generator=g, device="cuda").requires_grad_()
        table = torch.randn(b.rows, ht, generator=g, device="cuda").requires_grad_()
        ds, dt = torch.autograd.grad((sq.add_relpos_bias(scores, table, b) * w).sum(), (scores, table))
        full = torch.zeros(b.rows, 3, device="cuda").requires_grad_()
        (df,) = torch.autograd.grad((sq.add_relpos_bias(torch.zeros_like(w), full, b) * w).sum(), full)
        assert torch.equal(ds, w if hs == 3 else w.sum(1, keepdim=True))
        assert dt.shape == table.shape and torch.equal(dt, df if ht == 3 else df.sum(1, keepdim=True))


def test_calls_go_to_the_tensors_device(monkeypatch):
    """Stream and device of every call are those of the tensors, not the current ones (seen on the host: one GPU is enough)."""
    asked, entered = [], []
    current, guard = torch.cuda.current_stream, torch.cuda.device

    class Guard(guard):
        def __init__(self, device):
            entered.append(device)
            super().__init__(device)

    def current_stream(device=None):
        asked.append(device)
        return current(device)

    x = torch.zeros(4, 8, device="cuda").requires_grad_()
    table = torch.zeros(2, 3, device="cuda").requires_grad_()
    scores, off, b = torch.zeros(1, 3, 4, 4, device="cuda"), torch.tensor([0, 4], device="cuda"), mb.RelposBuckets([0, 1])
    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
    monkeypatch.setattr(torch.cuda, "device", Guard)

    def seen(fn):
        del asked[:], entered[:]
        result = fn()
        assert entered and all(d == x.device for d in asked + entered), (asked, entered)
        return result

    h, _ = seen(lambda: sq.gated_recurrence(x, x.detach(), off))
    seen(lambda: h.sum().backward())
    bias = seen(lambda: sq.add_relpos_bias(scores, table, b))
    seen(lambda: bias.sum().backward())
    opt = seen(lambda: sq.AdamW([x, table]))
    seen(opt.step)
    assert asked == [x.device]


def test_second_derivative_of_the_recurrence_is_refused():
    """Its gradient has no graph; a penalty on it must not vanish without a word."""
    x = torch.randn(6, 8, device="cuda").requires_grad_()
    h, _ = sq.gated_recurrence(x, x, torch.tensor([0, 6], device="cuda"))
    (d,) = torch.autograd.grad(h.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (h.sum() + d.square().sum()).backward()


@pytest.mark.parametrize("two_sided,causal", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("added", [True, False])
def test_second_derivatives_of_the_bias(two_sided, causal, added):
    """A loss with a penalty on the gradients of the table and of the scores, against the same bias by indexing in 64 bits.  2 heads x 2 x 7 x 9 places of
    values around 3 at most: sums of a few hundred terms below 100, u = 2^-24 each, pass through at most three products."""
    g = torch.Generator(device="cuda").manual_seed(9)
    starts, off, Lq, Lk = [0, 1, 2, 4], 3, 7, 9
    b = mb.RelposBuckets(starts, two_sided, causal)
    r = torch.arange(Lk)[None, :] - torch.arange(Lq)[:, None] - off
    d = r.abs() if two_sided else (-r).clamp(min=0)
    k = torch.bucketize(d, torch.tensor(starts), right=True) - 1
    k = (torch.where(r > 0, k + 4, k) if two_sided else k).cuda()
    seen = torch.ones_like(k, dtype=torch.bool) if not causal else (r <= 0).cuda()
    scores = torch.randn(2, 2, Lq, Lk, generator=g, device="cuda").requires_grad_()
    table = torch.randn(b.rows, 2, generator=g, device="cuda").requires_grad_()
    s64, t64 = scores.detach().double().requires_grad_(), table.detach().double().requires_grad_()

    def loss(s, t, own):
        if own:
            x = sq.add_relpos_bias(s, t, b, off) if added else s + sq.relpos_bias(t, b, Lq, Lk, off)
        else:
            x = s + torch.where(seen, t.t()[:, k], float("-inf"))
        x = torch.where(seen, x, 0.0)
        ds, dt = torch.autograd.grad(x.square().sum() + x.sum(), (s, t), create_graph=True)
        return x.sum() + dt.square().sum() * 0.01 + ds.square().sum()

    got = torch.autograd.grad(loss(scores, table, True), (scores, table))
    want = torch.autograd.grad(loss(s64, t64, False), (s64, t64))
    for x, y in zip(got, want):
        assert float((x.double() - y).abs().max()) <= 1e-4 * max(1.0, float(y.abs().max()))
    assert float(want[1].abs().max()) > 1.0


def test_gradient_of_the_tables_gradient_in_16_bits():
    """What the mask hides gets 0, whatever the direction holds; values are the direction's, rounded once."""
    b = mb.RelposBuckets([0, 2], causal=True)
    grad = torch.randn(3, 1, 5, 6, device="cuda").bfloat16().requires_grad_()
    dt = sq._TableGradient.apply(grad, b, 1)
    way = torch.tensor([[float("inf")], [0.3]], device="cuda")
    (dd,) = torch.autograd.grad(dt, grad, way)
    r = torch.arange(6)[None, :] - torch.arange(5)[:, None] - 1
    want = torch.where(r > 0, 0.0, torch.where(r > -2, float("inf"), 0.3)).bfloat16().cuda()
    assert dd.dtype == torch.bfloat16 and torch.equal(dd, want.expand(3, 1, 5, 6))


@pytest.mark.parametrize("masters,dtype", [(False, torch.float32), (True, torch.bfloat16)])
def test_adamw_follows_a_parameter_whose_storage_is_replaced(masters, dtype):
    """The same steps with and without moving a parameter between them: the same values, and the old storage stays as it was."""
    results = []
    for move in (False, True):
        g = torch.Generator(device="cuda").manual_seed(5)
        params = [torch.randn(40, 9, generator=g, device="cuda").to(dtype).requires_grad_() for _ in range(3)]
        opt = sq.AdamW(params, lr=1e-2, masters=masters)
        for k in range(4):
            if move and k == 2:
                old = params[1].data
                params[1].data = old.clone()
                kept = old.clone()
            for p in params:
                p.grad.copy_(torch.randn(40, 9, generator=g, device="cuda"))
            opt.step()
        if move:
            assert torch.equal(old, kept) and not torch.equal(params[1].data, kept)
        results.append([p.detach().clone() for p in params] + (opt.masters or []))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_adamw_takes_loaded_weights_into_its_masters():
    w = torch.randn(30, 8, device="cuda").bfloat16().requires_grad_()
    opt = sq.AdamW([w], lr=1e-3, weight_decay=0.0, masters=True)
    w.grad.fill_(1.0)
    for _ in range(3):
        opt.step()
    fine = opt.masters[0].clone()
    opt.refresh_masters()
    assert torch.equal(opt.masters[0], fine)               # they round to the parameter: nothing to take
    with torch.no_grad():
        w[:10] = 5.0                                       # in place
        opt.refresh_masters()
    assert bool((opt.masters[0][:10] == 5.0).all()) and torch.equal(opt.masters[0][10:], fine[10:])
    w.data = torch.full_like(w, 7.0)                       # other storage: taken at the next step
    opt.step()
    assert float((opt.masters[0] - 7.0).abs().max()) < 2e-3


def test_adamw_refuses_shared_and_changed_parameters():
    w = torch.ones(6, 8, device="cuda")
    a, b = w[:4].detach(), w[3:].detach()
    for params in ([w, w], [a, b], [w, a]):
        with pytest.raises(ValueError):
            sq.AdamW([p.requires_grad_() for p in params])
    p = torch.ones(6, 8, device="cuda").requires_grad_()
    q = torch.ones(6, 8, device="cuda").requires_grad_()
    opt = sq.AdamW([p, q])
    for bad in (torch.ones(5, 8, device="cuda"), torch.ones(8, 6, device="cuda").t(), q.data):
        p.grad = None
        p.data = bad
        p.grad = torch.ones_like(bad)
        with pytest.raises(ValueError):
            opt.step()
    assert opt.steps == 0 and bool((q == 1.0).all())


@pytest.mark.parametrize("S", [3, 80])                      # by chunks, and a thread for every channel of a sequence
def test_recurrence_reports_offsets_that_do_not_fit(S):
    x = torch.randn(60, 16, device="cuda").requires_grad_()
    good = torch.linspace(0, 60, S + 1).long().cuda()
    for k, bad in ((S, 59), (S, 61), (0, 1), (1, -3), (1, 45)):
        off = good.clone()
        off[k] = bad
        with pytest.raises(ValueError):
            sq.gated_recurrence(x, x, off, check=True)
    h, _ = sq.gated_recurrence(x, x, good, check=True)
    h.sum().backward()
    off = good.clone()                                     # changed between the two: the backward says so
    h, _ = sq._GatedRecurrence.apply(x, x, off, None, True)
    off.data[1] = 45
    with pytest.raises(ValueError):
        h.sum().backward()
