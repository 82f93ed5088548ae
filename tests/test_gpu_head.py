"""The head of the tower inside torch's autograd, its functions together as a tower uses them, on other streams and in captured graphs."""
import math
import os
import sys

import pytest
import torch

from paper_2305_01515_b200 import binding as mb
from paper_2305_01515_b200 import head as hd
from paper_2305_01515_b200 import sequence as sq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def rms64(x, w, res=None, eps=1e-6):
    r = x if res is None else x + res
    return r / (r.square().mean(1, keepdim=True) + eps).sqrt() * w, r


def near(got, want, units):
    """Within `units` of 2^-24 of the largest value."""
    assert got.shape == want.shape
    assert float((got.double() - want).abs().max()) <= units * 2.0 ** -24 * max(float(want.abs().max()), 1e-30)


@pytest.mark.parametrize("residual", [False, True])
def test_rms_norm_in_autograd(residual):
    g = torch.Generator(device=DEV).manual_seed(0)
    both = torch.randn(37, 2 * 200, generator=g, device=DEV).requires_grad_()
    w = torch.randn(200, generator=g, device=DEV).requires_grad_()
    a, b = torch.randn(37, 200, generator=g, device=DEV), torch.randn(37, 200, generator=g, device=DEV)
    x, res = both.chunk(2, 1)                                # column ranges of one projection
    got = hd.rms_norm(x, w, res if residual else None)
    out, total = got if residual else (got, None)
    loss = (out * a).sum() + ((total * b).sum() if residual else 0.0)
    grads = torch.autograd.grad(loss, (both, w))
    b64, w64 = both.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    x64, r64 = b64.chunk(2, 1)
    o64, t64 = rms64(x64, w64, r64 if residual else None)
    want = torch.autograd.grad((o64 * a.double()).sum() + ((t64 * b.double()).sum() if residual else 0.0), (b64, w64))
    near(out.detach(), o64.detach(), 100)
    for x_, y_ in zip(grads, want):                          # sums of 200 and of 37 terms
        near(x_, y_, 400)


def test_only_some_outputs_and_inputs_take_part():
    x, res = torch.randn(9, 40, device=DEV).requires_grad_(), torch.randn(9, 40, device=DEV).requires_grad_()
    w = torch.ones(40, device=DEV).requires_grad_()
    out, total = hd.rms_norm(x, w, res)
    dx, dr, dw = torch.autograd.grad(total.sum(), (x, res, w), allow_unused=True, retain_graph=True)
    assert bool((dx == 1).all()) and bool((dr == 1).all()) and dw is None
    out.sum().backward()                                     # an expanded gradient, of all ones
    assert torch.equal(x.grad, res.grad) and x.grad.data_ptr() != res.grad.data_ptr() and w.grad is not None
    out = hd.rms_norm(x.detach(), w)
    out.sum().backward()
    assert not hd.rms_norm(x.detach(), w.detach()).requires_grad
    assert not any(t.requires_grad for t in hd.rms_norm(x.detach(), w.detach(), res.detach()))


def test_log_probs_in_autograd():
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(21, 1003, generator=g, device=DEV).requires_grad_()
    t = torch.randint(-1, 1003, (21,), generator=g, device=DEV)
    a, b = torch.randn(21, generator=g, device=DEV), torch.randn(21, generator=g, device=DEV)
    r = hd.log_probs(x, t, top_k=4, scale=1.5)
    assert r.logp.requires_grad and r.entropy.requires_grad and not r.top_logp.requires_grad and r.top_index.dtype == torch.int64
    x64 = x.detach().double().requires_grad_()
    log = torch.log_softmax(x64 * 1.5, 1)
    l64 = torch.where(t < 0, 0.0, log.gather(1, t.clamp(min=0).unsqueeze(1))[:, 0])
    h64 = -(log.exp() * log).sum(1)
    for fa, fb in ((1, 1), (1, 0), (0, 1)):
        (got,) = torch.autograd.grad(fa * (r.logp * a).sum() + fb * (r.entropy * b).sum() if fa and fb else (r.logp * a).sum() if fa else (r.entropy * b).sum(), x,
                                     retain_graph=True)
        (want,) = torch.autograd.grad(fa * (l64 * a.double()).sum() + fb * (h64 * b.double()).sum(), x64, retain_graph=True)
        near(got, want, 400)
    near(r.logp.detach(), l64.detach(), 400)
    near(r.entropy.detach(), h64.detach(), 400)
    none = hd.log_probs(x.detach())
    assert none.logp is None and none.top_index is None and torch.equal(none.entropy, r.entropy) is False


def test_distillation_in_autograd():
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(13, 2000, generator=g, device=DEV).requires_grad_()
    index = torch.rand(13, 2000, generator=g, device=DEV).topk(20, 1)[1]
    teacher, rest, w = torch.randn(13, 20, generator=g, device=DEV), torch.randn(13, generator=g, device=DEV), torch.rand(13, generator=g, device=DEV)
    loss = hd.distill_loss(x, index, teacher, rest, scale=0.5)
    (got,) = torch.autograd.grad((loss * w).sum(), x, retain_graph=True)
    (twice,) = torch.autograd.grad((loss * w).sum(), x)      # the graph can be used again
    both, grad = hd.distill_loss_and_grad(x, index, teacher, rest, w, scale=0.5)
    assert torch.equal(both, loss.detach()) and torch.equal(grad, got) and torch.equal(twice, got) and not grad.requires_grad
    x64 = x.detach().double().requires_grad_()
    log = torch.log_softmax(x64 * 0.5, 1)
    q = torch.softmax(torch.cat([teacher.double() * 0.5, rest.double().unsqueeze(1)], 1), 1)
    others = torch.logsumexp(log.scatter(1, index, -math.inf), 1, keepdim=True)
    l64 = (q * (q.log() - torch.cat([log.gather(1, index), others], 1))).sum(1)
    (want,) = torch.autograd.grad((l64 * w.double()).sum(), x64)
    near(loss.detach(), l64.detach(), 400)
    near(got, want, 400)


def test_second_derivatives_are_refused():
    x = torch.randn(4, 60, device=DEV).requires_grad_()
    w = torch.ones(60, device=DEV)
    t, index = torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, 1, dtype=torch.int64, device=DEV)
    for out in (hd.rms_norm(x, w).square().sum(), hd.log_probs(x, t).logp.square().sum(), hd.distill_loss(x, index, torch.zeros(4, 1, device=DEV)).square().sum()):
        (d,) = torch.autograd.grad(out, x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            d.sum().backward()


def test_refusals():
    x, w, t = torch.zeros(4, 8, device=DEV), torch.ones(8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    index, teacher = torch.zeros(4, 3, dtype=torch.int64, device=DEV), torch.zeros(4, 3, device=DEV)
    for fn in (lambda: hd.rms_norm(x[0], w), lambda: hd.rms_norm(x, w[:4]), lambda: hd.rms_norm(x, w.cpu()), lambda: hd.rms_norm(x, w, x.half()),
               lambda: hd.rms_norm(x, w, x[:2]), lambda: hd.rms_norm(x, w, x.cpu()), lambda: hd.rms_norm_8bit(x.clone().requires_grad_(), w),
               lambda: hd.rows_from_8bit(x, w), lambda: hd.rows_from_8bit(x.to(torch.float8_e4m3fn), torch.zeros(4, 2, device=DEV)),
               lambda: hd.rows_from_8bit(x.to(torch.float8_e4m3fn), torch.zeros(4, 1)),
               lambda: hd.log_probs(x, t[:3]), lambda: hd.log_probs(x, t.int()), lambda: hd.log_probs(x, t.cpu()), lambda: hd.log_probs(x[0]),
               lambda: hd.distill_loss(x, index[:3], teacher), lambda: hd.distill_loss(x, index.int(), teacher), lambda: hd.distill_loss(x, index, teacher[:, :2]),
               lambda: hd.distill_loss(x, index, teacher.cpu()), lambda: hd.distill_loss(x, index.cpu(), teacher), lambda: hd.distill_loss(x, index, teacher, w),
               lambda: hd.distill_loss(x, index, teacher.clone().requires_grad_()), lambda: hd.distill_loss_and_grad(x, index, teacher, weights=w),
               lambda: hd.distill_loss_and_grad(x, index, teacher, weights=torch.ones(4))):
        with pytest.raises(ValueError):
            fn()
    for fn in (lambda: hd.rms_norm(x.double(), w), lambda: hd.log_probs(x.double()), lambda: hd.distill_loss(x, index, teacher.double()), lambda: hd.rms_norm(x, w.long()),
               lambda: hd.rows_from_8bit(x.to(torch.float8_e4m3fn), torch.zeros(4, 1, device=DEV), dtype=torch.float64)):
        with pytest.raises(TypeError):
            fn()
    for fn in (lambda: hd.log_probs(x, t, top_k=9), lambda: hd.log_probs(x, t, scale=0.0), lambda: hd.rms_norm(x, w, eps=-1.0), lambda: hd.rms_norm_8bit(x, w, group=48),
               lambda: hd.log_probs(x, t, top_k=-1)):
        with pytest.raises(mb.MtsError):
            fn()


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

    x, w, t = torch.randn(4, 8, device=DEV).requires_grad_(), torch.ones(8, device=DEV).requires_grad_(), torch.zeros(4, dtype=torch.int64, device=DEV)
    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
    monkeypatch.setattr(torch.cuda, "device", Guard)

    def seen(fn):
        del asked[:], entered[:]
        result = fn()
        assert entered and asked and all(d == x.device for d in asked + entered), (asked, entered)
        return result

    out = seen(lambda: hd.rms_norm(x, w))
    seen(lambda: out.sum().backward())
    codes, scales = seen(lambda: hd.rms_norm_8bit(x.detach(), w.detach()))
    seen(lambda: hd.rows_from_8bit(codes, scales))
    r = seen(lambda: hd.log_probs(x, t))
    seen(lambda: r.logp.sum().backward())
    loss = seen(lambda: hd.distill_loss(x, t.unsqueeze(1), torch.zeros(4, 1, device=DEV)))
    seen(lambda: loss.sum().backward())
    seen(lambda: hd.distill_loss_and_grad(x, t.unsqueeze(1), torch.zeros(4, 1, device=DEV)))


class Head(torch.nn.Module):
    """Two layers on a residual stream and the scores over a catalogue."""

    def __init__(self, D, V, seed, dtype=torch.float32):
        super().__init__()
        g = torch.Generator(device=DEV).manual_seed(seed)
        new = lambda *s: torch.nn.Parameter((torch.randn(*s, generator=g, device=DEV) * s[0] ** -0.5).to(dtype))  # noqa: E731
        self.a, self.b, self.items = new(D, D), new(D, D), new(D, V)
        self.w = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(D, device=DEV, dtype=dtype)) for _ in range(3)])

    def scores(self, x, norm):
        y, _ = norm(x, self.w[0], None)
        y, stream = norm(y @ self.a, self.w[1], x)
        y, stream = norm(torch.tanh(y) @ self.b, self.w[2], stream)
        return y @ self.items


def own_norm(x, w, res):
    return (hd.rms_norm(x, w), x) if res is None else hd.rms_norm(x, w, res)


def losses(head, x, t, index, teacher, rest):
    scores = head.scores(x, own_norm)
    r = hd.log_probs(scores, t, top_k=5)
    return -r.logp.mean() - 0.01 * r.entropy.mean() + hd.distill_loss(scores, index, teacher, rest, scale=0.5).mean(), r


def test_a_tower_trained_by_all_of_them_together():
    """Gradients of every parameter through norms, log probabilities, entropy and distillation, against the same in torch in 64 bits."""
    D, V, N = 72, 1501, 50
    g = torch.Generator(device=DEV).manual_seed(5)
    head = Head(D, V, 6)
    x, t = torch.randn(N, D, generator=g, device=DEV), torch.randint(-1, V, (N,), generator=g, device=DEV)
    index, teacher, rest = torch.rand(N, V, generator=g, device=DEV).topk(9, 1)[1], torch.randn(N, 9, generator=g, device=DEV), torch.randn(N, generator=g, device=DEV)
    loss, r = losses(head, x, t, index, teacher, rest)
    loss.backward()
    wide = Head(D, V, 6).double()
    s = wide.scores(x.double(), lambda a, w, res: rms64(a, w, res))
    log = torch.log_softmax(s, 1)
    logp = torch.where(t < 0, 0.0, log.gather(1, t.clamp(min=0).unsqueeze(1))[:, 0])
    half = torch.log_softmax(s * 0.5, 1)
    q = torch.softmax(torch.cat([teacher.double() * 0.5, rest.double().unsqueeze(1)], 1), 1)
    others = torch.logsumexp(half.scatter(1, index, -math.inf), 1, keepdim=True)
    want = -logp.mean() + 0.01 * (log.exp() * log).sum(1).mean() + (q * (q.log() - torch.cat([half.gather(1, index), others], 1))).sum(1).mean()
    want.backward()
    # products of 72 and 1501 terms in fp32 on the way, the device's default for them
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-4
    for p, q_ in zip(head.parameters(), wide.parameters()):
        assert float((p.grad.double() - q_.grad).norm()) <= 1e-4 * float(q_.grad.norm())
    top = torch.sort(s.detach(), dim=1, descending=True)
    clear = (top[0][:, :5] - top[0][:, 1:6] > 1e-4).all(1)   # no two scores nearer than rounding
    assert torch.equal(r.top_index[clear], top[1][clear][:, :5]) and float(clear.float().mean()) > 0.5
    opt = sq.AdamW(list(head.parameters()), lr=1e-3)
    opt.step()                                               # the gradients are what the optimizer takes


def test_serving_in_8_bits():
    """Single events through norms in 8 bits, scores and best items: near the same in full precision."""
    g = torch.Generator(device=DEV).manual_seed(9)
    head = Head(64, 900, 8, torch.bfloat16)
    x = torch.randn(3, 64, generator=g, device=DEV).bfloat16()
    with torch.no_grad():
        for group in (0, 32):
            codes, scales, stream = hd.rms_norm_8bit(x, head.w[0], x, group=group)
            y = hd.rows_from_8bit(codes, scales, group)
            full, total = hd.rms_norm(x, head.w[0], x)
            assert torch.equal(stream, total)
            # half a step of each code, of the largest where a code is below the normal numbers, and two roundings to bf16
            assert bool(((y - full).float().abs() <= full.float().abs() * (2.0 ** -4 + 2.0 ** -7) + 2e-4 * full.float().abs().amax(1, keepdim=True)).all())
            best = hd.log_probs(y @ head.items, top_k=10)
            assert best.top_index.shape == (3, 10) and bool((best.top_logp[:, :-1] >= best.top_logp[:, 1:]).all())


def test_on_another_stream():
    """Calls go to the current stream: a long product before them on that stream, and what waits for it sees their results."""
    g = torch.Generator(device=DEV).manual_seed(11)
    a = torch.randn(3000, 3000, generator=g, device=DEV)
    index, teacher, w = torch.zeros(3000, 1, dtype=torch.int64, device=DEV), torch.zeros(3000, 1, device=DEV), torch.ones(3000, device=DEV)
    want = a @ a @ a
    want = hd.rms_norm(want, w), hd.log_probs(want, index[:, 0], top_k=3), hd.distill_loss(want, index, teacher)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = a @ a @ a
        got = hd.rms_norm(b, w), hd.log_probs(b, index[:, 0], top_k=3), hd.distill_loss(b, index, teacher)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and all(torch.equal(p, q) for p, q in zip(got[1], want[1]))


def test_a_step_in_a_captured_graph():
    """Forward and backward captured and replayed on new inputs: what the same step gives outside, and two graphs side by side."""
    N, V = 16, 30001
    g = torch.Generator(device=DEV).manual_seed(12)
    weights = [torch.randn(V, generator=g, device=DEV).requires_grad_() for _ in range(2)]
    x, t = torch.zeros(N, V, device=DEV).requires_grad_(), torch.zeros(N, dtype=torch.int64, device=DEV)
    index, teacher, rest = torch.rand(N, V, generator=g, device=DEV).topk(9, 1)[1], torch.randn(N, 9, generator=g, device=DEV), torch.randn(N, generator=g, device=DEV)
    side, graphs, results = torch.cuda.Stream(), [], []

    def step(w):
        y, stream = hd.rms_norm(x, w, x)
        r = hd.log_probs(y, t, top_k=5)
        loss = hd.distill_loss(stream, index, teacher, rest)
        both, grad = hd.distill_loss_and_grad(y, index, teacher, None)
        return [r.logp, r.entropy, r.top_index, r.top_logp, loss, both, grad] + list(torch.autograd.grad(r.logp.sum() - r.entropy.sum() + loss.sum(), (x, w)))

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for w in weights:
            step(w)
    torch.cuda.current_stream().wait_stream(side)
    for w in weights:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(step(w))
        graphs.append(graph)
    for k in range(3):
        with torch.no_grad():
            x.copy_(torch.randn(N, V, generator=g, device=DEV))
        t.copy_(torch.randint(V, (N,), generator=g, device=DEV))
        torch.cuda.synchronize()
        for graph in graphs:                                 # both at once
            with torch.cuda.stream(torch.cuda.Stream()):
                graph.replay()
        torch.cuda.synchronize()
        for w, got in zip(weights, results):
            assert all(torch.equal(a, b) for a, b in zip(got, step(w)))


def test_results_are_the_same_in_every_run():
    g = torch.Generator(device=DEV).manual_seed(13)
    x = torch.randn(700, 5003, generator=g, device=DEV).bfloat16().requires_grad_()
    t, index = torch.randint(5003, (700,), generator=g, device=DEV), torch.rand(700, 5003, generator=g, device=DEV).topk(30, 1)[1]
    w = torch.randn(5003, generator=g, device=DEV).requires_grad_()
    first = None
    for _ in range(5):
        r = hd.log_probs(x, t, top_k=32)
        y = hd.rms_norm(x, w)
        loss = hd.distill_loss(x, index, torch.ones(700, 30, device=DEV))
        now = [r.logp, r.entropy, r.top_index, r.top_logp, y, loss] + list(torch.autograd.grad(r.logp.sum() + r.entropy.sum() + loss.sum() + y.float().square().sum(), (x, w)))
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_the_example_scores_a_catalogue():
    """The example's step on next items: its gradients against the same tower with torch's own norm and softmax, and that it runs, trains a table and serves."""
    import history_tower

    tower = history_tower.HistoryTower(rows=2000, S=12, L=24, seed=3, items=701)
    g = torch.Generator(device=DEV).manual_seed(4)
    indices, item = torch.randint(2000, (12 * 24,), generator=g, device=DEV), torch.randint(-1, 701, (12,), generator=g, device=DEV)
    teacher = (torch.rand(12, 701, generator=g, device=DEV).topk(9)[1], torch.randn(12, 9, generator=g, device=DEV), torch.randn(12, generator=g, device=DEV))
    with torch.no_grad():
        tower.p["bias"].copy_(torch.randn(tower.p["bias"].shape, generator=g, device=DEV))
    events = tower.table.forward(indices, tower.bag, 12 * 24).requires_grad_()
    leaves = [events, *tower.p.values()]
    got = torch.autograd.grad(tower.next_loss(events, item, teacher).sum(), leaves)
    read, state = tower.read(events)
    r = read + state
    scores = (r / (r.square().mean(1, keepdim=True) + 1e-6).sqrt() * tower.p["norm"]) @ tower.p["items"]
    logp = torch.where(item < 0, 0.0, torch.log_softmax(scores, 1).gather(1, item.clamp(min=0).unsqueeze(1))[:, 0])
    half = torch.log_softmax(scores * 0.5, 1)
    q = torch.softmax(torch.cat([teacher[1] * 0.5, teacher[2].unsqueeze(1)], 1), 1)
    others = torch.logsumexp(half.scatter(1, teacher[0], -math.inf), 1, keepdim=True)
    want = torch.autograd.grad((-logp + (q * (q.log() - torch.cat([half.gather(1, teacher[0]), others], 1))).sum(1)).sum(), leaves)
    for x, y in zip(got, want):                              # both in fp32, sums of up to 701 terms and products on the way
        assert float((x - y).norm()) <= 1e-4 * float(y.norm())
    before = tower.table.weights_numpy()
    assert all(math.isfinite(float(tower.next_step(indices, item, teacher))) for _ in range(3))
    assert (before != tower.table.weights_numpy()).any()
    best, logp = tower.recommend(indices, 5)
    assert best.shape == (12, 5) and bool((logp[:, :-1] >= logp[:, 1:]).all()) and bool(((best >= 0) & (best < 701)).all())
    tower.close()


def test_the_trace_tells_the_heads_kernels_apart():
    x, w, t = torch.randn(5, 64, device=DEV).requires_grad_(), torch.ones(64, device=DEV), torch.zeros(5, dtype=torch.int64, device=DEV)
    mb.trace_enable(True)
    try:
        codes, scales = hd.rms_norm_8bit(x.detach(), w)
        hd.rows_from_8bit(codes, scales)
        hd.rms_norm(x, w).sum().backward()
        hd.log_probs(x, t).logp.sum().backward()
        hd.distill_loss_and_grad(x, t.unsqueeze(1), torch.zeros(5, 1, device=DEV))
        launches = {k: v[1] for k, v in mb.trace_report().items()}
    finally:
        mb.trace_enable(False)
    assert launches == {"rms_norm_forward": 2, "rows_from_8bit": 1, "rms_norm_backward": 1, "logprobs_forward": 1, "logprobs_backward": 1, "distill_loss": 1}
