"""Loss against a teacher's best items (mts_distill_loss) and its gradient, against the formulas in 64 bits.

Units u = 2^-24.  As for log probabilities, the logarithms of the student's sums are off by L = (170 + V / 256 + 2 E[d]) u at most (of the sum over
the items that are not listed: with its own mean of d); the teacher's are sums of at most 257 terms, off by 300 u + 2 d u.  The loss is a sum of at most 257
terms q (log q - log p), each off by its factors' errors."""
import math

import pytest
import torch

from paper_2305_01515_b200 import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = (torch.float32, torch.float16, torch.bfloat16)
KIND = {torch.float32: mb.DTYPE_FP32, torch.float16: mb.DTYPE_FP16, torch.bfloat16: mb.DTYPE_BF16}
INF = math.inf


def placed(x, dtype, pad=0, shift=0):
    N, V = x.shape
    room = torch.full((shift + N * (V + pad) + 64,), 77.0, dtype=dtype, device=DEV)
    view = torch.as_strided(room, (N, V), (V + pad, 1), shift)
    view.copy_(x)
    return view, room


def call(x, index, teacher, rest=None, weights=None, scale=1.0, to=None, grad=True, loss=True):
    N, V = x.shape
    out = None if not grad else torch.full((N, V), 55.0, dtype=x.dtype, device=DEV) if to is None else to
    value = torch.full((N,), -9.0, device=DEV) if loss else None
    mb.distill_loss(x, x.stride(0), KIND[x.dtype], N, V, scale, index, teacher, KIND[teacher.dtype], index.shape[1], rest, weights, value, out,
                    V if out is None else out.stride(0))
    torch.cuda.synchronize()
    return value, out


def formula(x, index, teacher, rest, weights, scale):
    """(loss, its bound, gradient, its bound) in 64 bits."""
    N, V = x.shape
    x = x.double() * scale
    t = torch.where(index >= 0, teacher.double() * scale, -INF)
    r = torch.full((N, 1), -INF, dtype=torch.float64, device=DEV) if rest is None else rest.double().unsqueeze(1)
    both = torch.cat([t, r], 1)
    m = both.amax(1, keepdim=True)
    both = both - torch.where(m == -INF, 0.0, m)
    total = both.exp().sum(1, keepdim=True)
    any_ = total > 0
    q = torch.where(any_, both.exp() / total, 0.0)
    log_q = both - total.log()
    m = x.amax(1, keepdim=True)
    z = x - torch.where(m == -INF, 0.0, m)
    e = z.exp()
    S = e.sum(1, keepdim=True)
    p = torch.where(S > 0, e / S, 0.0)
    listed = torch.zeros(N, V + 1, dtype=torch.bool, device=DEV).scatter_(1, torch.where(index >= 0, index, V), True)[:, :V]
    others = torch.where(listed, 0.0, e).sum(1, keepdim=True)
    log_p = torch.cat([torch.where(index >= 0, z.gather(1, index.clamp(min=0)), -INF), others.log()], 1) - S.log()
    log_p = torch.where(S > 0, log_p, -INF)
    terms = torch.where(q > 0, q * (log_q - log_p), 0.0)
    loss = terms.sum(1)
    d = torch.where(e > 0, -z, 0.0)
    mean = lambda w: (w * d).sum(1, keepdim=True) / w.sum(1, keepdim=True).clamp(min=1e-300)  # noqa: E731
    off_s = (170 + V / 256 + 2 * mean(e)) * U
    off_o = (170 + V / 256 + 2 * mean(torch.where(listed, 0.0, e))) * U
    off_q = (300 + 4 * torch.where(both.isfinite(), -both, 0.0) + 2 * (q * torch.where(both.isfinite(), -both, 0.0)).sum(1, keepdim=True)) * U
    finite = lambda a: torch.where(a.isfinite(), a.abs(), 0.0)  # noqa: E731
    loss_bound = (q * (2 * off_q * (1 + finite(log_q) + finite(log_p)) + off_s + off_o + 8 * U * (finite(log_q) + finite(log_p)))).sum(1)
    want = torch.zeros(N, V + 1, dtype=torch.float64, device=DEV).scatter_add_(1, torch.where(index >= 0, index, V), q[:, :-1])[:, :V]
    off_want = torch.zeros(N, V + 1, dtype=torch.float64, device=DEV).scatter_add_(1, torch.where(index >= 0, index, V), (q * off_q)[:, :-1])[:, :V]
    share = torch.where(listed, 0.0, torch.where(others > 0, e / others, 0.0) * q[:, -1:])
    w = scale * (torch.ones(N, device=DEV) if weights is None else weights).double().unsqueeze(1)
    w = torch.where(any_, w, 0.0)
    g = w * torch.where(listed, p - want, p - share)
    off_e = (12 + 4 * d) * U
    bound = w.abs() * (p * (off_s + off_e) + off_want + want * 4 * U + share * (off_o + off_e + 2 * off_q[:, -1:])) + 4 * U * g.abs()
    return loss, loss_bound, g, bound


def close(got, want, bound):
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine) and torch.equal(got[~fine].double(), want[~fine])
    err = (got.double() - want).abs()[fine]
    assert bool((err <= bound[fine]).all()), (float((err - bound[fine]).max()), int((err > bound[fine]).sum()), got.shape)


def check(x, index, teacher, rest=None, weights=None, scale=1.0, to=None):
    loss, dx = call(x, index, teacher, rest, weights, scale, to)
    want, bound, g, g_bound = formula(x, index, teacher, rest, weights, scale)
    close(loss, want, bound)
    close(dx, g, g_bound + g.abs() * torch.finfo(x.dtype).eps / 2 + 2.0 ** -25 * (x.dtype == torch.float16) + 1e-37)
    alone, _ = call(x, index, teacher, rest, weights, scale, grad=False)
    _, only = call(x, index, teacher, rest, weights, scale, loss=False)
    assert torch.equal(alone, loss) and torch.equal(only, dx)
    return loss, dx


def places(N, V, K, g):
    """K different items for each row where there are as many, in no order."""
    return torch.rand(N, V, generator=g, device=DEV).topk(K, 1)[1] if K <= V else torch.randint(V, (N, K), generator=g, device=DEV)


SHAPES = [(1, 2, 1, 0, 0), (3, 7, 7, 0, 1), (4, 100, 5, 3, 3), (7, 255, 128, 0, 0), (5, 1001, 256, 0, 0), (40, 4096, 32, 0, 0), (9, 5001, 64, 7, 0), (3, 20000, 50, 0, 0),
          (160, 9000, 17, 0, 0), (3, 32003, 64, 0, 0), (2, 65536, 100, 8, 8), (300, 66001, 3, 0, 0), (1, 131072, 256, 0, 0), (2, 262145, 40, 1, 1), (1, 700001, 33, 0, 0), (2, 1100000, 20, 0, 0)]


@pytest.mark.parametrize("N,V,K,pad,shift", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_rest", [False, True])
def test_loss_and_gradient(N, V, K, pad, shift, dtype, with_rest):
    g = torch.Generator(device=DEV).manual_seed(N * 41 + V)
    x, _ = placed(2 * torch.randn(N, V, generator=g, device=DEV), dtype, pad, shift)
    index = places(N, V, K, g)
    teacher = (3 * torch.randn(N, K, generator=g, device=DEV)).to(dtype if N % 2 else torch.float32)
    if N > 2 and K > 2:
        index[1, 2:] = -1                                    # a row with fewer
        index[2] = -1                                        # and with none
        teacher[0, 1] = -INF
    rest = 2 * torch.randn(N, generator=g, device=DEV) if with_rest else None
    if with_rest and N > 2:
        rest[2] = -INF
    if with_rest and K == V:
        rest[:] = -INF                                       # every item is listed: there are no others
    weights = torch.randn(N, generator=g, device=DEV) if N % 2 == 0 else None
    to, room = placed(torch.zeros(N, V), dtype, 3, 2)
    _, dx = check(x, index, teacher, rest, weights, 1.0 if K % 2 else 0.6, to)
    mask = torch.ones_like(room, dtype=torch.bool)
    torch.as_strided(mask, to.shape, to.stride(), to.storage_offset()).fill_(False)
    assert bool((room[mask] == 77.0).all())
    same, _ = placed(x, dtype, pad, shift)                   # in place
    call(same, index, teacher, rest, weights, 1.0 if K % 2 else 0.6, same)
    assert torch.equal(same, dx)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 40000])
def test_items_that_the_student_rules_out(dtype, V):
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(6, V, generator=g, device=DEV)
    index = places(6, V, 8, g)
    x[0].masked_fill_(torch.rand(V, generator=g, device=DEV) < 0.5, -INF)
    x[0].scatter_(0, index[0], 1.0)                          # only others ruled out: a finite loss
    x[1, index[1, 3]] = -INF                                 # one that the teacher gives weight to
    x[2] = -INF                                              # all
    x[3] = torch.finfo(dtype).min                            # none by value: all alike
    x[4] = torch.finfo(dtype).min
    x[4].scatter_(0, index[4], 0.5)
    teacher = torch.randn(6, 8, generator=g, device=DEV)
    x = x.to(dtype)
    loss, dx = check(x, index, teacher)
    assert loss[[1, 2]].tolist() == [INF, INF] and bool(torch.isfinite(dx).all())
    rest = torch.zeros(6, device=DEV)
    x[5] = -INF
    x[5].scatter_(0, index[5], 0.5)                          # the others have nothing, the teacher gives them something
    loss, dx = check(x, index, teacher, rest)
    assert float(loss[5]) == INF and bool(torch.isfinite(dx).all())


def test_the_same_item_twice():
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(5, 700, generator=g, device=DEV)
    index = torch.randint(700, (5, 40), generator=g, device=DEV)
    index[0] = 13
    index[1, ::2] = 699
    teacher = torch.randn(5, 40, generator=g, device=DEV)
    check(x, index, teacher)
    check(x, index, teacher, torch.ones(5, device=DEV), scale=2.0)


def test_places_out_of_range_and_values_that_are_not_finite():
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(9, 3001, generator=g, device=DEV)
    index = places(9, 3001, 6, g)
    teacher = torch.randn(9, 6, generator=g, device=DEV)
    clean, clean_dx = call(x, index, teacher)
    bad, t = index.clone(), teacher.clone()
    y = x.clone()
    bad[0, 2] = 3001
    bad[1, 0] = 1 << 40
    bad[2, 5] = -(1 << 62)                                   # left out
    t[3, 1] = float("nan")
    t[4, 1] = INF
    y[5, 77] = float("nan")
    y[6, 77] = INF
    for rest in (None, torch.zeros(9, device=DEV)):
        loss, dx = call(y, bad, t, rest)
        for r in (0, 1, 3, 4, 5, 6):
            assert bool(loss[r].isnan()), r
        for r in (0, 1, 3, 4, 5):
            assert bool(dx[r].isnan().all()), r
        assert bool(dx[6].isnan().any())
        assert bool(torch.isfinite(loss[[2, 7, 8]]).all()) and bool(torch.isfinite(dx[[2, 7, 8]]).all())
    assert torch.equal(call(y, bad, t)[0][7:], clean[7:]) and torch.equal(call(y, bad, t)[1][7:], clean_dx[7:])
    loss, dx = call(y, bad, t, None, torch.zeros(9, device=DEV))
    assert bool((dx == 0).all())                             # rows of weight 0


def test_gradient_against_differences():
    """The 64-bit formula that the kernel is held to, against differences of the loss in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn(3, 9, generator=g, device=DEV, dtype=torch.float64)
    index = torch.tensor([[0, 4, 7], [3, 3, 1], [8, -1, 2]], device=DEV)
    teacher, rest, w = torch.randn(3, 3, generator=g, device=DEV), torch.randn(3, generator=g, device=DEV), torch.tensor([1.0, -0.5, 2.0], device=DEV)
    for r in (None, rest):
        _, _, want, _ = formula(x, index, teacher, r, w, 0.8)
        value = lambda y: float((formula(y, index, teacher, r, w, 0.8)[0] * w.double()).sum())  # noqa: E731
        for i in range(3):
            for j in range(9):
                e = torch.zeros_like(x)
                e[i, j] = 1e-6
                assert abs((value(x + e) - value(x - e)) / 2e-6 - float(want[i, j])) < 1e-8


def test_no_rows_and_rows_far_apart():
    mb.distill_loss(None, 10, 0, 0, 10, 1.0, None, None, 0, 3, None, None, torch.empty(0, device=DEV), None, 0)
    N, V, stride = 5, 2001, 500_000_000                     # places behind 2^31 elements and 2^32 bytes
    room = torch.zeros((N - 1) * stride + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(room, (N, V), (stride, 1))
    g = torch.Generator(device=DEV).manual_seed(8)
    x.copy_(torch.randn(N, V, generator=g, device=DEV))
    index, teacher = places(N, V, 12, g), torch.randn(N, 12, generator=g, device=DEV)
    _, dx = check(x, index, teacher, torch.zeros(N, device=DEV))
    call(x, index, teacher, torch.zeros(N, device=DEV), to=x)
    assert torch.equal(x, dx)


@pytest.mark.parametrize("V,dtype", [(900001, torch.float32), (1700003, torch.bfloat16)])
def test_rows_longer_than_the_bits_of_their_batches(V, dtype):
    """Too many rows for a cluster each, and listed items at a row's end, behind the batches that have a bit each."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x, _ = placed(torch.randn(75, V, generator=g, device=DEV), dtype, 0, 1)
    index = torch.randint(V, (75, 30), generator=g, device=DEV)
    index[:, 0] = V - 1 - torch.arange(75, device=DEV)
    index[:, 1] = V - 1
    index[:40, 2] = V - 2
    check(x, index, torch.randn(75, 30, generator=g, device=DEV), torch.randn(75, generator=g, device=DEV))


@pytest.mark.parametrize("N,V", [(600, 3001), (3, 60001)])
def test_results_are_the_same_in_every_run(N, V):
    """Listed items many to a batch and the same ones twice: the order in which threads find them does not matter."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V, generator=g, device=DEV).bfloat16()
    index = torch.randint(64, (N, 200), generator=g, device=DEV) * torch.randint(1, V // 64, (N, 1), generator=g, device=DEV)
    teacher, rest = torch.randn(N, 200, generator=g, device=DEV), torch.randn(N, generator=g, device=DEV)
    first = call(x, index, teacher, rest)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, call(x, index, teacher, rest)))


@pytest.mark.parametrize("mask", [-1e10, -1e30, "lowest"])
@pytest.mark.parametrize("scale", [0.25, 0.5, 1.0, 1e4, 1e10, 1e30])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [100, 3000, 70001])
def test_masks_of_large_finite_values_at_every_scale(mask, scale, dtype, V):
    """scale * score far beyond what fp32 has digits for, in some places, in whole threads' places and in whole rows; scores at scales up to the largest."""
    g = torch.Generator(device=DEV).manual_seed(V)
    low = torch.finfo(dtype).min
    low = low if mask == "lowest" else max(mask, low)
    x = 10 * torch.randn(6, V, generator=g, device=DEV)
    x[0].masked_fill_(torch.rand(V, generator=g, device=DEV) < 0.5, low)
    x[1, :V * 3 // 4] = low
    x[2] = low
    x[2, V // 3] = 7.0
    x[3] = low
    x[4, V // 2:] = low
    x = x.to(dtype)
    index = places(6, V, 8, g)
    index[2, 0] = V // 3
    scale = float(torch.tensor(scale, dtype=torch.float32))
    teacher = torch.randn(6, 8, generator=g, device=DEV) / scale
    weights = torch.full((6,), 1.0 / scale, device=DEV)
    loss, dx = call(x, index, teacher, None, weights, scale)
    want, bound, d, d_bound = formula(x, index, teacher, None, weights, scale)
    want = torch.where(want > torch.finfo(torch.float32).max, INF, want)     # weights of about 1/8 times up to 3.4e68: fp32 has no number for them
    close(loss, want, bound)
    close(dx, d, d_bound + d.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -25 * (dtype == torch.float16) + 1e-37)


def formula_of_far_items(x, index, teacher, rest, scale):
    """(loss, its bound, gradient, its bound) in 64 bits through logarithms, for listed items any distance above the others (all different, rest given).  The bounds are
    `formula`'s: the two logarithms of sums off by off_o and off_a, the teacher's by off_q, differences of logarithms rounded a few times."""
    V = x.shape[1]
    z = x.double() * scale
    listed = torch.zeros(x.shape, dtype=torch.bool, device=DEV).scatter_(1, index, True)
    others = z.masked_fill(listed, -INF)
    lse, lse_o = torch.logsumexp(z, 1, keepdim=True), torch.logsumexp(others, 1, keepdim=True)
    t = torch.cat([teacher.double() * scale, rest.double().unsqueeze(1)], 1)
    log_q = torch.log_softmax(t, 1)
    q = log_q.exp()
    log_p = torch.cat([z.gather(1, index), lse_o], 1) - lse
    loss = (q * (log_q - log_p)).sum(1)
    p, share = (z - lse).exp(), (others - lse_o).exp() * q[:, -1:]
    g = scale * (p - torch.where(listed, torch.zeros_like(p).scatter_(1, index, q[:, :-1]), share))
    mean = lambda w, top: (w * torch.where(w > 0, top - z, 0.0)).sum(1, keepdim=True)  # noqa: E731
    top, top_o = z.amax(1, keepdim=True), others.amax(1, keepdim=True)
    off_a = (170 + V / 256 + 2 * mean(p, top)) * U
    off_o = (170 + V / 256 + 2 * mean((others - lse_o).exp(), top_o)) * U
    far = t.amax(1, keepdim=True) - t
    off_q = (300 + 4 * far + 2 * (q * far).sum(1, keepdim=True)) * U
    loss_bound = (q * (2 * off_q * (1 + log_q.abs() + log_p.abs()) + off_a + off_o + 8 * U * (log_q.abs() + log_p.abs()))).sum(1)
    off_e = (12 + 4 * (torch.where(listed, top, top_o) - z)) * U
    p_rest = log_p[:, -1:].exp()
    part = torch.where(listed, 0.0, (others - lse_o).exp())        # of an other: (p_rest - q_rest) times this
    bound = scale * torch.where(listed, p * (off_a + off_e + (12 + 4 * (top - z)) * U) + q.new_zeros(p.shape).scatter_(1, index, (q * (off_q + 4 * U))[:, :-1]),
                                part * (p_rest * (off_a + off_o + (12 + 4 * (top - top_o)) * U) + q[:, -1:] * 2 * off_q[:, -1:] + (p_rest + q[:, -1:]) * (off_o + off_e)))
    return loss, loss_bound, g, bound + 4 * U * g.abs()


@pytest.mark.parametrize("above", [-40.0, 0.0, 60.0, 85.0, 100.0, 1000.0])
@pytest.mark.parametrize("scale", [0.5, 1.0, 8.0])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,K", [(5, 100, 3), (7, 3001, 50), (3, 70003, 20), (600, 9000, 33)])
def test_listed_items_far_above_the_others(above, scale, dtype, N, V, K):
    """The rest's place keeps its loss and the others their gradients however little the student gives them: the loss is infinite only where the student rules out all."""
    g = torch.Generator(device=DEV).manual_seed(V + K)
    x = torch.randn(N, V, generator=g, device=DEV)
    index = places(N, V, K, g)
    index[0] = torch.arange(K, device=DEV) + V - K               # at the row's end
    x.scatter_add_(1, index, torch.full((N, K), above / scale, device=DEV))
    x, _ = placed(x, dtype, 1, 3)
    teacher, rest = 2 * torch.randn(N, K, generator=g, device=DEV), scale + torch.randn(N, generator=g, device=DEV)
    loss, dx = call(x, index, teacher, rest, None, scale)
    want, bound, d, d_bound = formula_of_far_items(x, index, teacher, rest, scale)
    close(loss, want, bound)
    close(dx, d, d_bound + d.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -25 * (dtype == torch.float16) + 1e-37)


def test_formula_of_far_items_against_the_plain_one():
    g = torch.Generator(device=DEV).manual_seed(9)
    x = torch.randn(4, 60, generator=g, device=DEV)
    index, teacher, rest = places(4, 60, 5, g), torch.randn(4, 5, generator=g, device=DEV), torch.randn(4, generator=g, device=DEV)
    a, b = formula(x, index, teacher, rest, None, 0.8), formula_of_far_items(x, index, teacher, rest, 0.8)
    assert float((a[0] - b[0]).abs().max()) < 1e-12 and float((a[2] - b[2]).abs().max()) < 1e-12


@pytest.mark.parametrize("with_rest", [False, True])
@pytest.mark.parametrize("scale,size,apart", [(1.3e6, 10.0, 2.0 ** -20), (1000.0, 10.0, 1e-3), (1e-3, 1e4, 700.0), (1e30, 1e9, 100.0), (1e30, -1e9, 100.0), (1.0, -3e38, 2e31), (1e30, 0.0, 1e-30)])
def test_teachers_scores_at_large_scales(with_rest, scale, size, apart):
    """A teacher's scores whose product with the scale has no digits for their differences, or is no number of fp32: only differences count; the rest beside, above and
    below them."""
    g = torch.Generator(device=DEV).manual_seed(int(abs(size)) % 1000)
    N, V, K = 7, 900, 12
    scale = float(torch.tensor(scale, dtype=torch.float32))
    x = torch.randn(N, V, generator=g, device=DEV) / max(scale, 1.0)
    index = places(N, V, K, g)
    teacher = (size + apart * torch.randint(-4, 5, (N, K), generator=g, device=DEV).double()).float()
    rest = None
    if with_rest:
        rest = (teacher.double().amax(1) * scale + torch.tensor([0.0, 1.0, -1.0, 30.0, -30.0, 3e38, -3e38], device=DEV).double()).clamp(-3.4e38, 3.4e38).float()
    weights = torch.full((N,), 1.0 / max(scale, 1.0), device=DEV)
    check(x, index, teacher, rest, weights, scale)


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -124, 1e-30, 0.25])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_rest", [False, True])
def test_scores_whose_difference_is_no_number(scale, dtype, with_rest):
    """Scores of both signs up to the type's largest, the student's and the teacher's: their difference overflows, its product with a small scale does not."""
    g = torch.Generator(device=DEV).manual_seed(1)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    x = ((torch.rand(4, 3001, generator=g, device=DEV) * 2 - 1) * 3.3e38).to(dtype)
    index = places(4, 3001, 9, g)
    index[0, 0], index[1, 0] = x[0].argmin(), x[1].argmax()
    teacher = ((torch.rand(4, 9, generator=g, device=DEV) * 2 - 1) * 3.3e38).to(dtype)
    rest = torch.zeros(4, device=DEV) if with_rest else None
    weights = torch.full((4,), 1.0 / scale, device=DEV)
    check(x, index, teacher, rest, weights, scale)


@pytest.mark.parametrize("N,V,K", [(2401, 900, 5), (2399, 5001, 33), (1203, 3002, 64), (1203, 8001, 200), (700, 20003, 12), (40, 100003, 256), (300, 30, 30)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_rest", [False, True])
def test_rows_by_one_two_four_and_more_warps(N, V, K, dtype, with_rest):
    """As many rows as keep the GPU busy with few warps a row, and fewer; the same items more than once, places out of use, rows off boundaries."""
    g = torch.Generator(device=DEV).manual_seed(N + V)
    x, _ = placed(2 * torch.randn(N, V, generator=g, device=DEV), dtype, 1, 1)
    index = torch.randint(-1, V, (N, K), generator=g, device=DEV)
    index[::3] = torch.where(index[::3] < 0, -1, index[::3] % 17 % V)         # many to a batch
    index[1::3] = torch.where(index[1::3] < 0, -1, V - 1 - index[1::3] % 11 % V)
    teacher = torch.randn(N, K, generator=g, device=DEV).to(dtype)
    rest = None
    if with_rest:
        rest = torch.randn(N, generator=g, device=DEV)
        listed = torch.zeros(N, V + 1, dtype=torch.bool, device=DEV).scatter_(1, torch.where(index >= 0, index, V), True)[:, :V]
        rest[listed.all(1)] = -INF
    check(x, index, teacher, rest, torch.randn(N, generator=g, device=DEV), 0.8)
