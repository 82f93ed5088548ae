"""Log probabilities of given items, entropy and best alternatives (mts_logprobs_*) against the formulas in 64 bits.

Units u = 2^-24.  With d = scale (m - x) >= 0: an exponential is off by 4 u of itself from the function and by 2 d u from its argument; sums of
positive terms add at most 160 + V / 256 of them one after the other or over levels.  So log S is off by L = (170 + V / 256 + 2 E[d]) u at most, where E[d] is the
mean of d under p; what is computed from it is rounded a few times more.  A gradient in 16 bits is rounded once more: half a step."""
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


def forward(x, targets, k=0, scale=1.0, stride=None):
    N, V = x.shape
    logp, ent, stats = torch.full((N,), -9.0, device=DEV), torch.full((N,), -9.0, device=DEV), torch.full((N, 2), -9.0, device=DEV)
    ti, tl = torch.full((N, max(k, 1)), -9, dtype=torch.int64, device=DEV), torch.full((N, max(k, 1)), -9.0, device=DEV)
    mb.logprobs_forward(x, x.stride(0) if stride is None else stride, KIND[x.dtype], N, V, scale, targets, k, logp, ent, stats, ti, tl)
    torch.cuda.synchronize()
    return logp, ent, stats, ti[:, :k], tl[:, :k]


def plain(x, scale):
    """(log p, p, entropy, d, bound of the error of log S) in 64 bits; rows without an item have p = 0."""
    x = x.double() * scale
    m = x.amax(1, keepdim=True)
    z = x - torch.where(m == -INF, 0.0, m)
    e = z.exp()
    S = e.sum(1, keepdim=True)
    p = torch.where(S > 0, e / S, 0.0)
    log = torch.where(S > 0, z - S.log(), -INF)
    d = torch.where(p > 0, -z, 0.0)
    entropy = torch.where(p > 0, -p * log, 0.0).sum(1)
    mean_d = (p * d).sum(1)
    return log, p, entropy, d, (170 + x.shape[1] / 256 + 2 * mean_d) * U, mean_d


def close(got, want, bound):
    want = torch.where(want < -3.4028235e38, -INF, want)     # what fp32 has no number for
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine) and torch.equal(got[~fine].double(), want[~fine])
    err = (got.double() - want).abs()[fine]
    bound = bound.expand_as(want)[fine]
    assert bool((err <= bound).all()), (float((err - bound).max()), int((err > bound).sum()), got.shape)


def check(x, targets, k, scale):
    logp, ent, stats, ti, tl = forward(x, targets, k, scale)
    log, p, H, d, L, mean_d = plain(x, scale)
    at = targets.clamp(0, x.shape[1] - 1).unsqueeze(1)
    want = torch.where(targets < 0, 0.0, log.gather(1, at)[:, 0])
    close(logp, want, L + 6 * U * torch.where(want.isfinite(), want.abs(), 0.0))
    close(ent, H, 2 * L * (1 + mean_d) + 4 * U * H)
    if k:
        best = torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :k]
        assert torch.equal(ti, best), (ti[(ti != best).any(1)][:2], best[(ti != best).any(1)][:2])
        want = log.gather(1, best)
        close(tl, want, L.unsqueeze(1) + 8 * U * torch.where(want.isfinite(), want.abs(), 0.0))
    some = ~(x == -INF).all(1)
    assert torch.equal(stats[:, 0].double(), torch.where(some, x.double().amax(1), 0.0)) and bool((stats[~some][:, 1] == 0).all())


# rows, items, padding, shift, best: one row and many, one item, odd sizes, sizes around what a thread, a warp, a block and a cluster take
SHAPES = [(1, 1, 0, 0, 1), (3, 5, 0, 1, 5), (2, 32, 0, 0, 32), (5, 33, 3, 3, 10), (40, 100, 0, 0, 3), (7, 255, 0, 5, 32), (9, 1000, 0, 0, 8), (6, 1001, 7, 0, 8),
          (33, 4096, 0, 0, 20), (5, 5001, 0, 0, 10), (300, 5001, 0, 0, 1), (3, 20000, 0, 0, 32), (200, 20001, 0, 0, 16), (1, 100000, 0, 0, 20), (2, 131072, 0, 0, 32), (3, 131071, 1, 1, 5),
          (1, 262145, 0, 0, 10), (40, 70000, 0, 0, 10), (200, 66000, 0, 0, 7), (1, 1000003, 0, 0, 32)]


@pytest.mark.parametrize("N,V,pad,shift,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["spread", "masked", "ties"])
def test_forward(N, V, pad, shift, k, dtype, kind):
    g = torch.Generator(device=DEV).manual_seed(N * 31 + V)
    x = 3 * torch.randn(N, V, generator=g, device=DEV)
    if kind == "masked":                                     # almost all ruled out, some rows altogether, fewer than k left in others
        x.masked_fill_(torch.rand(N, V, generator=g, device=DEV) < torch.rand(N, 1, generator=g, device=DEV), -INF)
        x[::3] = -INF
        x[::3, V // 2] = 1.5
        x[::6] = -INF
    if kind == "ties":
        x = torch.round(x).clamp(-2, 2)                      # five values
        x[::2] = 0.25                                        # one value
    x, room = placed(x, dtype, pad, shift)
    targets = torch.randint(-1, V, (N,), generator=g, device=DEV)
    check(x, targets, k, 1.0 if N % 2 else 0.7)


@pytest.mark.parametrize("order", ["up", "down", "saw", "last", "first", "signs"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(3, 40000), (200, 9999), (2, 777)])
def test_forward_of_ordered_rows(order, dtype, N, V):
    """Rows in which every item is better than all before it, in which the best lie in one thread's items, at an end, and zeros of both signs."""
    i = torch.arange(V, device=DEV).double()
    x = {"up": i / V * 20, "down": -i / V * 20, "saw": torch.where(i % 2048 < 8, 5 + i / V, -i / V), "last": torch.where(i == V - 1, 9.0, 0.0),
         "first": torch.where(i == 0, 9.0, 0.0), "signs": torch.where(i % 3 == 0, 0.0, -0.0)}[order]
    x, _ = placed(x.expand(N, V).float(), dtype)
    check(x, torch.full((N,), V // 2, device=DEV), 32, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_lowest_values_and_large_ones(dtype):
    """Masks of the type's lowest value instead of -infinity, in some places and in whole rows, and scores as large as the type has them."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.randn(5, 3000, device=DEV).to(dtype)
    x[0, ::2] = low
    x[1] = low
    x[2] = low
    x[2, 7] = high
    x[3] = high
    x[4, 5] = -INF
    x[4, 6] = low
    check(x, torch.tensor([1, 5, 7, 8, 5], device=DEV), 4, 1.0)
    check(x, torch.tensor([1, 5, 7, 8, 6], device=DEV), 4, 3.0)


def test_values_that_are_not_finite():
    x = torch.randn(6, 5000, device=DEV)
    x[0, 17] = float("nan")
    x[1, 4999] = INF
    x[2] = float("nan")
    x[3, 100:] = -INF
    logp, ent, stats, ti, tl = forward(x, torch.zeros(6, dtype=torch.int64, device=DEV), 5)
    for r in (0, 1, 2):
        assert bool(logp[r].isnan()) and bool(ent[r].isnan()) and bool(tl[r].isnan().all())
    clean = x[0].clone()
    clean[17] = -INF
    assert torch.equal(ti[0], torch.sort(clean, dim=0, descending=True, stable=True)[1][:5]) and int(ti[1, 0]) == 4999 and ti[2].tolist() == [0, 1, 2, 3, 4]
    check(x[3:], torch.zeros(3, dtype=torch.int64, device=DEV), 5, 1.0)


def test_rows_with_more_nan_than_numbers():
    """Fewer numbers than alternatives are asked for: NaN come behind them, the lowest index first."""
    x = torch.full((3, 3000), float("nan"), device=DEV)
    x[0, 2000], x[0, 5], x[0, 9] = 1.0, 2.0, -INF
    x[1, 2999] = 3.0
    _, _, _, ti, tl = forward(x, torch.zeros(3, dtype=torch.int64, device=DEV), 6)
    assert ti[0].tolist() == [5, 2000, 9, 0, 1, 2] and ti[1].tolist() == [2999, 0, 1, 2, 3, 4] and ti[2].tolist() == [0, 1, 2, 3, 4, 5]


def test_targets_out_of_range_and_outputs_left_out():
    x = torch.randn(4, 600, device=DEV)
    t = torch.tensor([0, 599, 600, -7], device=DEV)
    logp, ent, _, ti, tl = forward(x, t, 3)
    assert bool(logp[2].isnan()) and float(logp[3]) == 0.0 and bool(torch.isfinite(logp[:2]).all())
    a, b, c, d = torch.empty(4, device=DEV), torch.empty(4, device=DEV), torch.empty(4, 3, dtype=torch.int64, device=DEV), torch.empty(4, 3, device=DEV)
    mb.logprobs_forward(x, 600, 0, 4, 600, 1.0, t, 0, a, None, None, None, None)
    mb.logprobs_forward(x, 600, 0, 4, 600, 1.0, None, 0, None, b, None, None, None)
    mb.logprobs_forward(x, 600, 0, 4, 600, 1.0, None, 3, None, None, None, c, None)
    mb.logprobs_forward(x, 600, 0, 4, 600, 1.0, None, 3, None, None, None, None, d)
    mb.logprobs_forward(None, 600, 0, 0, 600, 1.0, None, 0, None, None, None, None, None)
    torch.cuda.synchronize()
    assert torch.equal(a.nan_to_num(5.0), logp.nan_to_num(5.0)) and torch.equal(b, ent) and torch.equal(c, ti) and torch.equal(d, tl)


def backward(x, targets, stats, ent, gl, gh, scale, to=None):
    N, V = x.shape
    out = torch.full((N, V), 55.0, dtype=x.dtype, device=DEV) if to is None else to
    mb.logprobs_backward(x, x.stride(0), KIND[x.dtype], N, V, scale, targets, stats, ent, gl, gh, out, out.stride(0))
    torch.cuda.synchronize()
    return out


def gradient64(x, targets, gl, gh, scale):
    log, p, H, d, L, mean_d = plain(x, scale)
    one = torch.arange(x.shape[1], device=DEV) == targets.unsqueeze(1)
    gl, gh = (torch.zeros(len(x), device=DEV) if g is None else g for g in (gl, gh))
    gl = torch.where(targets < 0, 0.0, gl.double()).unsqueeze(1)
    gh = gh.double().unsqueeze(1)
    plogp = torch.where(p > 0, p * log, 0.0)
    want = scale * (gl * (one.double() - p) - gh * (plogp + p * H.unsqueeze(1)))
    # p is off by L + (6 + 4 d) u of itself, log p + H by the errors of both; the sums in it are rounded a few times
    off = (L.unsqueeze(1) + (10 + 4 * d) * U)
    size = scale * (p * gl.abs() + gh.abs() * (plogp.abs() + p * H.unsqueeze(1) + p * (1 + mean_d.unsqueeze(1))))
    return want, size * 4 * off + 2 * U * want.abs()


@pytest.mark.parametrize("N,V,pad,shift,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_backward(N, V, pad, shift, k, dtype, which):
    g = torch.Generator(device=DEV).manual_seed(N * 37 + V)
    x = 2 * torch.randn(N, V, generator=g, device=DEV)
    x.masked_fill_(torch.rand(N, V, generator=g, device=DEV) < 0.1, -INF)
    if N > 2:
        x[1] = -INF
    x, _ = placed(x, dtype, pad, shift)
    targets = torch.randint(-1, V, (N,), generator=g, device=DEV)
    gl = torch.randn(N, generator=g, device=DEV) * 8 if which != "entropy" else None
    gh = torch.randn(N, generator=g, device=DEV) * 8 if which != "logp" else None
    scale = 1.0 if N % 2 else 1.3
    _, ent, stats, _, _ = forward(x, targets, 0, scale)
    want, bound = gradient64(x, targets, gl, gh, scale)
    bound = bound + want.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -25 * (dtype == torch.float16) + 1e-37
    to, room = placed(torch.zeros(N, V), dtype, 3, 2)
    close(backward(x, targets, stats, ent, gl, gh, scale, to), want, bound)
    mask = torch.ones_like(room, dtype=torch.bool)
    torch.as_strided(mask, to.shape, to.stride(), to.storage_offset()).fill_(False)
    assert bool((room[mask] == 77.0).all())
    same = x.clone() if pad == 0 and shift == 0 else placed(x.float(), dtype, pad, shift)[0]
    backward(same, targets, stats, ent, gl, gh, scale, same)                 # in place
    assert torch.equal(same, to)


def test_gradient_against_differences():
    """The 64-bit formula that the kernel is held to, against differences of log probability and entropy in 64 bits."""
    x = torch.randn(2, 9, device=DEV, dtype=torch.float64)
    t, gl, gh = torch.tensor([3, -1], device=DEV), torch.tensor([0.7, 2.0], device=DEV), torch.tensor([-0.4, 1.1], device=DEV)

    def value(y):
        log, _, H, _, _, _ = plain(y, 1.3)
        return gl[0].double() * log[0, 3] + (gh.double() * H).sum()

    want, _ = gradient64(x, t, gl, gh, 1.3)
    for i in range(2):
        for j in range(9):
            e = torch.zeros_like(x)
            e[i, j] = 1e-6
            assert abs(float((value(x + e) - value(x - e)) / 2e-6 - want[i, j])) < 1e-8


def test_rows_without_gradient_are_zero_whatever_they_hold():
    x = torch.randn(4, 3001, device=DEV)
    x[0] = float("nan")
    x[1] = INF
    t = torch.tensor([5, 6, 7, -1], device=DEV)
    _, ent, stats, _, _ = forward(x, t)
    d = backward(x, t, stats, ent, torch.tensor([0.0, 0.0, 1.0, 1.0], device=DEV), torch.zeros(4, device=DEV), 1.0)
    assert bool((d[[0, 1, 3]] == 0).all()) and float(d[2].abs().max()) > 0.5
    d = backward(x, torch.full((4,), 3001, device=DEV), stats, ent, torch.ones(4, device=DEV), None, 1.0)
    assert bool(d.isnan().all())                                             # a target that is not there


def test_offsets_past_32_bits():
    """5 rows of 500,000,000 elements apart: places behind 2^31 elements and 2^32 bytes."""
    N, V, stride = 5, 3000 + 1, 500_000_000
    room = torch.zeros((N - 1) * stride + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(room, (N, V), (stride, 1))
    x.copy_(torch.randn(N, V, device=DEV))
    t = torch.randint(V, (N,), device=DEV)
    check(x, t, 9, 1.0)
    _, ent, stats, _, _ = forward(x, t)
    gl = torch.ones(N, device=DEV)
    want, bound = gradient64(x, t, gl, None, 1.0)
    backward(x, t, stats, ent, gl, None, 1.0, x)
    close(x, want, bound + want.abs() * 2.0 ** -8 + 1e-37)


@pytest.mark.parametrize("N,V,k,dtype", [(80, 300001, 32, torch.float32), (76, 1200007, 20, torch.bfloat16), (151, 150001, 5, torch.float32)])
@pytest.mark.parametrize("kind", ["spread", "up", "few"])
def test_best_of_long_rows_by_single_blocks(N, V, k, dtype, kind):
    """Rows of more groups than a thread keeps maxima of, too many for a cluster each."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V, generator=g, device=DEV)
    if kind == "up":
        x = x * 0.001 + torch.arange(V, device=DEV) / V * 8
    if kind == "few":
        x.masked_fill_(torch.rand(N, V, generator=g, device=DEV) < 1 - 40 / V, -INF)
    x, _ = placed(x, dtype, 0, 3)
    check(x, torch.randint(-1, V, (N,), generator=g, device=DEV), k, 1.0)


MASKS = [-1e10, -1e30, "lowest"]


def masked_rows(V, dtype, mask):
    """Rows with masks of large finite values: half of the places, long runs of them, all places but one, all of them, and none."""
    g = torch.Generator(device=DEV).manual_seed(V)
    low = torch.finfo(dtype).min
    x = 10 * torch.randn(6, V, generator=g, device=DEV)
    x[0].masked_fill_(torch.rand(V, generator=g, device=DEV) < 0.5, max(mask, low) if mask != "lowest" else low)
    x[1, :V * 3 // 4] = max(mask, low) if mask != "lowest" else low
    x[2] = max(mask, low) if mask != "lowest" else low
    x[2, V // 3] = 7.0
    x[3] = max(mask, low) if mask != "lowest" else low
    x[4, V // 2:] = max(mask, low) if mask != "lowest" else low
    return x.to(dtype)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("scale", [0.25, 0.5, 1.0, 1e4, 1e10, 1e30])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [100, 3000, 70001])
def test_masks_of_large_finite_values_at_every_scale(mask, scale, dtype, V):
    """scale * score far beyond what fp32 has digits for, in some places, in whole threads' places and in whole rows; scores at scales up to the largest."""
    x = masked_rows(V, dtype, mask)
    t = torch.tensor([1, V - 1, V // 3, 5, 3, 2], device=DEV)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    check(x, t, 4, scale)
    _, ent, stats, _, _ = forward(x, t, 0, scale)
    gl, gh = torch.ones(6, device=DEV) / scale, torch.full((6,), 0.5, device=DEV) / scale
    want, bound = gradient64(x, t, gl, gh, scale)
    close(backward(x, t, stats, ent, gl, gh, scale), want, bound + want.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -25 * (dtype == torch.float16) + 1e-37)


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -124, 1e-30, 0.25])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [60, 5000, 70001])
def test_scores_whose_difference_is_no_number(scale, dtype, V):
    """Scores of both signs up to the type's largest: their difference overflows, its product with a small scale does not."""
    g = torch.Generator(device=DEV).manual_seed(V)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    x = ((torch.rand(4, V, generator=g, device=DEV) * 2 - 1) * 3.3e38).to(dtype)
    t = torch.stack([x[0].argmin(), x[1].argmax(), torch.tensor(7, device=DEV), torch.tensor(-1, device=DEV)])
    check(x, t, 5, scale)
    check(x, t, min(V, 32), scale)
    _, ent, stats, _, _ = forward(x, t, 0, scale)
    gl, gh = torch.ones(4, device=DEV) / scale, torch.ones(4, device=DEV) / scale
    want, bound = gradient64(x, t, gl, gh, scale)
    close(backward(x, t, stats, ent, gl, gh, scale), want, bound + want.abs() * torch.finfo(dtype).eps / 2 + 1e-37)


def test_a_target_that_is_not_there_and_whose_gradient_is_zero():
    """A loss that leaves a row out by a gradient of 0 leaves it out altogether, and the entropy's gradient does not see its target."""
    x = torch.randn(3, 500, device=DEV)
    t = torch.tensor([500, 1 << 40, 500], device=DEV)
    _, ent, stats, _, _ = forward(x, t)
    gl, gh = torch.tensor([0.0, -0.0, 1.0], device=DEV), torch.tensor([0.0, 2.0, 0.0], device=DEV)
    d = backward(x, t, stats, ent, gl, gh, 1.0)
    want, bound = gradient64(x, torch.full_like(t, -1), gl, gh, 1.0)
    assert bool((d[0] == 0).all()) and bool(d[2].isnan().all())
    close(d[1], want[1], bound[1])


@pytest.mark.parametrize("N,V,k", [(2401, 700, 9), (2403, 2050, 32), (2399, 2801, 10), (1203, 6001, 17), (700, 20003, 5), (310, 50001, 32), (40, 100003, 3), (2400, 33, 33 - 1)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["spread", "masked", "ties", "nan"])
def test_rows_by_one_two_four_and_more_warps(N, V, k, dtype, kind):
    """As many rows as keep the GPU busy with few warps a row, and fewer, off boundaries."""
    g = torch.Generator(device=DEV).manual_seed(N + V)
    x = 3 * torch.randn(N, V, generator=g, device=DEV)
    if kind == "masked":
        x.masked_fill_(torch.rand(N, V, generator=g, device=DEV) < torch.rand(N, 1, generator=g, device=DEV), -INF)
        x[::5] = -INF
        x[::5, V // 2:V // 2 + 3] = 1.5
    if kind == "ties":
        x = torch.round(x).clamp(-2, 2)
    x, _ = placed(x, dtype, 1, 1)
    t = torch.randint(-1, V, (N,), generator=g, device=DEV)
    if kind != "nan":
        return check(x, t, k, 1.0)
    x[::4, V // 3] = float("nan")                            # one NaN: its row's statistics, and no other's
    logp, ent, _, ti, tl = forward(x, t, k)
    assert bool(ent[::4].isnan().all()) and bool(logp[::4][t[::4] >= 0].isnan().all()) and bool((logp[::4][t[::4] < 0] == 0).all()) and bool(tl[::4].isnan().all())
    best = torch.sort(x.float().nan_to_num(nan=-INF, neginf=-INF), dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(ti, best) or k == V - 1
    some = torch.arange(N, device=DEV) % 4 != 0
    log, _, H, _, L, mean_d = plain(x[some], 1.0)
    want = torch.where(t[some] < 0, 0.0, log.gather(1, t[some].clamp(min=0).unsqueeze(1))[:, 0])
    close(logp[some], want, L + 6 * U * want.abs())
    close(ent[some], H, 2 * L * (1 + mean_d) + 4 * U * H)
    want = log.gather(1, best[some])
    close(tl[some], want, L.unsqueeze(1) + 8 * U * want.abs())
