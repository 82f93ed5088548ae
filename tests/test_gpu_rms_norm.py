"""Norm of the residual stream (mts_rms_norm_*) against the formula in 64 bits.

Units u = 2^-24.  A sum over a row adds at most 128 terms one after the other and joins such chains over at most 10 levels, products before it are
rounded twice: off by at most 160 u of the sum of the terms' sizes.  The root halves the relative error of the sum of squares: c is
off by at most 90 u.  A result in 16 bits is rounded once more: half a step, eps(T) / 2 of it (and 2^-25 below the normal numbers of fp16)."""
import pytest
import torch

from paper_2305_01515_b200 import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-6
TYPES = (torch.float32, torch.float16, torch.bfloat16)
KIND = {torch.float32: mb.DTYPE_FP32, torch.float16: mb.DTYPE_FP16, torch.bfloat16: mb.DTYPE_BF16}
SUM, C = 160 * U, 90 * U


def half(dtype):
    return torch.finfo(dtype).eps / 2


def placed(x, dtype, pad, shift):
    """x in a buffer of its own, rows `pad` elements longer than they need and `shift` elements behind a boundary; the rest holds 7."""
    N, D = x.shape
    room = torch.full((shift + N * (D + pad) + 64,), 7.0, dtype=dtype, device=DEV)
    view = torch.as_strided(room, (N, D), (D + pad, 1), shift)
    view.copy_(x)
    return view, room


def untouched(view, room):
    mask = torch.ones_like(room, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((room[mask] == 7.0).all())


def norm64(r, w, eps=EPS):
    c = 1.0 / (r.square().mean(1, keepdim=True) + eps).sqrt()
    return r * c * w, c


def close(got, want, bound):
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), int((err > bound).sum()), got.shape)


# rows, columns, padding, shift: one token, odd widths, widths around what a warp, a group of warps and a block hold, the widest
SHAPES = [(1, 1, 0, 0), (3, 7, 0, 1), (5, 128, 0, 0), (192, 128, 0, 0), (70, 200, 0, 0), (33, 256, 8, 8), (17, 257, 0, 0), (9, 333, 3, 2), (40, 512, 0, 0),
          (5, 1000, 24, 0), (300, 1024, 0, 0), (3, 1025, 0, 0), (7, 2048, 0, 4), (4, 4104, 0, 0), (2, 8192, 0, 0), (3, 8200, 8, 0), (2, 16384, 0, 0), (3, 20001, 1, 3),
          (2, 32768, 0, 0)]


@pytest.mark.parametrize("N,D,pad,shift", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_forward(N, D, pad, shift, dtype, residual):
    g = torch.Generator(device=DEV).manual_seed(N * 7 + D)
    x, _ = placed(torch.randn(N, D, generator=g, device=DEV), dtype, pad, shift)
    res, _ = placed(torch.randn(N, D, generator=g, device=DEV) * 2, dtype, pad, 0) if residual else (None, None)
    w = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(torch.float32 if D % 2 else dtype)
    total, room_t = placed(torch.zeros(N, D), dtype, pad, shift) if residual else (None, None)
    out, room = placed(torch.zeros(N, D), dtype, pad, shift)
    inv = torch.full((N,), -1.0, device=DEV)
    mb.rms_norm_forward(x, D + pad, res, D + pad, w, KIND[w.dtype], KIND[dtype], N, D, EPS, total, D + pad, out, D + pad, inv)
    torch.cuda.synchronize()
    r = x
    if residual:
        assert torch.equal(total, (x.float() + res.float()).to(dtype)) and untouched(total, room_t)
        r = total
    want, c = norm64(r.double(), w.double())
    close(inv, c[:, 0], C * c[:, 0])
    close(out, want, want.abs() * (half(dtype) + C + 4 * U) + 2.0 ** -25 * (dtype == torch.float16))
    assert untouched(out, room)


def nearest8(v):
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


@pytest.mark.parametrize("N,D,pad,shift", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
def test_8bit(N, D, pad, shift, dtype, group):
    g = torch.Generator(device=DEV).manual_seed(N * 11 + D + group)
    x, _ = placed(torch.randn(N, D, generator=g, device=DEV) * torch.exp(torch.randn(D, generator=g, device=DEV)), dtype, pad, shift)
    res, _ = placed(torch.randn(N, D, generator=g, device=DEV), dtype, 0, 0)
    w = 1 + 0.3 * torch.randn(D, generator=g, device=DEV)
    n = group or D
    G = -(-D // n)
    total, codes, scales = torch.empty(N, D, dtype=dtype, device=DEV), torch.full((N, D + 5), 99, dtype=torch.uint8, device=DEV), torch.zeros(N, G, device=DEV)
    mb.rms_norm_forward_8bit(x, D + pad, res, D, w, 0, KIND[dtype], N, D, EPS, total, D, codes, D + 5, scales, group, None)
    for t in TYPES:
        back, room = placed(torch.zeros(N, D), t, 3, 1)
        mb.rows_from_8bit(codes, D + 5, scales, group, N, D, back, KIND[t], D + 3)
        torch.cuda.synchronize()
        held = codes[:, :D].contiguous().view(torch.float8_e4m3fn).double() * scales.double().repeat_interleave(n, 1)[:, :D]
        close(back, held, held.abs() * (half(t) + U) + 2.0 ** -25 * (t == torch.float16))
        assert untouched(back, room)
    assert bool((codes[:, D:] == 99).all()) and torch.equal(total, (x.float() + res.float()).to(dtype))
    y, _ = norm64(total.double(), w.double())
    top = torch.nn.functional.pad(y.abs(), (0, G * n - D)).view(N, G, n).amax(2).clamp(min=2.0 ** -100)
    close(scales, top / 448.0, top / 448.0 * (C + 6 * U))
    # half a step of four significant bits, of 2^-9 below 2^-6; at the top a scale that is rounded down moves no code over 448
    s = (top / 448.0).repeat_interleave(n, 1)[:, :D]
    close(held, y, y.abs() * (2.0 ** -4 + 2 * C + 16 * U) + s * 2.0 ** -10 * (1 + 1e-4))
    # and the nearest code itself where the value is not near a border between two
    v = y / s
    clear = (nearest8(v * (1 + 1e-4)) == nearest8(v * (1 - 1e-4)))
    got = codes[:, :D].contiguous().view(torch.float8_e4m3fn).double()
    assert bool((got == nearest8(v))[clear].all()) and float(clear.double().mean()) > 0.9


@pytest.mark.parametrize("group", [0, 64])
def test_8bit_rows_of_zeros_and_of_what_is_not_finite(group):
    x = torch.randn(5, 128, device=DEV)
    x[0] = 0.0
    x[1, 3] = float("nan")
    x[2, 100] = float("inf")
    x[3] *= 1e-30
    w = torch.ones(128, device=DEV)
    w[:64] = 0.0
    codes, scales = torch.empty(5, 128, dtype=torch.uint8, device=DEV), torch.empty(5, 2 if group else 1, device=DEV)
    mb.rms_norm_forward_8bit(x, 128, None, 0, w, 0, 0, 5, 128, 1e-6, None, 0, codes, 128, scales, group, None)
    back = torch.empty(5, 128, device=DEV)
    mb.rows_from_8bit(codes, 128, scales, group, 5, 128, back, 0, 128)
    torch.cuda.synchronize()
    assert bool((back[0] == 0).all()) and bool(back[1].isnan().all()) and bool(back[2, 100].isnan()) and bool((back[4, :64] == 0).all())
    assert bool(torch.isfinite(scales[[0, 3, 4]]).all()) and bool((scales[0] == 2.0 ** -100 / 448).all())
    want, _ = norm64(x[4:].double(), w.double())
    assert float((back[4:].double() - want).abs().max()) <= float(want.abs().max()) * 2.0 ** -4


def backward64(x, w, dy, ds, eps=EPS):
    c = 1.0 / (x.square().mean(1, keepdim=True) + eps).sqrt()
    a = (dy * w * x).mean(1, keepdim=True) * c * c
    dx = c * (dy * w - x * a)
    size = c * ((dy * w).abs() + x.abs() * (dy * w * x).abs().mean(1, keepdim=True) * c * c)      # what the terms' errors are relative to
    return dx if ds is None else dx + ds, size + (0 if ds is None else ds.abs()), (dy * x * c).sum(0), (dy * x * c).abs().sum(0), c


@pytest.mark.parametrize("N,D,pad,shift", SHAPES + [(2000, 96, 0, 0), (1500, 260, 0, 0), (5000, 16, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_sum", [False, True])
def test_backward(N, D, pad, shift, dtype, with_sum):
    g = torch.Generator(device=DEV).manual_seed(N * 13 + D)
    x, _ = placed(torch.randn(N, D, generator=g, device=DEV) * 2, dtype, pad, shift)
    dy, _ = placed(torch.randn(N, D, generator=g, device=DEV), dtype, pad, 0)
    ds, _ = placed(torch.randn(N, D, generator=g, device=DEV), dtype, 0, shift) if with_sum else (None, None)
    w = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dtype if D % 2 else torch.float32)
    _, c = norm64(x.double(), w.double())
    inv = c[:, 0].float()
    dx, room = placed(torch.zeros(N, D), dtype, pad, shift)
    dw = torch.full((D,), -5.0, device=DEV)
    ws = torch.full((mb.rms_norm_workspace_bytes(N, D),), 255, dtype=torch.uint8, device=DEV)
    mb.rms_norm_backward(x, D + pad, w, KIND[w.dtype], KIND[dtype], N, D, inv, dy, D + pad, ds, D, dx, D + pad, dw, ws, ws.numel())
    torch.cuda.synchronize()
    want, size, dw64, dw_size, _ = backward64(x.double(), w.double(), dy.double(), None if ds is None else ds.double())
    close(dx, want, want.abs() * half(dtype) + size * (SUM + 10 * U) + 2.0 ** -25 * (dtype == torch.float16))
    # rows are added one after the other in fp32 (at most N of them), the blocks' sums in 64 bits
    close(dw, dw64, dw_size * (min(N, 600) + 6) * U)
    assert untouched(dx, room)
    again = torch.zeros_like(dx)
    mb.rms_norm_backward(x, D + pad, w, KIND[w.dtype], KIND[dtype], N, D, inv, dy, D + pad, ds, D, again, D, None, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(again, dx)                        # without the weight's gradient, no workspace


def test_backward_against_differences():
    """The 64-bit formula that the kernels are held to, against differences of the norm itself."""
    g = torch.Generator(device=DEV).manual_seed(3)
    x, w, dy = (torch.randn(3, 11, generator=g, device=DEV, dtype=torch.float64) for _ in range(3))
    w = w[0]
    dx, _, dw, _, _ = backward64(x, w, dy, None)
    h = 1e-6
    for i in range(3):
        for j in range(11):
            e = torch.zeros_like(x)
            e[i, j] = h
            slope = ((norm64(x + e, w)[0] - norm64(x - e, w)[0]) * dy).sum() / (2 * h)
            assert abs(float(slope - dx[i, j])) < 1e-8
    for j in range(11):
        e = torch.zeros_like(w)
        e[j] = h
        assert abs(float(((norm64(x, w + e)[0] - norm64(x, w - e)[0]) * dy).sum() / (2 * h) - dw[j])) < 1e-8


def test_stream_updated_in_place_and_gradients_in_place():
    x, res = torch.randn(50, 264, device=DEV).bfloat16(), torch.randn(50, 264, device=DEV).bfloat16()
    w = torch.ones(264, device=DEV)
    want = x + res
    outs = []
    for target in (None, "x", "residual"):
        a, b, out = x.clone(), res.clone(), torch.empty_like(x)
        total = torch.empty_like(x) if target is None else a if target == "x" else b
        mb.rms_norm_forward(a, 264, b, 264, w, 0, mb.DTYPE_BF16, 50, 264, EPS, total, 264, out, 264, None)
        torch.cuda.synchronize()
        assert torch.equal(total, want)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    inv = torch.rand(50, device=DEV)
    dx = []
    for target in (None, 0, 1):
        dy, ds = x.clone(), res.clone()
        to = torch.empty_like(x) if target is None else (dy, ds)[target]
        mb.rms_norm_backward(want, 264, w, 0, mb.DTYPE_BF16, 50, 264, inv, dy, 264, ds, 264, to, 264, None, None, 0)
        torch.cuda.synchronize()
        dx.append(to)
    assert torch.equal(dx[0], dx[1]) and torch.equal(dx[0], dx[2])


def test_no_rows():
    w, dw = torch.ones(8, device=DEV), torch.full((8,), 3.0, device=DEV)
    mb.rms_norm_forward(None, 8, None, 0, w, 0, 0, 0, 8, EPS, None, 0, None, 8, None)
    mb.rms_norm_forward_8bit(None, 8, None, 0, w, 0, 0, 0, 8, EPS, None, 0, None, 8, None, 0, None)
    mb.rows_from_8bit(None, 8, None, 0, 0, 8, None, 0, 8)
    ws = torch.empty(mb.rms_norm_workspace_bytes(0, 8), dtype=torch.uint8, device=DEV)
    mb.rms_norm_backward(None, 8, w, 0, 0, 0, 8, None, None, 8, None, 0, None, 8, dw, ws, ws.numel())
    torch.cuda.synchronize()
    assert bool((dw == 0).all())


def test_offsets_past_32_bits():
    """Rows of a buffer of more than 2^32 bytes, far apart: the last row is where it should be."""
    N, D, stride = 3, 40, 1_200_000_000
    room = torch.zeros(2 * stride + D, dtype=torch.float16, device=DEV)
    x = torch.as_strided(room, (N, D), (stride, 1))
    x.copy_(torch.randn(N, D, device=DEV))
    out, w = torch.empty(N, D, dtype=torch.float16, device=DEV), torch.ones(D, device=DEV)
    inv = torch.empty(N, device=DEV)
    mb.rms_norm_forward(x, stride, None, 0, w, 0, mb.DTYPE_FP16, N, D, EPS, None, 0, out, D, inv)
    torch.cuda.synchronize()
    want, c = norm64(x.double(), w.double())
    close(out, want, want.abs() * (2.0 ** -11 + 100 * U) + 2.0 ** -25)


@pytest.mark.parametrize("N,D", [(330, 2500), (500, 4104), (350, 8201), (310, 16384), (301, 16389), (200, 20008)])
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_of_wide_rows_many_to_a_block(N, D, dtype):
    """Rows that a block's warps share, several to a block one after the other; the gradient in the place of either input of it too."""
    g = torch.Generator(device=DEV).manual_seed(N + D)
    x, dy, ds = (torch.randn(N, D, generator=g, device=DEV).to(dtype) for _ in range(3))
    w = 1 + 0.3 * torch.randn(D, generator=g, device=DEV)
    inv = norm64(x.double(), w.double())[1][:, 0].float()
    ws = torch.full((mb.rms_norm_workspace_bytes(N, D),), 255, dtype=torch.uint8, device=DEV)

    def run(dy, ds, dx):
        dw = torch.full((D,), -5.0, device=DEV)
        mb.rms_norm_backward(x, D, w, 0, KIND[dtype], N, D, inv, dy, D, ds, D, dx, D, dw, ws, ws.numel())
        torch.cuda.synchronize()
        return dx, dw

    dx, dw = run(dy, ds, torch.empty_like(x))
    want, size, dw64, dw_size, _ = backward64(x.double(), w.double(), dy.double(), ds.double())
    close(dx, want, want.abs() * half(dtype) + size * (SUM + 10 * U) + 2.0 ** -25 * (dtype == torch.float16))
    close(dw, dw64, dw_size * (N + 6) * U)
    a, b = dy.clone(), ds.clone()
    assert all(torch.equal(p, q) for p, q in zip(run(a, ds, a), (dx, dw))) and all(torch.equal(p, q) for p, q in zip(run(dy, b, b), (dx, dw)))


@pytest.mark.parametrize("N,D", [(301, 4097), (297, 6144), (299, 6152), (149, 8192), (150, 8200), (298, 12296), (151, 16384), (149, 16392), (150, 24577), (149, 32767),
                                 (297, 32768)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_sum", [False, True])
def test_backward_of_widths_where_the_rows_shape_changes(N, D, dtype, with_sum):
    """The widths at which a warp takes two, four and eight chunks, by vectors and (odd ones) by elements, with more rows than blocks."""
    g = torch.Generator(device=DEV).manual_seed(N + D)
    x, dy, ds = (torch.randn(N, D, generator=g, device=DEV).to(dtype) for _ in range(3))
    ds = ds if with_sum else None
    w = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    inv = norm64(x.double(), w.double())[1][:, 0].float()
    dx, room = placed(torch.zeros(N, D), dtype, 0, 0)
    ws = torch.full((mb.rms_norm_workspace_bytes(N, D),), 255, dtype=torch.uint8, device=DEV)
    dw = torch.full((D,), -5.0, device=DEV)
    mb.rms_norm_backward(x, D, w, KIND[dtype], KIND[dtype], N, D, inv, dy, D, ds, D, dx, D, dw, ws, ws.numel())
    torch.cuda.synchronize()
    want, size, dw64, dw_size, _ = backward64(x.double(), w.double(), dy.double(), None if ds is None else ds.double())
    close(dx, want, want.abs() * half(dtype) + size * (SUM + 10 * U) + 2.0 ** -25 * (dtype == torch.float16))
    close(dw, dw64, dw_size * (N + 6) * U)
    assert untouched(dx, room)


@pytest.mark.parametrize("N,D,pad,shift", [(3, 7, 0, 1), (300, 256, 0, 0), (301, 264, 0, 8), (120, 1024, 0, 0), (90, 1000, 24, 0), (50, 333, 3, 2), (40, 4104, 0, 0), (9, 20001, 1, 3),
                                           (12, 32768, 0, 0), (40000, 256, 0, 0), (152000, 24, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
@pytest.mark.parametrize("wide_weight", [False, True])
def test_8bit_codes_are_those_of_x_and_weight_alone(N, D, pad, shift, dtype, group, wide_weight):
    """Every code, those between two numbers too, is e4m3(u (448 / max |u|)) with u = r weight in fp32: torch's own product, quotient, product and conversion give the same."""
    g = torch.Generator(device=DEV).manual_seed(N + D + group)
    x, _ = placed(torch.randn(N, D, generator=g, device=DEV), dtype, pad, shift)
    w = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(torch.float32 if wide_weight else dtype)
    n = group or D
    G = -(-D // n)
    codes, scales = torch.empty(N, D, dtype=torch.uint8, device=DEV), torch.empty(N, G, device=DEV)
    mb.rms_norm_forward_8bit(x, D + pad, None, 0, w, KIND[w.dtype], KIND[dtype], N, D, EPS, None, 0, codes, D, scales, group, None)
    torch.cuda.synchronize()
    u = torch.nn.functional.pad(x.float() * w.float(), (0, G * n - D)).view(N, G, n)
    top = u.abs().amax(2, keepdim=True)
    want = (u * (torch.full_like(top, 448.0) / top)).view(N, G * n)[:, :D].to(torch.float8_e4m3fn)
    assert torch.equal(codes, want.contiguous().view(torch.uint8)), int((codes != want.contiguous().view(torch.uint8)).sum())
    most = top[:, :, 0].double() * norm64(x.double(), w.double())[1]
    close(scales, most / 448.0, most / 448.0 * (C + 6 * U))


@pytest.mark.parametrize("group", [0, 32, 256])
@pytest.mark.parametrize("D", [512, 515])
def test_8bit_values_below_the_least_maximum(group, D):
    """Groups whose largest value is below 2^-100 have its scale: codes of 448 2^100 y, small ones of the type among them."""
    g = torch.Generator(device=DEV).manual_seed(D)
    x = torch.randn(20, D, generator=g, device=DEV)
    w = torch.exp2(torch.arange(D, device=DEV) // 32 * -1.0 - 96)
    G = -(-D // (group or D))
    codes, scales, inv = torch.empty(20, D, dtype=torch.uint8, device=DEV), torch.empty(20, G, device=DEV), torch.empty(20, device=DEV)
    mb.rms_norm_forward_8bit(x, D, None, 0, w, 0, 0, 20, D, EPS, None, 0, codes, D, scales, group, inv)
    torch.cuda.synchronize()
    n = group or D
    y = torch.nn.functional.pad(norm64(x.double(), w.double())[0], (0, G * n - D)).view(20, G, n)
    most = y.abs().amax(2).clamp(min=2.0 ** -100)
    close(scales, most / 448.0, most / 448.0 * (C + 6 * U))
    held = codes.view(torch.float8_e4m3fn).double()
    v = (y * (448.0 / most).unsqueeze(2)).view(20, G * n)[:, :D]
    close(held, v, v.abs() * (2.0 ** -4 + 2 * C + 16 * U) + 2.0 ** -10 * (1 + 1e-4))
    assert not group or bool((scales == 2.0 ** -100 / 448).any()) and bool((held == 0).any())


# short rows in such numbers that a warp has several (16 bits, on boundaries), the last of them with some to spare
MANY = [(151553, 16), (151559, 32), (75777, 40), (75781, 64), (37889, 128), (37893, 104), (18945, 256), (18947, 200), (18945, 512), (18949, 264)]


@pytest.mark.parametrize("N,D", MANY)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_many_short_rows(N, D, dtype, residual):
    """Forward in the type and in 8 bits, and backward, of rows of which a warp takes two to thirty-two."""
    g = torch.Generator(device=DEV).manual_seed(N + D)
    x, dy, ds = (torch.randn(N, D, generator=g, device=DEV).to(dtype) for _ in range(3))
    res = torch.randn(N, D, generator=g, device=DEV).to(dtype) if residual else None
    w = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    total = torch.empty_like(x) if residual else None
    out, room = placed(torch.zeros(N, D), dtype, 0, 0)
    inv = torch.full((N + 1,), -1.0, device=DEV)
    mb.rms_norm_forward(x, D, res, D, w, KIND[dtype], KIND[dtype], N, D, EPS, total, D, out, D, inv)
    torch.cuda.synchronize()
    r = x if res is None else total
    assert res is None or torch.equal(total, (x.float() + res.float()).to(dtype))
    want, c = norm64(r.double(), w.double())
    close(inv[:N], c[:, 0], C * c[:, 0])
    close(out, want, want.abs() * (half(dtype) + C + 4 * U) + 2.0 ** -25 * (dtype == torch.float16))
    assert untouched(out, room) and float(inv[N]) == -1.0
    for group in (0, 32, 128):
        n = group or D
        G = -(-D // n)
        codes, scales = torch.full((N + 1, D), 99, dtype=torch.uint8, device=DEV), torch.full((N + 1, G), -3.0, device=DEV)
        total8 = torch.empty_like(x) if residual else None
        mb.rms_norm_forward_8bit(x, D, res, D, w, KIND[dtype], KIND[dtype], N, D, EPS, total8, D, codes, D, scales, group, None)
        torch.cuda.synchronize()
        top = torch.nn.functional.pad(want.abs(), (0, G * n - D)).view(N, G, n).amax(2).clamp(min=2.0 ** -100)
        close(scales[:N], top / 448.0, top / 448.0 * (C + 6 * U))
        held = codes[:N].view(torch.float8_e4m3fn).double() * scales[:N].double().repeat_interleave(n, 1)[:, :D]
        close(held, want, want.abs() * (2.0 ** -4 + 2 * C + 16 * U) + (top / 448.0).repeat_interleave(n, 1)[:, :D] * 2.0 ** -10 * (1 + 1e-4))
        assert bool((codes[N] == 99).all()) and bool((scales[N] == -3.0).all()) and (res is None or torch.equal(total8, total))
    dx, room = placed(torch.zeros(N, D), dtype, 0, 0)
    dw, ws = torch.full((D,), -5.0, device=DEV), torch.full((mb.rms_norm_workspace_bytes(N, D),), 255, dtype=torch.uint8, device=DEV)
    mb.rms_norm_backward(r, D, w, KIND[dtype], KIND[dtype], N, D, inv, dy, D, ds, D, dx, D, dw, ws, ws.numel())
    torch.cuda.synchronize()
    want, size, dw64, dw_size, _ = backward64(r.double(), w.double(), dy.double(), ds.double())
    close(dx, want, want.abs() * half(dtype) + size * (SUM + C + 10 * U) + 2.0 ** -25 * (dtype == torch.float16))
    close(dw, dw64, dw_size * (600 + 90 + 6) * U)            # at most 600 rows one after the other, the root of the forward
    assert untouched(dx, room)


@pytest.mark.parametrize("N,D,stride,group", [(5, 64, 64, 0), (9, 264, 264, 32), (300, 2048, 2048, 64), (7, 2051, 2056, 128), (11, 4096, 4096, 0), (6, 4099, 4104, 256), (3, 20005, 20008, 32),
                                              (2, 32768, 32768, 0), (4, 4099, 4104, 0)])
@pytest.mark.parametrize("dtype", TYPES)
def test_values_from_8_bits_by_vectors(N, D, stride, group, dtype):
    """Codes and values on boundaries of eight, narrow and wide, with ends that fill no piece; the places behind them are left as they were."""
    g = torch.Generator(device=DEV).manual_seed(N + D)
    G = -(-D // group) if group else 1
    codes = torch.randint(256, (N, stride), generator=g, device=DEV, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 5                          # no NaN
    scales = torch.rand(N, G, generator=g, device=DEV) + 0.01
    out, room = placed(torch.zeros(N, D), dtype, stride - D, 0)
    assert out.data_ptr() % 16 == 0 and codes.data_ptr() % 8 == 0
    mb.rows_from_8bit(codes, stride, scales, group, N, D, out, KIND[dtype], stride)
    torch.cuda.synchronize()
    want = codes[:, :D].contiguous().view(torch.float8_e4m3fn).double() * scales.double().repeat_interleave(group or D, 1)[:, :D]
    close(out, want, want.abs() * (half(dtype) + U) + 2.0 ** -25 * (dtype == torch.float16))
    assert untouched(out, room)
