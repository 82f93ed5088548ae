"""Relative position bias by buckets (mts_relpos_bias_*) against plain loops in 64 bits.

The forward selects and rounds once: equality.  The gradient adds chains of at most 1024 fp32 terms before it goes on in 64
bits, and rounds the sum once: |error| <= 1024 u sum|terms| + u |sum|, u = 2^-24."""
import numpy as np
import pytest
import torch

from paper_2305_01515_b200 import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
KIND = {torch.float32: mb.DTYPE_FP32, torch.float16: mb.DTYPE_FP16, torch.bfloat16: mb.DTYPE_BF16}
STARTS = [0, 1, 2, 3, 4, 6, 9, 16, 16, 40, 100]          # one bucket holds nothing


def bucket_table(starts, two_sided, causal, Lq, Lk, off):
    """Row of the table for every (query, key), -1 where masked."""
    r = np.arange(Lk)[None, :] - (np.arange(Lq)[:, None] + off)
    d = np.abs(r) if two_sided else np.maximum(-r, 0)
    k = np.searchsorted(np.asarray(starts), d, side="right") - 1
    if two_sided:
        k = np.where(r > 0, k + len(starts), k)
    return np.where(r > 0, -1, k) if causal else k


def forward(starts, two_sided, causal, H, Lq, Lk, off, table, dtype, pad=0, shift=0):
    b = mb.RelposBuckets(starts, two_sided, causal)
    room = torch.full((H * Lq * (Lk + pad) + shift + 64,), 5.0, dtype=dtype, device=DEV)
    out = torch.as_strided(room, (H, Lq, Lk), (Lq * (Lk + pad), Lk + pad, 1), shift)
    mb.relpos_bias_forward(b, table, KIND[table.dtype], H, Lq, Lk, off, out, KIND[dtype], Lq * (Lk + pad), Lk + pad)
    torch.cuda.synchronize()
    return out, room


SHAPES = [(1, 1, 1, 0), (3, 1, 777, 776), (2, 5, 3, 0), (1, 64, 64, 0), (3, 33, 47, 14), (2, 40, 1000, -30), (4, 257, 129, 5),
          (1, 300, 2100, 1700), (2, 7, 60, 100000), (2, 9, 60, -100000)]


@pytest.mark.parametrize("H,Lq,Lk,off", SHAPES)
@pytest.mark.parametrize("two_sided,causal", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_forward(H, Lq, Lk, off, two_sided, causal, dtype):
    table = torch.randn(len(STARTS) * (2 if two_sided else 1), H, device=DEV)
    out, _ = forward(STARTS, two_sided, causal, H, Lq, Lk, off, table, dtype)
    k = torch.from_numpy(bucket_table(STARTS, two_sided, causal, Lq, Lk, off)).to(DEV)
    want = torch.where(k < 0, float("-inf"), table.t()[:, k.clamp(min=0)]).to(dtype)
    assert torch.equal(out, want)


# Enough rows that a block writes several of them by whole windows of the vector.
@pytest.mark.parametrize("H,Lq,Lk,off,pad,shift", [(7, 61, 131, 0, 0, 0), (3, 129, 2049, 1900, 3, 1), (1, 300, 77, -5, 0, 3), (33, 8, 8, 0, 0, 0), (9, 31, 1, 3, 0, 0),
                                                   (2, 131, 4100, 4000, 12, 4), (260, 1, 40, 39, 1, 2), (40, 8, 4, 0, 5, 7)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_forward_of_many_rows(H, Lq, Lk, off, pad, shift, causal, dtype):
    table = torch.randn(2 * len(STARTS), H, device=DEV)
    out, room = forward(STARTS, True, causal, H, Lq, Lk, off, table, dtype, pad, shift)
    k = torch.from_numpy(bucket_table(STARTS, True, causal, Lq, Lk, off)).to(DEV)
    assert torch.equal(out, torch.where(k < 0, float("-inf"), table.t()[:, k.clamp(min=0)]).to(dtype))
    touched = torch.zeros_like(room, dtype=torch.bool)
    torch.as_strided(touched, out.shape, out.stride(), shift).fill_(True)
    assert bool((room[~touched] == 5.0).all())


@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 8), (1, 5), (0, 4)])
@pytest.mark.parametrize("table_dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forward_strides_and_types(pad, shift, table_dtype, dtype):
    H, Lq, Lk, off = 3, 70, 205, 40
    table = torch.randn(2 * len(STARTS), H, device=DEV).to(table_dtype)
    out, room = forward(STARTS, True, False, H, Lq, Lk, off, table, dtype, pad, shift)
    k = torch.from_numpy(bucket_table(STARTS, True, False, Lq, Lk, off)).to(DEV)
    assert torch.equal(out, table.float().t()[:, k].to(dtype))
    touched = torch.zeros_like(room, dtype=torch.bool)
    torch.as_strided(touched, out.shape, out.stride(), shift).fill_(True)
    assert (room[~touched] == 5.0).all()                  # nothing between the rows, before or behind


def test_forward_with_one_and_with_the_most_buckets():
    table = torch.randn(1, 2, device=DEV)
    out, _ = forward([0], False, False, 2, 30, 50, 0, table, torch.float32)
    assert torch.equal(out, table.t()[:, :, None].expand(2, 30, 50))
    starts = [3 * k for k in range(mb.RELPOS_MAX_BUCKETS)]
    table = torch.randn(2 * len(starts), 2, device=DEV)
    out, _ = forward(starts, True, False, 2, 500, 600, 50, table, torch.float32)
    k = torch.from_numpy(bucket_table(starts, True, False, 500, 600, 50)).to(DEV)
    assert torch.equal(out, table.t()[:, k])


def test_forward_values_that_overflow_or_are_not_finite():
    table = torch.tensor([[1e30, float("nan")], [float("inf"), -1e30]], device=DEV)
    out, _ = forward([0, 1], False, False, 2, 20, 20, 0, table, torch.float16)
    k = torch.from_numpy(bucket_table([0, 1], False, False, 20, 20, 0)).to(DEV)
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(table.t()[:, k].half()))


def backward(starts, two_sided, causal, off, grad, shape=None):
    B, H, Lq, Lk = shape or grad.shape
    b = mb.RelposBuckets(starts, two_sided, causal)
    out = torch.full((b.rows, H), 9.0, device=DEV)
    ws = torch.full((mb.relpos_bias_workspace_bytes(b, H),), 255, dtype=torch.uint8, device=DEV)
    sb, sh, sr, _ = grad.stride()
    mb.relpos_bias_backward(b, grad, KIND[grad.dtype], B, H, Lq, Lk, off, sb, sh, sr, out, ws, ws.numel())
    torch.cuda.synchronize()
    return out


def check_gradient(got, grad, starts, two_sided, causal, off):
    B, H, Lq, Lk = grad.shape
    k = bucket_table(starts, two_sided, causal, Lq, Lk, off).reshape(-1)
    g = grad.double().cpu().numpy().transpose(1, 0, 2, 3).reshape(H, B, -1)
    rows = len(starts) * (2 if two_sided else 1)
    for h in range(H):
        total, size = np.zeros(rows), np.zeros(rows)
        for b in range(B):
            keep = k >= 0
            total += np.bincount(k[keep], g[h, b][keep], rows)
            size += np.bincount(k[keep], np.abs(g[h, b][keep]), rows)
        err = np.abs(got[:, h].double().cpu().numpy() - total)
        assert (err <= 1024 * U * size + U * np.abs(total)).all(), (h, err.max())


@pytest.mark.parametrize("H,Lq,Lk,off", SHAPES)
@pytest.mark.parametrize("two_sided,causal", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_gradient(H, Lq, Lk, off, two_sided, causal, dtype):
    grad = torch.randn(3, H, Lq, Lk, device=DEV).to(dtype)
    check_gradient(backward(STARTS, two_sided, causal, off, grad), grad, STARTS, two_sided, causal, off)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1), (0, 4)])
def test_gradient_strides(dtype, pad, shift):
    """Rows apart, heads before the batch, a base off the vector boundary; what lies between is NaN and must not be read into the sums."""
    B, H, Lq, Lk = 4, 3, 150, 264
    room = torch.full((B * H * Lq * (Lk + pad) + 64,), float("nan"), dtype=dtype, device=DEV)
    grad = torch.as_strided(room, (B, H, Lq, Lk), (Lq * (Lk + pad), B * Lq * (Lk + pad), Lk + pad, 1), shift)
    grad.copy_(torch.randn(B, H, Lq, Lk, device=DEV))
    check_gradient(backward(STARTS, True, False, 20, grad), grad, STARTS, True, False, 20)


def test_gradient_of_a_broadcast_batch_and_a_large_batch():
    grad = torch.randn(1, 2, 60, 80, device=DEV).expand(7, 2, 60, 80)            # batch stride 0
    check_gradient(backward(STARTS, False, False, 0, grad), grad, STARTS, False, False, 0)
    grad = torch.randn(300, 1, 17, 24, device=DEV).bfloat16()
    check_gradient(backward(STARTS, True, False, 0, grad), grad, STARTS, True, False, 0)


def test_gradient_ignores_what_the_mask_hides():
    grad = torch.randn(2, 2, 200, 260, device=DEV)
    k = torch.from_numpy(bucket_table(STARTS, False, True, 200, 260, 30)).to(DEV)
    for bad in (float("nan"), float("inf"), -3.4e38):
        g = torch.where(k < 0, bad, grad)
        got = backward(STARTS, False, True, 30, g)
        check_gradient(got, torch.where(k < 0, 0.0, grad), STARTS, False, True, 30)
    every = torch.full((2, 2, 10, 16), float("nan"), device=DEV)                 # every key ahead: nothing counts
    assert (backward(STARTS, False, True, -100, every) == 0).all()


def test_gradient_of_nothing_is_zero():
    for shape in ((0, 2, 4, 4), (2, 2, 0, 4), (2, 2, 4, 0)):
        assert (backward(STARTS, True, False, 0, torch.empty(shape, device=DEV), shape) == 0).all()


def test_gradient_is_the_transpose_of_the_forward():
    """The forward is linear in the table: sum(grad * bias(way)) is the difference quotient along `way`, without an error of its own."""
    H, Lq, Lk, off = 3, 90, 140, 50
    grad = torch.randn(2, H, Lq, Lk, device=DEV)
    got = backward(STARTS, True, False, off, grad).double()
    way = torch.randn(2 * len(STARTS), H, device=DEV)
    bias, _ = forward(STARTS, True, False, H, Lq, Lk, off, way, torch.float32)
    diff = (grad.double() * bias.double()).sum()
    room = 1025 * U * (grad.double().abs() * bias.double().abs()).sum()
    assert abs((got * way.double()).sum() - diff) <= room


def test_gradient_is_the_same_every_time_and_on_a_side_stream():
    grad = (torch.randn(6, 4, 500, 520, device=DEV)).bfloat16()
    b = mb.RelposBuckets(STARTS, True, False)
    ws = torch.empty(mb.relpos_bias_workspace_bytes(b, 4), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    results = []
    for k in range(4):
        out = torch.full((b.rows, 4), 9.0, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        sb, sh, sr, _ = grad.stride()
        mb.relpos_bias_backward(b, grad, mb.DTYPE_BF16, 6, 4, 500, 520, 10, sb, sh, sr, out, ws, ws.numel(), side if k % 2 else None)
        torch.cuda.synchronize()
        results.append(out)
    assert all(torch.equal(results[0], r) for r in results)


@pytest.mark.parametrize("Lq", [65535 * 128 + 5, (1 << 29) - 1])
def test_forward_of_as_many_queries_as_there_may_be(Lq):
    """One key: the column is the table's rows by distance, then the last one to the end."""
    table = torch.tensor([[1.0], [2.0], [3.0]], device=DEV)
    b = mb.RelposBuckets([0, 1, 70])
    out = torch.zeros(Lq, dtype=torch.bfloat16, device=DEV)
    mb.relpos_bias_forward(b, table, mb.DTYPE_FP32, 1, Lq, 1, 0, out, mb.DTYPE_BF16, Lq, 1)
    torch.cuda.synchronize()
    assert float(out[0]) == 1.0 and bool((out[1:70] == 2.0).all()) and bool((out[70:] == 3.0).all())


# Blocks with long runs of patches (8 rows x 32 lanes of 16 bytes, or of four columns): several for every warp, runs that go on from one batch entry to the
# next, and bands of more than 768, after which the sums are handed on.  592 blocks are shared by the heads; from 297 heads on each has one.
@pytest.mark.parametrize("B,H,Lq,Lk,off,heads_alike", [(3, 5, 1000, 1200, 100, False), (3, 5, 997, 1203, 100, False), (17, 297, 400, 400, 0, True),
                                                     (17, 297, 397, 403, 10, True), (130, 297, 64, 136, -20, True), (900, 300, 9, 33, 5, True)])
@pytest.mark.parametrize("two_sided,causal", [(True, False), (False, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_many_patches(B, H, Lq, Lk, off, heads_alike, two_sided, causal, dtype):
    grad = torch.randn(B, 1 if heads_alike else H, Lq, Lk, device=DEV).to(dtype)
    got = backward(STARTS, two_sided, causal, off, grad.expand(B, H, Lq, Lk)).double()
    k = torch.from_numpy(bucket_table(STARTS, two_sided, causal, Lq, Lk, off)).to(DEV).reshape(-1)
    rows = len(STARTS) * (2 if two_sided else 1)
    for h in range(grad.shape[1]):
        g = grad[:, h].double().reshape(B, -1)
        total = torch.zeros(rows + 1, dtype=torch.float64, device=DEV).index_add_(0, k % (rows + 1), g.sum(0))[:rows]
        size = torch.zeros(rows + 1, dtype=torch.float64, device=DEV).index_add_(0, k % (rows + 1), g.abs().sum(0))[:rows]
        for x in (got if heads_alike else got[:, h:h + 1]).unbind(1):
            assert bool(((x - total).abs() <= 1024 * U * size + U * total.abs()).all()), float((x - total).abs().max())
