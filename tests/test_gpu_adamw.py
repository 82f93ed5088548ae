"""AdamW over many tensors (mts_adamw_*) against the formula in 64 bits, and its 8-bit moments bit for bit against the same
operations in numpy's fp32 (which rounds every product and sum, as the kernel does).

Tolerances, u = 2^-24: m is two products and a sum of one rounding each (and the scaled gradient's): 4 u of the terms' sizes; v the
same with the square: 6 u.  The update carries half of v's relative error, a square root, a reciprocal factor, a quotient
(2 units) and m's error relative to its own terms: 16 u of rate * (terms of m) / root; the parameter two roundings."""
import numpy as np
import pytest
import torch

from paper_2305_01515_b200 import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
KIND = {torch.float32: mb.DTYPE_FP32, torch.float16: mb.DTYPE_FP16, torch.bfloat16: mb.DTYPE_BF16}
HALF_UNIT = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
B = mb.ADAMW_BLOCK
SIZES = [1, 2, 255, 256, 257, 0, 4096, 7, 10000, 2048, 2049, 33]


class Problem:
    def __init__(self, sizes=SIZES, param=torch.float32, grad=torch.float32, bits=32, master=False, shift=0, decays=None, seed=0,
                 lr=1e-2, decay=0.1, clip=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        make = lambda n, t, s: torch.zeros(n + shift + 8, device=DEV, dtype=t)[shift:shift + n].copy_(torch.randn(n, generator=g, device=DEV) * s)  # noqa: E731
        self.sizes, self.bits, self.lr, self.decay, self.pt, self.decays = sizes, bits, lr, decay, param, decays
        self.params = [make(n, param, 1.0) for n in sizes]
        self.masters = [make(n, torch.float32, 1.0) for n in sizes] if master else None
        if master:
            for p, w in zip(self.params, self.masters):
                p.copy_(w)
        self.grads = [make(n, grad, 10.0 ** -(k % 5)) for k, n in enumerate(sizes)]
        self.clip = None if clip is None else torch.tensor([clip], device=DEV)
        self.h = mb.AdamW(sizes, KIND[param], KIND[grad], bits, self.params, self.grads, self.masters, decays)
        room = [-(-n // B) * B for n in sizes]
        self.first = np.concatenate([[0], np.cumsum(room)]).astype(np.int64)
        assert self.h.elements == self.first[-1]
        self.state = torch.zeros(max(self.h.state_bytes, 1), dtype=torch.uint8, device=DEV)
        self.step_no = 0

    def step(self, seed=0, stream=None):
        self.step_no += 1
        mb.adamw_step(self.h, self.state, self.lr, 0.9, 0.999, 1e-8, self.decay, self.step_no, self.clip, seed, stream)

    def moments(self):
        m, v = torch.full((2, self.h.elements), 9.0, device=DEV).unbind(0)
        mb.adamw_export_state(self.h, self.state, m, v)
        torch.cuda.synchronize()
        return m.cpu().numpy(), v.cpu().numpy()

    def of(self, flat, k):
        return flat[self.first[k]:self.first[k] + self.sizes[k]]

    def check_step(self, seed=0):
        """One step against the formula, from the values that are there before it."""
        weights = [t.double().cpu().numpy() for t in (self.masters or self.params)]
        m0, v0 = self.moments()
        self.step(seed)
        m1, v1 = self.moments()
        clip = 1.0 if self.clip is None else float(self.clip)
        t = self.step_no
        for k, n in enumerate(self.sizes):
            g = self.grads[k].double().cpu().numpy() * clip
            mo, vo = self.of(m0, k).astype(np.float64), self.of(v0, k).astype(np.float64)
            m, v = 0.9 * mo + (1 - 0.9) * g, 0.999 * vo + (1 - 0.999) * g * g
            size = 0.9 * np.abs(mo) + (1 - 0.9) * np.abs(g)
            root = np.sqrt(v / (1 - 0.999 ** t)) + 1e-8
            rate = self.lr / (1 - 0.9 ** t)
            decay = self.lr * self.decay if self.decays is None or self.decays[k] else 0.0
            want = weights[k] * (1 - decay) - rate * m / root
            bound = 2 * U * (np.abs(weights[k]) + np.abs(want)) + 16 * U * rate * size / root
            if self.masters:
                assert (np.abs(self.masters[k].double().cpu().numpy() - want) <= bound).all()
                assert torch.equal(self.params[k], self.masters[k].to(self.pt))
            got = self.params[k].double().cpu().numpy()
            assert (np.abs(got - want) <= bound + HALF_UNIT[self.pt] * (np.abs(want) + bound) + TINY[self.pt]).all()
            if self.bits == 32:
                assert (np.abs(self.of(m1, k) - m) <= 4 * U * size).all() and (np.abs(self.of(v1, k) - v) <= 6 * U * v).all()
            else:          # within half a code for m and one for v (an eighth of the octave's start), or the smallest code
                top_m, top_v = ([np.repeat([np.abs(x[i:i + B]).max() for i in range(0, n, B)], B)[:n] for x in (m, v)] if n else (m, v))
                assert (np.abs(self.of(m1, k) - m) <= (1 / 16 + 1e-5) * np.abs(m) + 2.0 ** -15 * top_m).all()
                assert (np.abs(self.of(v1, k) - v) <= (1 / 8 + 1e-5) * v + 2.0 ** -31 * top_v).all()
        pads = np.ones(self.h.elements, bool)
        for k, n in enumerate(self.sizes):
            pads[self.first[k]:self.first[k] + n] = False
        assert (m1[pads] == 0).all() and (v1[pads] == 0).all()


@pytest.mark.parametrize("param,master", [(torch.float32, False), (torch.float16, False), (torch.float16, True), (torch.bfloat16, True)])
@pytest.mark.parametrize("grad", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_three_steps(param, master, grad, bits):
    p = Problem(param=param, grad=grad, bits=bits, master=master, decays=[k % 3 != 0 for k in range(len(SIZES))], clip=0.3)
    for k in range(3):
        p.check_step(seed=k)


@pytest.mark.parametrize("shift", [1, 3, 4])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16])
def test_tensors_off_the_vector_boundary(shift, bits, param):
    p = Problem(param=param, grad=torch.bfloat16, bits=bits, shift=shift, seed=1)
    p.check_step()
    p.check_step()
    for t, n in zip(p.params + p.grads, 2 * SIZES):        # what follows a tensor is not written
        assert (torch.as_strided(t, (8,), (1,), t.storage_offset() + n) == 0).all() if n else True


def test_one_tensor_many_tensors_and_nothing():
    Problem([1]).check_step()
    Problem([3] * 700, bits=8).check_step()
    q = Problem([0, 0])
    q.step()
    torch.cuda.synchronize()


def emulate(m, v, g, clip, seed, first):
    """The step's moments and their codes' values in numpy fp32, operation by operation (blocks of 256)."""
    f = np.float32
    g = (g.astype(f) * f(clip)).astype(f)
    m = m * f(0.9) + g * f(1.0 - 0.9)
    v = v * f(0.999) + (g * g) * f(1.0 - 0.999)
    return held(m, False, None), held(v, True, random_bits(len(m), seed, first))


def random_bits(n, seed, first):
    w = (np.arange(n, dtype=np.uint32) + np.uint32(first)) * np.uint32(0x9E3779B1) + np.uint32(seed * 0x85EBCA77 & 0xFFFFFFFF)
    w = (w ^ (w >> np.uint32(15))) * np.uint32(0x2C1B3C6D)
    w = (w ^ (w >> np.uint32(12))) * np.uint32(0x297A2D39)
    return (w >> np.uint32(16)) << np.uint32(4)


def held(x, second, add):
    out = np.zeros_like(x)
    base = 0x3F8 - (255 if second else 127)
    for i in range(0, len(x), B):
        c = x[i:i + B]
        top = np.abs(c).max()
        if top < 2.0 ** -120:
            continue
        inv = np.float32(1.0) / top
        a = np.uint32(0x80000) if add is None else add[i:i + B]
        q = np.minimum(((np.abs(c) * inv).astype(np.float32).view(np.uint32) + a) >> np.uint32(20), 0x3F8)
        q = np.where(c == 0, 0, np.maximum(q, base + 1)) if second else np.where(q > base, q, 0)
        y = np.where(q > base, (q << 20).astype(np.uint32).view(np.float32) * top, np.float32(0))
        out[i:i + B] = np.where(c < 0, -y, y)
    return out


@pytest.mark.parametrize("clip", [None, 0.37])
def test_8bit_moments_bit_for_bit(clip):
    p = Problem([1000, 256, 5, 40000], bits=8, seed=2, clip=clip)
    for seed in (0, 1, 0xFFFFFFFF):
        m0, v0 = p.moments()
        p.step(seed)
        m1, v1 = p.moments()
        for k, n in enumerate(p.sizes):
            m, v = emulate(p.of(m0, k), p.of(v0, k), p.grads[k].cpu().numpy(), 1.0 if clip is None else clip, seed, p.first[k])
            assert np.array_equal(p.of(m1, k), m) and np.array_equal(p.of(v1, k), v)


def test_8bit_second_moments_follow_their_mean():
    """3000 steps of one gradient per element: v approaches g^2 by a thousandth of the difference a step, far less than half a code.  The
    rounding is right in the mean: over 64 blocks the mean of v over g^2 (1 - 0.999^3000) is within 2 % (a code is at most 12.5 %, its
    spread over 16,384 elements a tenth of a percent); rounded to nearest it would stay where it first got stuck."""
    p = Problem([64 * B], bits=8, seed=3, lr=0.0)
    p.grads[0].copy_(torch.exp(torch.randn(64 * B, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))))
    for k in range(3000):
        p.step(seed=k)
    _, v = p.moments()
    g = p.grads[0].cpu().numpy().astype(np.float64)
    ratio = v / (g * g * (1 - 0.999 ** 3000))
    assert abs(ratio.mean() - 1.0) < 0.02 and ratio.min() > 0.5 and ratio.max() < 2.0


def test_import_and_export_are_inverse():
    for bits in (32, 8):
        p = Problem(bits=bits, seed=4)
        p.step()
        p.step()
        m, v = p.moments()
        other = torch.zeros_like(p.state)
        mb.adamw_import_state(p.h, other, torch.from_numpy(m).to(DEV), torch.from_numpy(v).to(DEV))
        mo, vo = torch.empty((2, p.h.elements), device=DEV).unbind(0)
        mb.adamw_export_state(p.h, other, mo, vo)
        torch.cuda.synchronize()
        # values that codes stand for are kept as they are (a block whose largest took its second largest code gets a smaller scale)
        assert np.array_equal(mo.cpu().numpy(), m) and np.array_equal(vo.cpu().numpy(), v)
    # rounding to nearest on the way in
    p = Problem([5000], bits=8, seed=5)
    m = torch.randn(p.h.elements, device=DEV)
    v = torch.rand(p.h.elements, device=DEV)
    mb.adamw_import_state(p.h, p.state, m, v)
    gm, gv = p.moments()
    assert np.array_equal(gm, held(m.cpu().numpy(), False, None)) and np.array_equal(gv, held(v.cpu().numpy(), True, None))


def test_gradients_that_are_not_finite():
    """They reach their own parameter; the moments of the rest of the block are as without them."""
    for bits in (32, 8):
        p, q = Problem([1000], bits=bits, seed=6), Problem([1000], bits=bits, seed=6)
        for t, x in ((p, (float("nan"), float("inf"))), (q, (0.0, 0.0))):
            t.grads[0][10], t.grads[0][700] = x
            t.step()
        (m, v), (mq, vq) = p.moments(), q.moments()
        torch.cuda.synchronize()
        rest = np.ones(1000, bool)
        rest[[10, 700]] = False
        assert torch.isnan(p.params[0][[10, 700]]).all()
        assert torch.equal(p.params[0][torch.from_numpy(rest).to(DEV)], q.params[0][torch.from_numpy(rest).to(DEV)])
        assert np.array_equal(m[:1000][rest], mq[:1000][rest]) and np.array_equal(v[:1000][rest], vq[:1000][rest])
        if bits == 8:
            assert (m[[10, 700]] == 0).all() and (v[[10, 700]] == 0).all()


def test_tiny_and_zero_gradients():
    p = Problem([600], bits=8, seed=7, lr=1e-2, decay=0.0)
    before = p.params[0].clone()
    p.grads[0].zero_()
    p.step()
    m, v = p.moments()
    assert torch.equal(p.params[0], before) and not m.any() and not v.any()
    p.grads[0].fill_(1e-30)                                # squares underflow: the update is bounded by m / eps
    p.step()
    m, v = p.moments()
    assert torch.isfinite(p.params[0]).all() and not v.any()


def test_new_gradient_pointers_and_a_side_stream():
    p, q = Problem(seed=8), Problem(seed=8)
    fresh = [torch.randn_like(g) for g in p.grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mb.adamw_set_grads(p.h, fresh, side)
    p.step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for g, f in zip(q.grads, fresh):
        g.copy_(f)
    q.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p.params, q.params))


def test_first_step_on_a_stream_that_does_not_wait_for_the_default_one():
    """The description is on the device when create returns: 3,000 tensors, the first step at once on a stream of its own."""
    sizes = [300] * 3000
    params, grads = torch.zeros(3000, 300, device=DEV), torch.ones(3000, 300, device=DEV)
    side = torch.cuda.Stream()
    for _ in range(3):
        params.zero_()
        state = torch.zeros(3000 * 512 * 8, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        h = mb.AdamW(sizes, 0, 0, 32, params.unbind(0), grads.unbind(0))
        assert h.state_bytes == state.numel()
        mb.adamw_step(h, state, 0.1, 0.9, 0.999, 1e-8, 0.0, 1, stream=side)
        torch.cuda.synchronize()
        assert float((params + 0.1).abs().max()) < 1e-6


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_gradient_whose_square_overflows(bits, grad):
    """One step with gradients of 1e20 and -3e38, then ordinary ones: a step of Adam moves a parameter by lr * sqrt(10) at most here ((1 - beta1) / sqrt(1 - beta2)
    = 0.1 / 0.0316, of corrected moments less), so ten of them stay within 32 lr.  The rest of the block is as without them."""
    p, q = (Problem([1000], grad=grad, bits=bits, seed=9, lr=1e-2, decay=0.0) for _ in range(2))
    hit = [10, 300, 301]
    rest = torch.ones(1000, dtype=torch.bool, device=DEV)
    rest[hit] = False
    start = p.params[0].clone()
    for k in range(10):
        g = torch.randn(1000, device=DEV, generator=torch.Generator(device=DEV).manual_seed(k)).to(grad)
        for x in (p, q):
            x.grads[0].copy_(g)
            x.grads[0][hit] = 0.0
        if k == 2:
            p.grads[0][hit] = torch.tensor([1e20, -3e38, 2e19], device=DEV).to(grad)
        if k > 2:
            p.grads[0][hit] = g[hit]
        p.step(seed=k)
        q.step(seed=k)
        moved = (p.params[0] - start).abs()
        assert float(moved.max()) <= 32 * 1e-2, (k, float(moved[hit].max()))
        if k == 2:
            assert torch.equal(p.params[0][hit], start[hit])
    assert torch.equal(p.params[0][rest], q.params[0][rest])
    m, v = p.moments()
    if bits == 8:
        assert np.isfinite(m).all() and np.isfinite(v).all() and (v[hit] > 0).all()
        assert float(moved[hit].min()) > 0
    else:
        assert np.isinf(v[hit]).all() and float(moved[hit].max()) == 0.0


def test_import_of_moments_that_are_not_finite():
    """Either one of an element: both are 0, the others as without it."""
    p = Problem([700], bits=8, seed=10)
    m = torch.randn(p.h.elements, device=DEV)
    v = torch.rand(p.h.elements, device=DEV)
    clean = [x.clone() for x in (m, v)]
    hit = [3, 4, 300, 301]
    for x in clean:
        x[hit] = 0.0
    m[3], m[300], v[4], v[301] = float("inf"), float("nan"), float("inf"), float("nan")
    mb.adamw_import_state(p.h, p.state, m, v)
    got = p.moments()
    mb.adamw_import_state(p.h, p.state, *clean)
    want = p.moments()
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    v[[3, 4, 300, 301, 600]], m[[3, 4, 300, 301]] = torch.tensor([0.0, -0.0, -1.0, -float("inf"), -0.0], device=DEV), 0.0
    clean[1][600] = 0.0
    mb.adamw_import_state(p.h, p.state, m, v)
    got = p.moments()
    mb.adamw_import_state(p.h, p.state, *clean)
    assert got[0][600] != 0 and all(np.array_equal(a, b) for a, b in zip(got, p.moments()))
