"""Gated linear recurrence (mts_recurrence_*) against a plain recurrence in 64 bits.

Tolerances, with u = 2^-24: z = 1 / (1 + exp(-g)) carries at most 24 u relative for the gates used here (|g| < 20: the fast
exponential is off by about 2 + 1.2 |g| units, the sum and the reciprocal by one each).  A state is a convex combination of values of
size at most M, so a wrong z adds 2 M z 24 u per step, which the factors (1 - z) of the later steps sum to 48 M u, and a step rounds three
times, products of factors along the way once more: 4 M u per step.  Hence |h - exact| <= M u (48 + 4 t) after t steps, and
alike for the sums G of the backward with the size of their terms added up.  16-bit outputs add half a unit of their type."""
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


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Problem:
    def __init__(self, lens, D, dtype, seed=0, h0=True, layout="packed", gate_shift=-1.0, grads=True):
        """layout: packed rows; "halves": gate and value are the halves of one projection with padded rows; "odd": bases and strides
        on no boundary but the element's."""
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.D, self.dtype, self.kind = np.asarray(lens, np.int64), D, dtype, KIND[dtype]
        self.S, self.N = len(lens), int(np.sum(lens))
        N, S = self.N, self.S
        self.off = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int64)
        self.offsets = torch.from_numpy(self.off).to(DEV)

        def rows(x):
            if layout == "packed":
                return x.to(dtype).contiguous()
            room = torch.full((N * (D + 5) + 16,), 7.0, device=DEV, dtype=dtype)
            v = torch.as_strided(room, (N, D), (D + 5, 1), 1)
            v.copy_(x)
            return v

        randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        gate, value = randn(N, D) * 2.0 + gate_shift, randn(N, D)
        if layout == "halves":
            both = torch.empty(N, 2 * D + 8, device=DEV, dtype=dtype)
            self.gate, self.value = both[:, :D], both[:, D:2 * D]
            self.gate.copy_(gate)
            self.value.copy_(value)
        else:
            self.gate, self.value = rows(gate), rows(value)
        self.h0 = randn(S, D) if h0 else None
        self.grad = rows(randn(N, D)) if grads else None
        self.grad_final = randn(S, D) if grads and h0 else None
        self.out = rows(torch.full((N, D), 9.0, device=DEV))
        self.d_gate, self.d_value = rows(torch.full((N, D), 9.0, device=DEV)), rows(torch.full((N, D), 9.0, device=DEV))
        self.final = torch.full((S, D), 9.0, device=DEV)
        self.d_h0 = torch.full((S, D), 9.0, device=DEV)
        self.entry = torch.full((max(mb.recurrence_chunks(N, D, self.kind), 1), D), float("nan"), device=DEV)
        self.ws = torch.full((max(mb.recurrence_workspace_bytes(N, S, D, self.kind), 256),), 255, dtype=torch.uint8, device=DEV)

    @staticmethod
    def stride(t):
        return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))

    def forward(self, stream=None, entry=True):
        mb.recurrence_forward(self.gate, self.stride(self.gate), self.value, self.stride(self.value), self.kind, self.N, self.D,
                              self.offsets, self.S, self.h0, self.out, self.stride(self.out), self.final,
                              self.entry if entry else None, self.ws, self.ws.numel(), stream)

    def backward(self, stream=None):
        mb.recurrence_backward(self.gate, self.stride(self.gate), self.value, self.stride(self.value), self.kind, self.N, self.D,
                               self.offsets, self.S, self.h0, self.entry, self.grad, self.stride(self.grad), self.grad_final,
                               self.d_gate, self.stride(self.d_gate), self.d_value, self.stride(self.d_value), self.d_h0,
                               self.ws, self.ws.numel(), stream)

    def exact(self, gate=None, value=None, h0=None):
        """States, final states and a bound of their size, in 64 bits."""
        gate = f64(self.gate) if gate is None else gate
        value = f64(self.value) if value is None else value
        h0 = (f64(self.h0) if self.h0 is not None else np.zeros((self.S, self.D))) if h0 is None else h0
        z = 1.0 / (1.0 + np.exp(-gate))
        h, before, final = np.zeros_like(value), np.zeros_like(value), h0.copy()
        for s in range(self.S):
            x = h0[s].copy()
            for t in range(self.off[s], self.off[s + 1]):
                before[t] = x
                x = x + z[t] * (value[t] - x)
                h[t] = x
            final[s] = x
        return z, h, before, final

    def check_forward(self):
        z, h, _, final = self.exact()
        M = max(np.abs(f64(self.value)).max(initial=0.0), np.abs(f64(self.h0)).max(initial=0.0) if self.h0 is not None else 0.0)
        steps = np.concatenate([np.arange(n) + 1 for n in self.lens] + [np.zeros(0)])[:, None]
        bound = M * U * (48 + 4 * steps)
        err = np.abs(f64(self.out) - h)
        assert (err <= bound + HALF_UNIT[self.dtype] * (np.abs(h) + bound) + TINY[self.dtype]).all(), err.max()
        assert (np.abs(f64(self.final) - final) <= M * U * (48 + 4 * self.lens[:, None])).all()
        assert mb.recurrence_status(self.ws) == 0

    def check_backward(self):
        z, h, before, _ = self.exact()
        d, x = f64(self.grad), f64(self.value)
        gf = f64(self.grad_final) if self.grad_final is not None else np.zeros((self.S, self.D))
        want_g, want_x, want_0 = np.zeros_like(d), np.zeros_like(d), gf.copy()
        M = max(np.abs(x).max(initial=0.0), np.abs(f64(self.h0)).max(initial=0.0) if self.h0 is not None else 0.0)
        bound_G, bound_0, size_G = np.zeros_like(d), np.zeros_like(gf), np.zeros_like(d)
        for s in range(self.S):
            carry, size = gf[s].copy(), np.abs(gf[s])
            top = size.copy()
            for k, t in enumerate(range(self.off[s + 1] - 1, self.off[s] - 1, -1)):
                G, size = d[t] + carry, np.abs(d[t]) + size
                top = np.maximum(top, size)
                want_x[t] = z[t] * G
                want_g[t] = z[t] * (1 - z[t]) * (x[t] - before[t]) * G
                carry, size = (1 - z[t]) * G, (1 - z[t]) * size
                size_G[t], bound_G[t] = top, top * U * (48 + 4 * (k + 1))
                bound_0[s] = bound_G[t]
            want_0[s] = carry
        steps = np.concatenate([np.arange(n) + 1 for n in self.lens] + [np.zeros(0)])[:, None]
        bound_h = M * U * (48 + 4 * steps)
        bound_x = bound_G + 26 * U * size_G
        bound_g = 0.25 * (2 * M * bound_G + size_G * bound_h) + 60 * U * 2 * M * size_G * 0.25
        for got, want, b in ((self.d_value, want_x, bound_x), (self.d_gate, want_g, bound_g)):
            err = np.abs(f64(got) - want)
            assert (err <= b + HALF_UNIT[self.dtype] * (np.abs(want) + b) + TINY[self.dtype]).all(), err.max()
        assert (np.abs(f64(self.d_h0) - want_0) <= bound_0 + 26 * U * np.abs(want_0)).all()
        assert mb.recurrence_status(self.ws) == 0


LENS = {
    "one token": [1],
    "single tokens": [1] * 37,
    "one sequence": [333],
    "chunk borders": [64, 1, 63, 128, 65, 127, 2],
    "empty ones": [0, 0, 5, 0, 70, 0, 0, 0, 1, 0],
    "mixed": [3, 200, 0, 17, 64, 0, 0, 129, 1, 1, 1, 90],
}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [1, 7, 64, 132])
def test_forward_and_backward(lens, dtype, D):
    p = Problem(LENS[lens], D, dtype, seed=D)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("layout", ["halves", "odd"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [5, 96, 256])
def test_strided_rows(layout, dtype, D):
    p = Problem([70, 0, 3, 130, 64], D, dtype, seed=3, layout=layout)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()
    if layout == "odd":                                    # what lies between the rows is not written
        for t in (p.out, p.d_gate, p.d_value):
            room = torch.as_strided(t, (p.N - 1, 5), (D + 5, 1), t.storage_offset() + D)
            assert (room == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_sequences_cross_many_chunks(dtype):
    """Sequences over many chunks, with slow gates so that a state reaches far, beside short ones."""
    p = Problem([9000, 1, 0, 5003, 64, 20011, 7], 40, dtype, seed=5, gate_shift=-6.0)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


def test_without_initial_state_and_final_gradient():
    p = Problem([10, 100, 0, 1], 33, torch.float32, seed=6, h0=False)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


def test_no_tokens_and_no_sequences():
    p = Problem([0, 0, 0], 16, torch.float32, seed=7)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    assert torch.equal(p.final, p.h0) and torch.equal(p.d_h0, p.grad_final)
    q = Problem([], 16, torch.float32, seed=7)
    q.forward()
    q.backward()
    torch.cuda.synchronize()


def test_kept_states_updated_in_place_token_by_token():
    """h_final == h0: five single-token calls give what one call over the five tokens gives, within the tolerance of both."""
    p = Problem([5] * 9, 48, torch.float32, seed=8)
    p.forward()
    state, off = p.h0.clone(), torch.arange(10, device=DEV)
    ws = torch.empty(mb.recurrence_workspace_bytes(9, 9, 48, p.kind), dtype=torch.uint8, device=DEV)
    for t in range(5):
        g, x = p.gate.view(9, 5, 48)[:, t], p.value.view(9, 5, 48)[:, t]        # strided rows
        out = torch.empty(9, 48, device=DEV)
        mb.recurrence_forward(g, 5 * 48, x, 5 * 48, p.kind, 9, 48, off, 9, state, out, 48, state, None, ws, ws.numel())
        assert torch.equal(out, state)
    M = float(p.value.abs().max().maximum(p.h0.abs().max()))
    assert float((state - p.final).abs().max()) <= 2 * M * U * (48 + 4 * 5)


def test_infinite_values_stay_in_their_sequence():
    p = Problem([40, 64, 30, 200, 0, 10], 24, torch.float32, seed=9)
    p.value[50] = float("inf")
    p.value[134 + 100] = float("nan")
    p.grad[300] = float("nan")
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    for t in (p.out, p.d_gate, p.d_value):
        assert torch.isfinite(t[:40]).all() and torch.isfinite(t[104:134]).all() and torch.isfinite(t[334:]).all()
    assert torch.isfinite(p.final[[0, 2, 4, 5]]).all() and torch.isfinite(p.d_h0[[0, 2, 4, 5]]).all()
    assert not torch.isfinite(p.final[1]).any() and torch.isnan(p.final[3]).all()
    assert torch.isnan(p.d_h0[3]).all()


def test_saturated_gates():
    """Gates of both infinities: the state is kept as it is, or replaced; the gradient of the gate is 0."""
    p = Problem([6, 70], 8, torch.float32, seed=10)
    p.gate[2::3] = float("-inf")
    p.gate[0::3] = float("inf")
    p.gate[1::3] = -3e38
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    want = p.value.clone()
    want[1::3] = want[0::3][:len(want[1::3])]
    want[2::3] = want[0::3][:len(want[2::3])]
    assert torch.equal(p.out, want)
    assert (p.d_gate == 0).all() and torch.isfinite(p.d_value).all()


def test_same_result_every_time_and_on_a_side_stream():
    p = Problem([5000, 3, 0, 700, 64, 3000], 128, torch.bfloat16, seed=11, gate_shift=-4.0)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    first = [t.clone() for t in (p.out, p.final, p.entry, p.d_gate, p.d_value, p.d_h0)]
    side = torch.cuda.Stream()
    for _ in range(5):
        for t in (p.out, p.final, p.d_gate, p.d_value, p.d_h0):
            t.fill_(3.0)
        side.wait_stream(torch.cuda.current_stream())
        p.forward(side)
        p.backward(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for a, b in zip(first, (p.out, p.final, p.entry, p.d_gate, p.d_value, p.d_h0)):
            assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))


def test_gradient_against_differences():
    """Central differences of the 64-bit recurrence along random directions; their own error is of order 1e-9."""
    p = Problem([12, 0, 70, 1], 6, torch.float32, seed=12)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    rng = np.random.default_rng(0)
    d, gf = f64(p.grad), f64(p.grad_final)
    base = [f64(p.gate), f64(p.value), f64(p.h0)]

    def loss(x):
        _, h, _, final = p.exact(*x)
        return (h * d).sum() + (final * gf).sum()

    for k, got in enumerate((p.d_gate, p.d_value, p.d_h0)):
        for _ in range(3):
            way = rng.standard_normal(base[k].shape)
            e = 1e-5
            up, down = list(base), list(base)
            up[k], down[k] = base[k] + e * way, base[k] - e * way
            diff = (loss(up) - loss(down)) / (2 * e)
            # every term of the product carries at most a few hundred u of the size of G (at most 71 terms) times values (at most 2 M)
            M = np.abs(base[1]).max() + np.abs(base[2]).max()
            room = 400 * U * np.abs(way).sum() * (np.abs(d).max() * 71 + np.abs(gf).max()) * max(1.0, 2 * M) + 1e-6 * abs(diff)
            assert abs(float((f64(got) * way).sum()) - diff) <= room


def test_offsets_out_of_order_are_clamped_and_reported():
    p = Problem([10, 20, 30], 16, torch.float32, seed=13)
    for bad in ([0, 25, 10, 60], [0, 10, 30, 1000], [-5, 10, 30, 60], [0, 10, 30, 40], [7, 10, 30, 60]):
        p.offsets.copy_(torch.tensor(bad))
        p.forward()
        assert mb.recurrence_status(p.ws) & 1
        p.backward()
        assert mb.recurrence_status(p.ws) & 1
