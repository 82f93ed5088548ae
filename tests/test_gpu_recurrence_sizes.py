"""Gated linear recurrence at the sizes that decide how a call is cut: chunks of 32 to 256 tokens (the small calls of the other tests have
chunks of 16), maps and walks taken in turn (more than 4,096 pieces of a kind), and the single-token kernel with sequences of several tokens.

The exact values: scans in 64 bits over spans of twice the length in each pass.

Tolerances, u = 2^-24, as bounds that run along with the recurrence.  z is off by 24 u z, a step or a map's step rounds four times at most, and
where chunks begin a state is put together from maps (7 of each of 3 levels and a kept state, two roundings each and one of what P was: 64 u); the
smallest chunks have 16 tokens.  So the error of a state grows by at most M u (48 z + 4), at every sixteenth token by 64 M u more, and shrinks by
1 - z, M the largest value or initial state.  The same for the sums G of the backward, with S_t = |grad_t| + (1 - z_{t+1}) S_{t+1} in the place of M."""
import numpy as np
import pytest
import torch

from paper_2305_01515_b200 import binding as mb
from test_gpu_recurrence import HALF_UNIT, KIND, TINY, U, Problem

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def scan(a, u):
    """x_t = a_t x_{t-1} + u_t along the first axis."""
    a, u, step = a.clone(), u.clone(), 1
    while step < len(u) and bool((a[step:] != 0).any()):
        u[step:] += a[step:] * u[:-step].clone()
        a[step:] *= a[:-step].clone()
        step *= 2
    return u


def workspace_bytes(N, D, chunk):
    """What the header's sizes come to for chunks of so many tokens: maps of four levels, eight to one, and the kept states."""
    n = [-(-N // chunk)]
    for _ in range(3):
        n.append(-(-n[-1] // 8))
    n.append(n[-1] + 1)
    counters = -(-(256 + 8 * sum(n) * -(-D // 32)) // 256) * 256
    return counters + 4 * (n[0] + 2 * sum(n)) * (-(-D // 4) * 4)


def borders(N, seed):
    """Offsets: long stretches without a border, short sequences, empty ones, and borders at and beside the multiples of 64 and 256."""
    r = np.random.RandomState(seed)
    at = [np.array([0, N, N, N - 1, N // 8, N // 8, N // 8])]
    for base in r.randint(N // 2, N - 2000, 40) // 256 * 256:
        at.append(base + r.choice([0, 1, 63, 64, 65, 127, 128, 129, 191, 193, 255, 256, 257, 511, 512, 513], 6))
    at.append(N // 4 + np.cumsum(r.randint(0, 40, 200)))               # many within a part
    at.append(N // 2 + np.cumsum(r.randint(100, 400, 100)))            # about one in a chunk
    at.append(r.randint(1, N // 8, 30))
    return np.sort(np.concatenate(at))


class Large:
    def __init__(self, N, D, dtype, padded, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.N, self.D, self.dtype, self.kind = N, D, dtype, KIND[dtype]
        off = borders(N, seed)
        self.S = len(off) - 1
        self.offsets = torch.from_numpy(off).to(DEV)

        def rows(x):
            if not padded:
                return x.to(dtype).contiguous()
            v = torch.as_strided(torch.full((N * (D + 5) + 16,), 7.0, device=DEV, dtype=dtype), (N, D), (D + 5, 1), 1)
            return v.copy_(x)

        def randn(*s):
            return torch.randn(*s, generator=g, device=DEV)

        # every channel has a time scale of its own, from a few tokens to more than a chunk
        self.gate = rows(randn(N, D) + torch.linspace(0.0, -9.0, D, device=DEV)[torch.randperm(D, generator=g, device=DEV)])
        self.value, self.grad = rows(randn(N, D)), rows(randn(N, D))
        self.h0, self.grad_final = randn(self.S, D), randn(self.S, D)
        self.out, self.d_gate, self.d_value = (rows(torch.full((1, 1), 9.0, device=DEV).expand(N, D)) for _ in range(3))
        self.final, self.d_h0 = torch.full((2, self.S, D), 9.0, device=DEV).unbind(0)
        self.entry = torch.full((mb.recurrence_chunks(N, D, self.kind), D), float("nan"), device=DEV)
        self.ws = torch.full((mb.recurrence_workspace_bytes(N, self.S, D, self.kind),), 255, dtype=torch.uint8, device=DEV)

    def run(self, in_place):
        h0 = self.h0
        if in_place:
            self.final.copy_(self.h0)
            h0 = self.final
        mb.recurrence_forward(self.gate, self.gate.stride(0), self.value, self.value.stride(0), self.kind, self.N, self.D, self.offsets, self.S, h0,
                              self.out, self.out.stride(0), self.final, self.entry, self.ws, self.ws.numel())
        assert mb.recurrence_status(self.ws) == 0
        mb.recurrence_backward(self.gate, self.gate.stride(0), self.value, self.value.stride(0), self.kind, self.N, self.D, self.offsets, self.S,
                               self.h0, self.entry, self.grad, self.grad.stride(0), self.grad_final, self.d_gate, self.d_gate.stride(0),
                               self.d_value, self.d_value.stride(0), self.d_h0, self.ws, self.ws.numel())
        assert mb.recurrence_status(self.ws) == 0

    def check(self, channels):
        N, off, c = self.N, self.offsets, torch.tensor(channels, device=DEV)
        f = lambda t: t.index_select(1, c).double()  # noqa: E731
        x, d, h0, gf = f(self.value), f(self.grad), f(self.h0), f(self.grad_final)
        z = torch.sigmoid(f(self.gate))
        at = torch.arange(N, device=DEV)
        seq = torch.bucketize(at, off[1:], right=True)
        first, last = (at == off[seq]).unsqueeze(1), (at == off[seq + 1] - 1).unsqueeze(1)
        full = (off[1:] > off[:-1]).unsqueeze(1)
        begins, ends = off[:-1].clamp(max=N - 1), (off[1:] - 1).clamp(min=0)
        keep = 1.0 - z
        M = max(float(x.abs().max()), float(h0.abs().max()))
        from_start = torch.where(first, 0.0, keep)
        h = scan(from_start, torch.where(first, keep * h0[seq] + z * x, z * x))
        border = 64.0 * (at % 16 == 0).double().unsqueeze(1)
        bound_h = scan(from_start, M * U * (48 * z + 4 + border))
        self.near("h", f(self.out), h, bound_h, self.dtype)
        self.near("final", f(self.final), torch.where(full, h[ends], h0), torch.where(full, bound_h[ends], 0.0))

        def back(a, u):
            return scan(a.flip(0), u.flip(0)).flip(0)

        after = torch.where(last, 0.0, torch.cat([keep[1:], keep[:1]]))
        G = back(after, torch.where(last, d + gf[seq], d))
        size = back(after, torch.where(last, d.abs() + gf[seq].abs(), d.abs()))
        step = U * size * (24 * z + 4)                                   # of (1 - z) G, as it comes to the token before; G itself rounds once
        came = torch.where(last, 0.0, torch.cat([step[1:], step[:1]]))
        bound_G = back(after, came + U * size * (1 + border + 64.0 * (at % 16 == 15).double().unsqueeze(1)))
        before = torch.where(first, h0[seq], torch.cat([h[:1], h[:-1]]))
        bound_before = torch.where(first, 0.0, torch.cat([bound_h[:1], bound_h[:-1]]))
        way, room = x - before, (x.abs() + before.abs())
        self.near("d_value", f(self.d_value), z * G, z * bound_G + 26 * U * z * size, self.dtype)
        self.near("d_gate", f(self.d_gate), z * keep * way * G, z * keep * (room * bound_G + size * bound_before) + 60 * U * z * size * room, self.dtype)
        self.near("d_h0", f(self.d_h0), torch.where(full, (keep * G)[begins], gf), torch.where(full, (keep * bound_G + step)[begins], 0.0))

    @staticmethod
    def near(what, got, want, bound, dtype=torch.float32):
        err = (got - want).abs()
        bad = ~(err <= bound + HALF_UNIT[dtype] * (want.abs() + bound) + TINY[dtype])
        assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), float(err[bad].max()))


# (tokens, channels, type, rows off every boundary, tokens of a chunk, maps and walks in turn)
CASES = [
    (80000, 8, torch.float32, False, 32, False),
    (160001, 33, torch.float16, False, 64, False),
    (310003, 40, torch.bfloat16, False, 128, False),
    (310003, 41, torch.float32, True, 128, False),
    (650001, 8, torch.float32, False, 256, False),
    (310007, 96, torch.float32, False, 256, False),
    (400001, 132, torch.float16, False, 256, False),
    (1100003, 3, torch.bfloat16, False, 256, True),
    (360001, 136, torch.float32, False, 256, True),
    (540001, 130, torch.bfloat16, True, 256, True),
    (140011, 1024, torch.bfloat16, False, 256, True),
]


@pytest.mark.parametrize("N,D,dtype,padded,chunk,in_turn", CASES)
def test_forward_and_backward_at_every_chunk_size(N, D, dtype, padded, chunk, in_turn):
    # the case is what its line says: the workspace shows the chunks, a strip is 32 lanes of as many channels as they hold
    assert mb.recurrence_workspace_bytes(N, 5, D, KIND[dtype]) == workspace_bytes(N, D, chunk)
    most = 2 if dtype == torch.float32 else 4
    lane = next(v for v in (4, 2, 1) if v <= most and (v == 1 or D > 16 * v))
    assert (-(-N // chunk) * -(-D // (32 * lane)) > 4096) == in_turn
    p = Large(N, D, dtype, padded, seed=N + D)
    p.run(in_place=padded)
    p.check(sorted({0, 1, D // 3, D // 2, D - 2, D - 1, min(63, D - 1), min(128, D - 1)}))


def test_same_result_every_time_with_maps_and_walks_in_turn():
    p = Large(360001, 136, torch.float32, False, seed=2)
    p.run(in_place=False)
    first = [t.clone() for t in (p.out, p.final, p.entry, p.d_gate, p.d_value, p.d_h0)]
    for _ in range(5):
        for t in (p.out, p.final, p.d_gate, p.d_value, p.d_h0):
            t.fill_(3.0)
        p.run(in_place=False)
        assert all(torch.equal(a, b) for a, b in zip(first, (p.out, p.final, p.entry, p.d_gate, p.d_value, p.d_h0)))


LENS = {
    "several among empty ones": [0, 3, 0, 0, 7, 0, 0, 0, 0, 1, 0, 12, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 2, 0],
    "one among empty ones": [0] * 200 + [300] + [0] * 200,
    "two of some": [1, 2, 0, 1, 1, 2, 0, 1] * 12,
    "the most tokens": [0] * 4095 + [4096],
    "more sequences than blocks": [1 if s % 40 == 3 else 0 for s in range(70000)],
}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("dtype,D", [(torch.float32, 5), (torch.bfloat16, 130)])
def test_a_thread_for_every_channel_of_a_sequence(lens, dtype, D):
    """No more tokens than sequences: the single-token kernel, here with several tokens in some of them."""
    p = Problem(LENS[lens], D, dtype, seed=20)
    assert p.N <= p.S and p.N <= 4096
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()
    state = p.h0.clone()                                   # kept states, in place
    mb.recurrence_forward(p.gate, p.D, p.value, p.D, p.kind, p.N, p.D, p.offsets, p.S, state, p.out, p.D, state, None, p.ws, p.ws.numel())
    assert torch.equal(state, p.final)


def test_single_token_kernel_checks_every_offset():
    lens = [0, 1, 2, 0, 0] * 1000
    p = Problem(lens, 8, torch.float32, seed=21)
    good = p.offsets.clone()
    p.forward()
    assert mb.recurrence_status(p.ws) == 0
    for k, bad in ((0, 1), (0, -1), (1, 3000), (2500, 0), (2500, 3001), (4999, -7), (5000, 2999), (5000, 3001)):
        p.offsets.copy_(good)
        p.offsets[k] = bad
        p.forward()
        assert mb.recurrence_status(p.ws) & 1, (k, bad)
    p.offsets.copy_(good)
    p.forward()
    assert mb.recurrence_status(p.ws) == 0
