"""The operators of the sequence tower beside the embedding tables, as cases to measure: a gated linear recurrence over
packed ragged histories, the learned relative position bias of the attention over them, and the AdamW step of the
tower's dense parameters.  `run` computes a case with the library (`own` true) or in plain torch operations."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
BLOCK = 256                                   # elements that share a scale in the 8-bit states
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 1e-3


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new event for each of 192 users whose states are kept: the serving step
        dict(name="recurrence_step", op="recurrence", dir="fwd", S=192, N=192, D=128, lens=0, dtype="fp32"),
        # scoring a batch of 1,000 histories of very different lengths, some of them empty
        dict(name="recurrence_fwd_ragged", op="recurrence", dir="fwd", S=1000, N=120007, D=256, lens=11, dtype="bf16"),
        # the same in training, forward and backward, with a width that is no power of two
        dict(name="recurrence_train_ragged", op="recurrence", dir="train", S=2048, N=250001, D=200, lens=12, dtype="bf16"),
        # one very long event stream: no parallelism over sequences
        dict(name="recurrence_fwd_long", op="recurrence", dir="fwd", S=1, N=524287, D=256, lens=13, dtype="fp16"),
        # the newest query against all keys: the single-token row of the bias
        dict(name="bias_row", op="bias", dir="fwd", B=1, H=8, Lq=1, Lk=2001, off=2000, n=32, far=128, two=False, causal=True, dtype="fp32"),
        # the bias of an encoder layer over histories of odd length
        dict(name="bias_fwd_odd", op="bias", dir="fwd", B=1, H=12, Lq=1023, Lk=1023, off=0, n=16, far=128, two=True, causal=False, dtype="bf16"),
        # a causal layer over long histories
        dict(name="bias_fwd_long", op="bias", dir="fwd", B=1, H=16, Lq=4096, Lk=4096, off=0, n=32, far=1024, two=False, causal=True, dtype="bf16"),
        # the table's gradient from the attention scores' gradient, summed over the batch
        dict(name="bias_grad", op="bias", dir="bwd", B=16, H=8, Lq=1024, Lk=1024, off=0, n=16, far=128, two=True, causal=False, dtype="bf16"),
        # the same in single precision, causal, with odd lengths and a prefix of keys
        dict(name="bias_grad_odd", op="bias", dir="bwd", B=5, H=12, Lq=777, Lk=1001, off=224, n=32, far=512, two=False, causal=True, dtype="fp32"),
        # a small ranking tower: twelve tensors, most of them tiny
        dict(name="adamw_small", op="adamw", tensors=12, total=180000, bits=32, param="fp32", grad="fp32", master=False, shift=0, sizes=21),
        # a large tower in bf16 with fp32 master weights
        dict(name="adamw_master", op="adamw", tensors=150, total=120000000, bits=32, param="bf16", grad="bf16", master=True, shift=0, sizes=22),
        # the states in 8 bits, over many tensors of odd sizes
        dict(name="adamw_8bit", op="adamw", tensors=333, total=100000000, bits=8, param="fp32", grad="bf16", master=False, shift=0, sizes=23),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(("recurrence", "bias", "adamw"))
    if op == "recurrence":
        D = rng.choice((_log(rng, 16, 1024), 8 * _log(rng, 2, 128)))
        N = _log(rng, 64, 50000000 // D)
        S = min(N, _log(rng, 1, 4096))
        return dict(op=op, dir=rng.choice(("fwd", "train")), S=S, N=N, D=D, lens=rng.randrange(1, 1 << 20),
                    dtype=rng.choice(tuple(TYPES)))
    if op == "bias":
        B, H = _log(rng, 1, 16), rng.randint(1, 16)
        Lq = rng.choice((1, _log(rng, 2, 2048), 8 * _log(rng, 1, 256)))
        Lk = rng.choice((Lq, Lq + _log(rng, 1, 900), 8 * _log(rng, 1, 256)))
        two = rng.random() < 0.5
        return dict(op=op, dir=rng.choice(("fwd", "bwd")), B=B, H=H, Lq=Lq, Lk=Lk, off=max(Lk - Lq, 0) if rng.random() < 0.5 else 0,
                    n=rng.choice((8, 16, 32)), far=rng.choice((64, 128, 500, 2048)), two=two,
                    causal=not two and rng.random() < 0.7, dtype=rng.choice(tuple(TYPES)))
    tensors = _log(rng, 1, 400)
    param = rng.choice(tuple(TYPES))
    return dict(op=op, tensors=tensors, total=max(_log(rng, 1000, 100000000), 4 * tensors), bits=rng.choice((8, 32)), param=param,
                grad=rng.choice((param, "fp32")), master=param != "fp32" and rng.random() < 0.7, shift=rng.choice((0, 0, 1)),
                sizes=rng.randrange(1, 1 << 20))


def lengths(case):
    """Lengths of the case's sequences: all one where N == S and lens is 0, else spread widely, a tenth of them empty."""
    S, N = case["S"], case["N"]
    if case["lens"] == 0:
        return np.full(S, N // S, np.int64)
    r = np.random.RandomState(case["lens"])
    w = r.lognormal(0.0, 1.0, S) * (r.rand(S) > 0.1)
    w[r.randint(S)] += 1.0
    n = np.floor(w / w.sum() * N).astype(np.int64)
    n[np.argmax(n)] += N - n.sum()
    return n


def tensor_sizes(case):
    """Sizes of the case's tensors: a few large ones hold most of the elements, biases and scales are tiny; the first third, at least one
    of them, are the vectors that take no weight decay."""
    r = np.random.RandomState(case["sizes"])
    w = r.lognormal(0.0, 2.0, case["tensors"])
    w.sort()
    n = np.maximum(np.floor(w / w.sum() * case["total"]).astype(np.int64), 1)
    n[-1] += max(case["total"] - int(n.sum()), 0)
    return n


def starts_of(case):
    """First distance of each bucket: the first half of the buckets hold one distance each, the others grow evenly in the logarithm
    and the last begins at `far`; in whole numbers, so that no rounding of a logarithm moves a border."""
    n, far = case["n"], case["far"]
    e = n // 2
    s = list(range(e))
    for k in range(n - e):                    # smallest d with (d / e)^(n-e-1) >= (far / e)^k
        p, d = max(n - e - 1, 1), e
        hi = max(far, e)
        while d < hi:
            mid = (d + hi) // 2
            if mid ** p * e ** k >= far ** k * e ** p:
                hi = mid
            else:
                d = mid + 1
        s.append(d)
    return s


def work(case):
    if case["op"] == "recurrence":
        n, e, S = case["N"] * case["D"], SIZE[case["dtype"]], case["S"] * case["D"] * 4
        b = 3 * n * e + 2 * S + 8 * (case["S"] + 1)
        if case["dir"] == "train":
            b += 5 * n * e + 2 * S
        return {"bytes": b, "flops": (8 if case["dir"] == "fwd" else 24) * n}
    if case["op"] == "bias":
        H, Lq, Lk, e = case["H"], case["Lq"], case["Lk"], SIZE[case["dtype"]]
        t = case["n"] * (2 if case["two"] else 1) * H * 4
        if case["dir"] == "fwd":
            return {"bytes": H * Lq * Lk * e + t, "flops": 0}
        seen = Lq * Lk
        if case["causal"]:                    # what a mask rules out has no gradient and need not be read
            i = np.arange(Lq, dtype=np.int64)
            seen = int(np.clip(i + case["off"] + 1, 0, Lk).sum())
        return {"bytes": case["B"] * H * seen * e + t, "flops": case["B"] * H * seen}
    n = int(tensor_sizes(case).sum())
    p, g = SIZE[case["param"]], SIZE[case["grad"]]
    b = n * ((p + 8 if case["master"] else 2 * p) + g)
    # 8 bits: the codes are read and written, and the values that they stand for are written out
    b += n * 16 if case["bits"] == 32 else n * (4 + 8) + 16 * (n // BLOCK)
    return {"bytes": b, "flops": 16 * n}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case)
    {"recurrence": _prepare_recurrence, "bias": _prepare_bias, "adamw": _prepare_adamw}[case["op"]](s, case, g)
    return s


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _prepare_recurrence(s, case, g):
    N, D, S, t = case["N"], case["D"], case["S"], TYPES[case["dtype"]]
    n = lengths(case)
    s["longest"] = int(n.max())
    s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(DEV)
    # gate logits: every channel has a time scale of its own, from a few events to hundreds
    scale = torch.linspace(0.0, -5.0, D, device=DEV)
    s["gate"] = (_randn(g, N, D) + scale).to(t)
    s["value"] = _randn(g, N, D).to(t)
    s["h0"] = 0.5 * _randn(g, S, D)
    train = case["dir"] == "train"
    if train:
        s["grad"] = _randn(g, N, D).to(t)
        s["grad_final"] = _randn(g, S, D)
    if own:
        from paper_2305_01515_b200 import binding as mb

        s["mb"], s["kind"] = mb, {"fp32": mb.DTYPE_FP32, "fp16": mb.DTYPE_FP16, "bf16": mb.DTYPE_BF16}[case["dtype"]]
        s["h"] = torch.empty(N, D, dtype=t, device=DEV)
        s["final"] = torch.empty(S, D, device=DEV)
        s["ws"] = torch.empty(mb.recurrence_workspace_bytes(N, S, D, s["kind"]), dtype=torch.uint8, device=DEV)
        if train:
            s["entry"] = torch.empty(mb.recurrence_chunks(N, D, s["kind"]), D, device=DEV)
            s["d_gate"], s["d_value"] = torch.empty_like(s["gate"]), torch.empty_like(s["value"])
            s["d_h0"] = torch.empty(S, D, device=DEV)


def _prepare_bias(s, case, g):
    t, H = TYPES[case["dtype"]], case["H"]
    rows = case["n"] * (2 if case["two"] else 1)
    s["starts"] = torch.tensor(starts_of(case), device=DEV)
    s["table"] = _randn(g, rows, H)
    if case["dir"] == "bwd":
        # gradients of scores: small, and of both signs
        s["grad"] = (_randn(g, case["B"], H, case["Lq"], case["Lk"]) * 0.01 + 0.001).to(t)
    if own:
        from paper_2305_01515_b200 import binding as mb

        s["mb"], s["kind"] = mb, {"fp32": mb.DTYPE_FP32, "fp16": mb.DTYPE_FP16, "bf16": mb.DTYPE_BF16}[case["dtype"]]
        s["plan"] = mb.RelposBuckets(starts_of(case), two_sided=case["two"], causal=case["causal"])
        if case["dir"] == "fwd":
            s["out"] = torch.empty(H, case["Lq"], case["Lk"], dtype=t, device=DEV)
        else:
            s["out"] = torch.empty(rows, H, device=DEV)
            s["ws"] = torch.empty(mb.relpos_bias_workspace_bytes(s["plan"], H), dtype=torch.uint8, device=DEV)


def _prepare_adamw(s, case, g):
    sizes = tensor_sizes(case)
    room = (sizes + BLOCK - 1) // BLOCK * BLOCK
    at = np.concatenate([[0], np.cumsum(room)])
    P, shift = int(at[-1]), case["shift"]
    tp, tg = TYPES[case["param"]], TYPES[case["grad"]]
    # all tensors lie in one buffer, each from a multiple of 256 elements on; what is between them stays zero
    seq = torch.from_numpy(np.repeat(np.arange(len(sizes)), room // BLOCK)).to(DEV)
    end = torch.from_numpy(at[:-1] + sizes).to(DEV)
    used = (torch.arange(P, device=DEV).view(-1, BLOCK) < end[seq].unsqueeze(1)).view(-1)

    def flat(x, dtype):
        b = torch.zeros(P + shift, dtype=dtype, device=DEV)[shift:]
        b.copy_(x * used)
        return b

    weights = _randn(g, P) * 0.05
    spread = torch.exp(2.0 * torch.randn(P // BLOCK, generator=g, device=DEV)).repeat_interleave(BLOCK)
    s["param"] = flat(weights, tp)
    s["master"] = flat(weights, torch.float32) if case["master"] else None
    s["grad"] = flat(_randn(g, P) * spread * 1e-3, tg)
    m0, v0 = _randn(g, P) * spread * 3e-4 * used, (_randn(g, P) * spread * 1e-3).square() * used
    s["clip"] = torch.tensor([0.7], device=DEV)
    s["step"] = 1000
    vectors = max(1, len(sizes) // 3)
    s["decays"] = (seq >= vectors).to(torch.float32).unsqueeze(1)
    if own:
        from paper_2305_01515_b200 import binding as mb

        kinds = {"fp32": mb.DTYPE_FP32, "fp16": mb.DTYPE_FP16, "bf16": mb.DTYPE_BF16}
        s["mb"] = mb
        cut = lambda b: [b[at[k]:at[k] + sizes[k]] for k in range(len(sizes))]  # noqa: E731
        s["plan"] = mb.AdamW([int(n) for n in sizes], kinds[case["param"]], kinds[case["grad"]], case["bits"], cut(s["param"]),
                             cut(s["grad"]), cut(s["master"]) if case["master"] else None,
                             decays=[k >= vectors for k in range(len(sizes))])
        s["state"] = torch.zeros(s["plan"].state_bytes, dtype=torch.uint8, device=DEV)
        mb.adamw_import_state(s["plan"], s["state"], m0, v0)
        s["m"], s["v"] = ((torch.empty(P, device=DEV), torch.empty(P, device=DEV)) if case["bits"] == 8 else
                          s["state"].view(torch.float32)[:2 * P].view(2, P).unbind(0))
    elif case["bits"] == 8:
        s["m"], s["v"] = _held_first(m0), _held_second(v0, None)
    else:
        s["m"], s["v"] = m0, v0


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"recurrence": _own_recurrence, "bias": _own_bias, "adamw": _own_adamw}[op](s, s["case"])
    return {"recurrence": _plain_recurrence, "bias": _plain_bias, "adamw": _plain_adamw}[op](s, s["case"])


def _own_recurrence(s, case):
    mb, N, D, S, k = s["mb"], case["N"], case["D"], case["S"], s["kind"]
    train = case["dir"] == "train"
    mb.recurrence_forward(s["gate"], D, s["value"], D, k, N, D, s["offsets"], S, s["h0"], s["h"], D, s["final"],
                          s["entry"] if train else None, s["ws"], s["ws"].numel())
    if not train:
        return {"h": s["h"], "final": s["final"]}
    mb.recurrence_backward(s["gate"], D, s["value"], D, k, N, D, s["offsets"], S, s["h0"], s["entry"], s["grad"], D, s["grad_final"],
                           s["d_gate"], D, s["d_value"], D, s["d_h0"], s["ws"], s["ws"].numel())
    return {"h": s["h"], "final": s["final"], "d_gate": s["d_gate"], "d_value": s["d_value"], "d_h0": s["d_h0"]}


def _own_bias(s, case):
    mb, H, Lq, Lk, off = s["mb"], case["H"], case["Lq"], case["Lk"], case["off"]
    if case["dir"] == "fwd":
        mb.relpos_bias_forward(s["plan"], s["table"], mb.DTYPE_FP32, H, Lq, Lk, off, s["out"], s["kind"], Lq * Lk, Lk)
    else:
        mb.relpos_bias_backward(s["plan"], s["grad"], s["kind"], case["B"], H, Lq, Lk, off, H * Lq * Lk, Lq * Lk, Lk, s["out"],
                                s["ws"], s["ws"].numel())
    return s["out"]


def _own_adamw(s, case):
    mb = s["mb"]
    s["step"] += 1
    mb.adamw_step(s["plan"], s["state"], LR, BETA1, BETA2, EPS, DECAY, s["step"], s["clip"], seed=s["step"])
    if case["bits"] == 8:
        mb.adamw_export_state(s["plan"], s["state"], s["m"], s["v"])
    return {"param": s["param"], "master": s["master"], "m": s["m"], "v": s["v"]}


def _doubling(a, u, longest):
    """h_t = a_t h_{t-1} + u_t along the first axis, for a that is 0 where a sequence begins: spans of twice the length in each pass."""
    step = 1
    while step < longest:
        u = torch.cat([u[:step], u[step:] + a[step:] * u[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return u


def _plain_recurrence(s, case):
    N, t, offsets = case["N"], TYPES[case["dtype"]], s["offsets"]
    x = s["value"].float()
    z = 1.0 / (1.0 + torch.exp(-s["gate"].float()))
    at = torch.arange(N, device=DEV)
    seq = torch.bucketize(at, offsets[1:], right=True)
    first = (at == offsets[seq]).unsqueeze(1)
    last = (at == offsets[seq + 1] - 1).unsqueeze(1)
    keep = 1.0 - z
    u = torch.where(first, z * x + keep * s["h0"][seq], z * x)
    h = _doubling(torch.where(first, 0.0, keep), u, s["longest"])
    ends = (offsets[1:] - 1).clamp(min=0)
    empty = (offsets[1:] == offsets[:-1]).unsqueeze(1)
    out = {"h": h.to(t), "final": torch.where(empty, s["h0"], h[ends])}
    if case["dir"] == "train":
        before = torch.where(first, s["h0"][seq], torch.cat([h[:1], h[:-1]]))
        d = s["grad"].float()
        d = torch.where(last, d + s["grad_final"][seq], d)
        after = torch.where(last, 0.0, torch.cat([keep[1:], keep[:1]]))
        G = _doubling(after.flip(0), d.flip(0), s["longest"]).flip(0)
        out["d_gate"] = (G * (x - before) * z * keep).to(t)
        out["d_value"] = (G * z).to(t)
        begins = offsets[:-1].clamp(max=N - 1)
        out["d_h0"] = torch.where(empty, s["grad_final"], (keep * G)[begins])
    return out


def _plain_bias(s, case):
    H, Lq, Lk, off = case["H"], case["Lq"], case["Lk"], case["off"]
    rows = case["n"] * (2 if case["two"] else 1)
    r = torch.arange(-(Lq - 1), Lk, device=DEV) - off            # every distance key - query there is
    d = r.abs() if case["two"] else (-r).clamp(min=0)
    bucket = torch.bucketize(d, s["starts"], right=True) - 1
    if case["two"]:
        bucket = torch.where(r > 0, bucket + case["n"], bucket)
    if case["dir"] == "fwd":
        line = s["table"].t()[:, bucket]
        if case["causal"]:
            line = torch.where(r > 0, -math.inf, line)
        line = line.to(TYPES[case["dtype"]])
        where = torch.arange(Lk, device=DEV) - torch.arange(Lq, device=DEV).unsqueeze(1) + (Lq - 1)
        return line[:, where]
    g = s["grad"].float().sum(0).flip(1)
    # with Lq columns of zeros behind each row, rows of one element less put each diagonal into a column
    g = torch.cat([g, g.new_zeros(H, Lq, Lq)], 2).view(H, -1)[:, :Lq * (Lk + Lq - 1)].view(H, Lq, Lk + Lq - 1).sum(1)
    if case["causal"]:
        g = torch.where(r > 0, 0.0, g)
    onehot = (bucket.unsqueeze(1) == torch.arange(rows, device=DEV)).float()
    return (g.unsqueeze(2) * onehot).sum(1).t().contiguous()


def _held_first(m):
    """What first moments held in 8 bits stand for: a sign and eight steps per octave under the block's largest, rounded to the nearest."""
    x = m.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    q = ((x.abs() * (1.0 / top)).view(torch.int32) + 0x80000 >> 20).clamp(max=0x3F8)
    near = torch.where(q > 0x379, q << 20, 0).view(torch.float32) * top
    return torch.where(top < 2.0 ** -120, 0.0, torch.where(x < 0, -near, near)).view(-1)


def _held_second(v, random16):
    """The same for second moments: no sign, 255 steps, rounded up or down by 16 random bits for each (None: to the nearest)."""
    x = v.view(-1, BLOCK)
    top = x.amax(1, keepdim=True)
    add = 0x80000 if random16 is None else (random16 << 4).view(-1, BLOCK)
    q = ((x * (1.0 / top)).view(torch.int32) + add >> 20).clamp(min=0x2FA, max=0x3F8)
    near = torch.where(x > 0, (q << 20).view(torch.float32) * top, 0.0)
    return torch.where(top < 2.0 ** -120, 0.0, near).view(-1)


def _mixed(P, seed):
    """16 random bits for each element and seed: two rounds of multiply and shift on 32-bit words."""
    w = torch.arange(P, device=DEV) * 0x9E3779B1 + seed * 0x85EBCA77 & 0xFFFFFFFF
    w = (w ^ w >> 15) * 0x2C1B3C6D & 0xFFFFFFFF
    w = (w ^ w >> 12) * 0x297A2D39 & 0xFFFFFFFF
    return (w >> 16).to(torch.int32)


def _plain_adamw(s, case):
    s["step"] += 1
    step = s["step"]
    g = s["grad"].float() * s["clip"]
    m = s["m"] * BETA1 + g * (1.0 - BETA1)
    v = s["v"] * BETA2 + (g * g) * (1.0 - BETA2)
    root = torch.sqrt(v) / math.sqrt(1.0 - BETA2 ** step) + EPS
    p = (s["master"] if case["master"] else s["param"]).float().view(-1, BLOCK)
    p = p - p * (s["decays"] * (LR * DECAY))
    p = p.view(-1) - m / root * (LR / (1.0 - BETA1 ** step))
    if case["master"]:
        s["master"].copy_(p)
    s["param"].copy_(p)
    if case["bits"] == 8:
        m, v = _held_first(m), _held_second(v, _mixed(len(v), step))
    s["m"], s["v"] = m, v
    return {"param": s["param"], "master": s["master"], "m": m, "v": v}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    return {"recurrence": _exact_recurrence, "bias": _exact_bias, "adamw": _exact_adamw}[case["op"]](case, prepare(case, seed))


def _exact_recurrence(case, s):
    N, D, S = case["N"], case["D"], case["S"]
    if N * D > 150_000_000 or s["longest"] > 600_000:
        return None
    f64 = lambda x: x.double().cpu().numpy()  # noqa: E731
    x, h0, start = f64(s["value"]), f64(s["h0"]), s["offsets"].cpu().numpy()
    n = start[1:] - start[:-1]
    order = np.argsort(-n, kind="stable")                        # longest first: those still running are the first k
    z = 1.0 / (1.0 + np.exp(-f64(s["gate"])))
    count = np.searchsorted(-n[order], -np.arange(s["longest"]), side="left")    # sequences longer than t
    h, state = np.empty((N, D)), h0[order].copy()
    begin = start[:-1][order]
    for t in range(s["longest"]):
        k = count[t]
        at = begin[:k] + t if k > 1 else slice(begin[0] + t, begin[0] + t + 1)
        state[:k] += z[at] * (x[at] - state[:k])
        h[at] = state[:k]
    final = np.empty((S, D))
    final[order] = state
    out = {"h": h, "final": final}
    if case["dir"] == "train":
        d = f64(s["grad"])
        G = f64(s["grad_final"])[order]                          # what arrives from the right, times 1 - z of the token there
        d_gate, d_value = np.empty((N, D)), np.empty((N, D))
        for t in range(s["longest"] - 1, -1, -1):
            k = count[t]
            at = begin[:k] + t if k > 1 else slice(begin[0] + t, begin[0] + t + 1)
            before = h0[order[:k]] if t == 0 else h[begin[:k] + t - 1]
            total = d[at] + G[:k]
            zt = z[at]
            d_value[at] = total * zt
            d_gate[at] = total * (x[at] - before) * zt * (1.0 - zt)
            G[:k] = total * (1.0 - zt)
        d_h0 = np.empty((S, D))
        d_h0[order] = G
        out.update(d_gate=d_gate, d_value=d_value, d_h0=d_h0)
    return out


def _exact_bias(case, s):
    H, Lq, Lk, off, n = case["H"], case["Lq"], case["Lk"], case["off"], case["n"]
    rows = n * (2 if case["two"] else 1)
    starts = starts_of(case)

    def bucket(r):
        d = abs(r) if case["two"] else max(-r, 0)
        return max(k for k in range(n) if starts[k] <= d) + (n if case["two"] and r > 0 else 0)

    of = {r: bucket(r) for r in range(-off - Lq + 1, Lk - off)}
    if case["dir"] == "fwd":
        table = s["table"].double().cpu().numpy()
        line = np.stack([np.full(H, -np.inf) if case["causal"] and r > 0 else table[of[r]] for r in sorted(of)], 1)
        out = np.empty((H, Lq, Lk))
        for i in range(Lq):
            out[:, i] = line[:, Lq - 1 - i:Lq - 1 - i + Lk]
        return out
    out = torch.zeros(rows, H, dtype=torch.float64, device=DEV)
    g = torch.zeros(H, Lq, Lk, dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        g += s["grad"][b].double()
    for r in of:
        if not (case["causal"] and r > 0):
            out[of[r]] += torch.diagonal(g, r + off, 1, 2).sum(1)
    return out


def _exact_adamw(case, s):
    # the moments that prepare() starts from, in 8 bits as they are held there
    step = s["step"] + 1
    g = s["grad"].double() * s["clip"].double()
    m, v = s["m"].double(), s["v"].double()
    m = m + (g - m) * (1.0 - BETA1)
    v = v + (g.square() - v) * (1.0 - BETA2)
    hat_m, hat_v = m / (1.0 - BETA1 ** step), v / (1.0 - BETA2 ** step)
    p = (s["master"] if case["master"] else s["param"]).double()
    decay = s["decays"].double().expand(-1, BLOCK).reshape(-1)
    p = p * (1.0 - LR * DECAY * decay) - LR * hat_m / (hat_v.sqrt() + EPS)
    if case["bits"] == 8:
        m, v = _nearest_in_64(m), _random_in_64(v, step)
    return {"param": p, "master": p if case["master"] else None, "m": m, "v": v}


def _steps(x, add):
    """x in (0, 1], down to three binary places behind the leading one after `add` (in units of the step) is put on top."""
    f, e = torch.frexp(x)                                        # x = f 2^e, f in [1/2, 1): steps of 1/16 there
    return torch.ldexp(torch.floor(f * 16.0 + add) / 16.0, e)


def _nearest_in_64(m):
    x = m.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    q = _steps((x / top).abs(), 0.5)
    q = torch.where(q < 1.25 * 2.0 ** -16, 0.0, q)               # the smallest of 127 steps below 1
    return torch.where(top < 2.0 ** -120, 0.0, q * top * x.sign()).view(-1)


def _random_in_64(v, seed):
    x = v.view(-1, BLOCK)
    top = x.amax(1, keepdim=True)
    w = np.arange(v.numel(), dtype=np.uint32) * np.uint32(0x9E3779B1) + np.uint32(seed * 0x85EBCA77 & 0xFFFFFFFF)
    w = (w ^ (w >> np.uint32(15))) * np.uint32(0x2C1B3C6D)
    w = (w ^ (w >> np.uint32(12))) * np.uint32(0x297A2D39)
    add = torch.from_numpy((w >> np.uint32(16)).astype(np.float64) / 65536.0).to(DEV).view(-1, BLOCK)
    q = _steps(x / top, add).clamp(min=1.25 * 2.0 ** -32)
    return torch.where(top < 2.0 ** -120, 0.0, torch.where(x > 0, q * top, 0.0)).view(-1)
