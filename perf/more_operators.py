"""The operators at the head of the sequence tower, as cases to measure: the root-mean-square norm of the residual stream (with an output
in 8 bits), the log probabilities of given items with entropy and best alternatives, and the loss that trains a tower by a teacher's best
items.  `run` computes a case with the library (`own` true) or in plain torch operations."""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-6
LEAST = 2.0 ** -100                           # least maximum of a group of 8-bit values
TOP8 = 448.0                                  # largest number of the 8-bit type


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # serving: one new event for each of 192 users, between two layers
        dict(name="norm_step", op="norm", dir="fwd", N=192, D=128, residual=True, dtype="bf16", weight="fp32", pad=0, group=-1),
        # the packed events of 1,000 histories, handed to a product in 8 bits with a scale for each event
        dict(name="norm_8bit_rows", op="norm", dir="fwd", N=120007, D=256, residual=True, dtype="bf16", weight="bf16", pad=0, group=0),
        # a wide layer, 8 bits with a scale for every 128 columns
        dict(name="norm_8bit_wide", op="norm", dir="fwd", N=8192, D=8192, residual=True, dtype="bf16", weight="fp32", pad=0, group=128),
        # training of a layer, forward and backward, the stream's own gradient included
        dict(name="norm_train", op="norm", dir="train", N=131072, D=1024, residual=True, dtype="bf16", weight="fp32", pad=0, group=-1),
        # a narrow tower in single precision with a width that is on no vector boundary, and no residual: the first norm
        dict(name="norm_train_odd", op="norm", dir="train", N=100003, D=333, residual=False, dtype="fp32", weight="fp32", pad=0, group=-1),
        # serving: scores of one user's next item over a catalogue, and what to show instead
        dict(name="logp_step", op="logp", dir="fwd", N=1, V=100000, k=20, scale=1.0, mask=0.01, dtype="bf16", pad=0),
        # scoring a small catalogue for many users, some items ruled out for each
        dict(name="logp_fwd_small", op="logp", dir="fwd", N=30011, V=5001, k=10, scale=1.25, mask=0.1, dtype="fp32", pad=0),
        # evaluation over a large catalogue
        dict(name="logp_fwd_large", op="logp", dir="fwd", N=2048, V=131072, k=16, scale=1.0, mask=0.0, dtype="bf16", pad=0),
        # the gradient of log probability and entropy, rows padded to whole vectors
        dict(name="logp_bwd", op="logp", dir="bwd", N=4099, V=50001, k=0, scale=0.8, mask=0.05, dtype="bf16", pad=7),
        # validation of a small tower against its teacher: the loss alone
        dict(name="distill_loss", op="distill", dir="fwd", N=64, V=20000, K=32, rest=False, scale=1.0, dtype="fp32", pad=0),
        # training against a teacher that tells how much the other items weigh; odd catalogue
        dict(name="distill_train_rest", op="distill", dir="train", N=2047, V=32003, K=64, rest=True, scale=0.5, dtype="fp16", pad=0),
        # training over a large catalogue
        dict(name="distill_train_large", op="distill", dir="train", N=4096, V=65536, K=50, rest=False, scale=1.0, dtype="bf16", pad=0),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(("norm", "logp", "distill"))
    dtype, pad = rng.choice(tuple(TYPES)), rng.choice((0, 0, rng.randint(1, 16)))
    if op == "norm":
        D = rng.choice((_log(rng, 16, 16384), 8 * _log(rng, 2, 2048)))
        direction = rng.choice(("fwd", "fwd", "train"))
        group = -1
        if direction == "fwd" and dtype != "fp32":
            group = rng.choice((-1, 0, 32, 64, 128, 256))
        return dict(op=op, dir=direction, N=_log(rng, 1, 100000000 // D), D=D, residual=rng.random() < 0.7, dtype=dtype,
                    weight=rng.choice((dtype, "fp32")), pad=pad, group=group)
    V = rng.choice((_log(rng, 100, 262144), 8 * _log(rng, 12, 32768)))
    N = _log(rng, 1, min(200000000 // V, 100000))
    if op == "logp":
        direction = rng.choice(("fwd", "bwd"))
        return dict(op=op, dir=direction, N=N, V=V, k=rng.choice((0, 1, rng.randint(2, 32))) if direction == "fwd" else 0,
                    scale=rng.choice((1.0, 0.7, 1.4)), mask=rng.choice((0.0, 0.02, 0.5)), dtype=dtype, pad=pad)
    return dict(op=op, dir=rng.choice(("fwd", "train", "train")), N=N, V=V, K=min(_log(rng, 4, 128), V // 2), rest=rng.random() < 0.5,
                scale=rng.choice((1.0, 0.5, 0.25)), dtype=dtype, pad=pad)


def work(case):
    N, e = case["N"], SIZE[case["dtype"]]
    if case["op"] == "norm":
        D, n, w = case["D"], N * case["D"], SIZE[case["weight"]] * case["D"]
        stream = n * e * (3 if case["residual"] else 1)                   # x alone, or x, residual and their sum
        if case["group"] < 0:
            b = stream + n * e + w
        else:                                                             # codes, scales, and the values that they stand for
            b = stream + n + 4 * N * (-(-D // case["group"]) if case["group"] else 1) + n * e + w
        if case["dir"] == "train":                                        # gradients of y and of the stream, gradient of x; of the weight
            b += n * e * (3 if case["residual"] else 2) + 4 * D
        return {"bytes": b, "flops": (6 if case["dir"] == "fwd" else 18) * n}
    n = N * case["V"]
    if case["op"] == "logp":
        if case["dir"] == "fwd":
            return {"bytes": n * e + N * (8 + 4 + 4 + 12 * case["k"]), "flops": 6 * n}
        return {"bytes": 2 * n * e + N * 28, "flops": 8 * n}
    b = n * e + N * (case["K"] * (8 + e) + 4 + 4 + (4 if case["rest"] else 0))
    return {"bytes": b + (n * e if case["dir"] == "train" else 0), "flops": (4 if case["dir"] == "fwd" else 8) * n}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case)
    if own:
        from paper_2305_01515_b200 import binding as mb

        kinds = {"fp32": mb.DTYPE_FP32, "fp16": mb.DTYPE_FP16, "bf16": mb.DTYPE_BF16}
        s["mb"], s["kind"] = mb, kinds[case["dtype"]]
        s["weight_kind"] = kinds[case.get("weight", case["dtype"])]
    {"norm": _prepare_norm, "logp": _prepare_logp, "distill": _prepare_distill}[case["op"]](s, case, g)
    return s


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _padded(x, case):
    """x in the case's type, its rows `pad` elements further apart than they are long."""
    room = torch.zeros(x.shape[0], x.shape[1] + case["pad"], dtype=TYPES[case["dtype"]], device=DEV)
    room[:, :x.shape[1]] = x
    return room[:, :x.shape[1]]


def _prepare_norm(s, case, g):
    N, D, t = case["N"], case["D"], TYPES[case["dtype"]]
    # a stream whose channels have sizes of their own, and what a layer adds to it
    size = torch.exp(0.5 * _randn(g, D))
    s["x"] = _padded(_randn(g, N, D) * 0.3, case)
    s["residual"] = _padded(_randn(g, N, D) * size, case) if case["residual"] else None
    if not case["residual"]:
        s["x"] = _padded(s["x"].float() * size * 3.0, case)
    s["weight"] = (1.0 + 0.1 * _randn(g, D)).to(TYPES[case["weight"]])
    train = case["dir"] == "train"
    if train:
        s["grad"] = _padded(_randn(g, N, D) * 1e-2, case)
        s["grad_sum"] = _padded(_randn(g, N, D) * 1e-2, case) if case["residual"] else None
    if own:
        s["stride"] = D + case["pad"]
        s["sum"] = torch.empty(N, D, dtype=t, device=DEV) if case["residual"] else None
        s["inv"] = torch.empty(N, device=DEV) if train else None
        s["out"] = torch.empty(N, D, dtype=t, device=DEV)
        if case["group"] >= 0:
            s["codes"] = torch.empty(N, D, dtype=torch.uint8, device=DEV)
            s["scales"] = torch.empty(N, -(-D // case["group"]) if case["group"] else 1, device=DEV)
        if train:
            s["dx"], s["dw"] = torch.empty(N, D, dtype=t, device=DEV), torch.empty(D, device=DEV)
            s["ws"] = torch.empty(s["mb"].rms_norm_workspace_bytes(N, D), dtype=torch.uint8, device=DEV)


def _share(case):
    """What a row's loss counts in the batch's mean; in fp16 times a loss scale, without which small gradients are lost."""
    return 1.0 / case["N"] if case["dtype"] != "fp16" else min(65536.0 / case["N"], 16384.0)


def _scores(g, case):
    """Scores over a catalogue: some items are liked by all, and each user has a taste."""
    N, V = case["N"], case["V"]
    liked = 1.5 * _randn(g, V)
    x = _randn(g, N, V) * (1.0 + 0.5 * torch.rand(N, 1, generator=g, device=DEV))
    return x.add_(liked)


def _prepare_logp(s, case, g):
    N, V, k = case["N"], case["V"], case["k"]
    x = _scores(g, case)
    if case["mask"]:                          # items that a user has seen are ruled out
        x.masked_fill_(torch.rand(N, V, generator=g, device=DEV) < case["mask"], -math.inf)
    s["target"] = torch.randint(V, (N,), generator=g, device=DEV)
    if case["dir"] == "bwd":                  # events that came were possible
        x[torch.arange(N, device=DEV), s["target"]] = 1.0
    if N > 4:                                 # padding of a batch: no event
        s["target"][torch.rand(N, generator=g, device=DEV) < 0.03] = -1
    s["x"] = _padded(x, case)
    if case["dir"] == "bwd":
        s["g_logp"] = -torch.rand(N, generator=g, device=DEV) * _share(case)
        s["g_entropy"] = 0.01 * _randn(g, N) * _share(case)
        del x
        # what the forward pass kept: the largest score, the logarithm of the sum relative to it, the entropy
        z = s["x"].double()
        top = z.amax(1, keepdim=True)
        z = (z - top) * case["scale"]
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        log = torch.log(total)
        s["entropy"] = (log - (torch.where(e > 0, e * z, 0.0)).sum(1, keepdim=True) / total)[:, 0].float()
        s["stats"] = torch.cat([top, log], 1).float()
    if own:
        s["stride"] = V + case["pad"]
        if case["dir"] == "fwd":
            s["logp"], s["ent"] = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
            s["top_index"] = torch.empty(N, k, dtype=torch.int64, device=DEV) if k else None
            s["top_logp"] = torch.empty(N, k, device=DEV) if k else None
        else:
            s["dx"] = torch.empty(N, V + case["pad"], dtype=TYPES[case["dtype"]], device=DEV)[:, :V]


def _prepare_distill(s, case, g):
    N, V, K, t = case["N"], case["V"], case["K"], TYPES[case["dtype"]]
    x = _scores(g, case)
    # the teacher's best items, in the order of its scores, all different: one out of each K-th of the catalogue
    part = torch.arange(K + 1, device=DEV) * V // K
    at = part[:-1] + (torch.rand(N, K, generator=g, device=DEV) * (part[1:] - part[:-1])).long().clamp(max=part[1:] - part[:-1] - 1)
    s["index"] = at.gather(1, torch.rand(N, K, generator=g, device=DEV).argsort(1))
    likes = 8.0 + 3.0 * _randn(g, N, K).sort(1, descending=True)[0]
    s["teacher"] = likes.to(t)
    x.scatter_add_(1, s["index"], 0.5 * likes)                            # the student has learned some of it
    # what the teacher gives to all other items together: from a tenth to about half
    s["rest"] = torch.logsumexp(s["teacher"].float() * case["scale"], 1) - 1.0 + 0.7 * _randn(g, N) if case["rest"] else None
    s["w"] = torch.rand(N, generator=g, device=DEV) * _share(case)
    s["x"] = _padded(x, case)
    if own:
        s["stride"] = V + case["pad"]
        s["loss"] = torch.empty(N, device=DEV)
        s["dx"] = torch.empty(N, V, dtype=t, device=DEV) if case["dir"] == "train" else None


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "logp": _own_logp, "distill": _own_distill}[op](s, s["case"])
    return {"norm": _plain_norm, "logp": _plain_logp, "distill": _plain_distill}[op](s, s["case"])


def _own_norm(s, case):
    mb, N, D, k, w, at = s["mb"], case["N"], case["D"], s["kind"], s["weight_kind"], s["stride"]
    if case["group"] >= 0:
        mb.rms_norm_forward_8bit(s["x"], at, s["residual"], at, s["weight"], w, k, N, D, EPS, s["sum"], D, s["codes"], D, s["scales"],
                                 case["group"], None)
        mb.rows_from_8bit(s["codes"], D, s["scales"], case["group"], N, D, s["out"], k, D)
        return {"sum": s["sum"], "scales": s["scales"], "values": s["out"]}
    mb.rms_norm_forward(s["x"], at, s["residual"], at, s["weight"], w, k, N, D, EPS, s["sum"], D, s["out"], D, s["inv"])
    if case["dir"] == "fwd":
        return {"sum": s["sum"], "out": s["out"]}
    r, r_at = (s["sum"], D) if case["residual"] else (s["x"], at)
    mb.rms_norm_backward(r, r_at, s["weight"], w, k, N, D, s["inv"], s["grad"], at, s["grad_sum"], at, s["dx"], D, s["dw"], s["ws"],
                         s["ws"].numel())
    return {"sum": s["sum"], "out": s["out"], "dx": s["dx"], "dw": s["dw"]}


def _own_logp(s, case):
    mb, N, V, k = s["mb"], case["N"], case["V"], case["k"]
    if case["dir"] == "bwd":
        mb.logprobs_backward(s["x"], s["stride"], s["kind"], N, V, case["scale"], s["target"], s["stats"], s["entropy"], s["g_logp"],
                             s["g_entropy"], s["dx"], s["stride"])
        return s["dx"]
    mb.logprobs_forward(s["x"], s["stride"], s["kind"], N, V, case["scale"], s["target"], k, s["logp"], s["ent"], None, s["top_index"],
                        s["top_logp"])
    return {"logp": s["logp"], "entropy": s["ent"], "top_index": s["top_index"], "top_logp": s["top_logp"]}


def _own_distill(s, case):
    s["mb"].distill_loss(s["x"], s["stride"], s["kind"], case["N"], case["V"], case["scale"], s["index"], s["teacher"], s["kind"], case["K"],
                         s["rest"], s["w"], s["loss"], s["dx"], case["V"])
    return {"loss": s["loss"], "dx": s["dx"]}


def _plain_norm(s, case):
    D, t, group = case["D"], TYPES[case["dtype"]], case["group"]
    total = None
    r = s["x"].float()
    if case["residual"]:
        total = (r + s["residual"].float()).to(t)
        r = total.float()                                                 # what is normalised is the stream as it is stored
    c = 1.0 / torch.sqrt((r * r).sum(1, keepdim=True) / D + EPS)
    w = s["weight"].float()
    y = r * c * w
    if group >= 0:
        n = group or D
        if D % n:
            y = torch.cat([y, y.new_zeros(len(y), n - D % n)], 1)
        y = y.view(len(y), -1, n)
        top = y.abs().amax(2, keepdim=True).clamp(min=LEAST)
        scale = top / TOP8
        code = (y * (TOP8 / top)).to(torch.float8_e4m3fn)
        values = (code.float() * scale).view(len(y), -1)[:, :D].to(t)
        return {"sum": total, "scales": scale[:, :, 0], "values": values}
    if case["dir"] == "fwd":
        return {"sum": total, "out": y.to(t)}
    dy = s["grad"].float()
    a = dy * w
    dx = c * (a - r * ((a * r).sum(1, keepdim=True) / D * (c * c)))
    if case["residual"]:
        dx = dx + s["grad_sum"].float()
    return {"sum": total, "out": y.to(t), "dx": dx.to(t), "dw": (dy * r * c).sum(0)}


def _softmax(x, scale):
    """(scores relative to the largest, times scale; their exponentials; the sum of these), where nothing is left of a row all 0."""
    top = x.amax(1, keepdim=True)
    z = (x - torch.where(top == -math.inf, 0.0, top)) * scale
    e = torch.exp(z)
    return z, e, e.sum(1, keepdim=True)


def _best(x, k):
    """The k largest of each row, the lowest index first among equals: distinct whole numbers that are ordered alike."""
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits)
    key = (key << 31) + (0x7FFFFFFF - torch.arange(x.shape[1], device=DEV))
    return 0x7FFFFFFF - (torch.topk(key, k, 1)[0] & 0x7FFFFFFF)


def _plain_logp(s, case):
    k, target = case["k"], s["target"]
    given = target >= 0
    at = target.clamp(min=0).unsqueeze(1)
    x = s["x"].float()
    if case["dir"] == "bwd":
        z = (x - s["stats"][:, :1]) * case["scale"]
        log = z - s["stats"][:, 1:]
        p = torch.exp(log)
        gl = torch.where(given, s["g_logp"], 0.0).unsqueeze(1)
        gh = s["g_entropy"].unsqueeze(1)
        d = -p * gl - torch.where(p > 0, gh * p * (log + s["entropy"].unsqueeze(1)), 0.0)
        d = d.scatter_add(1, at, gl)
        return (d * case["scale"]).to(TYPES[case["dtype"]])
    z, e, total = _softmax(x, case["scale"])
    log = torch.log(total)
    out = {"logp": torch.where(given, (z.gather(1, at) - log)[:, 0], 0.0)}
    out["entropy"] = (log - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / total)[:, 0]
    out["top_index"] = _best(x, k) if k else None
    out["top_logp"] = z.gather(1, out["top_index"]) - log if k else None
    return out


def _plain_distill(s, case):
    scale, index, rest = case["scale"], s["index"], s["rest"]
    x = s["x"].float()
    t = s["teacher"].float() * scale
    if rest is not None:
        t = torch.cat([t, rest.unsqueeze(1)], 1)
    zq, eq, total_q = _softmax(t, 1.0)
    q = eq / total_q
    log_q = zq - torch.log(total_q)
    z, e, total = _softmax(x, scale)
    log_p = z.gather(1, index) - torch.log(total)
    if rest is not None:
        others = torch.log(e.scatter(1, index, 0.0).sum(1, keepdim=True)) - torch.log(total)
        log_p = torch.cat([log_p, others], 1)
    out = {"loss": torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1), "dx": None}
    if case["dir"] == "train":
        p = e / total
        d = p if rest is None else p * (1.0 - q[:, -1:] / torch.exp(log_p[:, -1:]))
        d = d.scatter(1, index, p.gather(1, index) - q[:, :index.shape[1]])
        out["dx"] = (d * (s["w"].unsqueeze(1) * scale)).to(TYPES[case["dtype"]])
    return out


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    rows = max(1, 40_000_000 // case["D" if case["op"] == "norm" else "V"])
    parts = []
    for a in range(0, case["N"], rows):                                   # some rows at a time: 64 bits take room
        cut = lambda k: None if s.get(k) is None else s[k][a:a + rows].double()  # noqa: E731
        parts.append({"norm": _exact_norm, "logp": _exact_logp, "distill": _exact_distill}[case["op"]](case, s, cut, slice(a, a + rows)))
    if not isinstance(parts[0], dict):
        return torch.cat(parts)
    out = {}
    for key in parts[0]:
        some = [p[key] for p in parts]
        out[key] = None if some[0] is None else torch.stack(some).sum(0) if key == "dw" else torch.cat(some)
    return out


def _nearest8(v):
    """The numbers of the 8-bit type (four significant bits, steps of 2^-9 below 2^-6) nearest to v, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(v / step) * step).clamp(-TOP8, TOP8)


def _exact_norm(case, s, cut, rows):
    D, group, t = case["D"], case["group"], TYPES[case["dtype"]]
    r, total, w = cut("x"), None, s["weight"].double()
    if case["residual"]:
        total = r + cut("residual")
        r = total.to(t).double()                                          # by definition the sum is rounded once, then normalised
    ms = r.square().mean(1, keepdim=True) + EPS
    y = r * w / ms.sqrt()
    if group >= 0:
        n = group or D
        scales, values = [], []
        for a in range(0, D, n):
            part = y[:, a:a + n]
            scales.append(part.abs().amax(1, keepdim=True).clamp(min=LEAST) / TOP8)
            values.append(_nearest8(part / scales[-1]) * scales[-1])
        return {"sum": total, "scales": torch.cat(scales, 1), "values": torch.cat(values, 1)}
    if case["dir"] == "fwd":
        return {"sum": total, "out": y}
    unit, dy = r / ms.sqrt(), cut("grad")
    d_unit = dy * w
    dx = (d_unit - unit * (d_unit * unit).mean(1, keepdim=True)) / ms.sqrt()
    if case["residual"]:
        dx = dx + cut("grad_sum")
    return {"sum": total, "out": y, "dx": dx, "dw": (dy * unit).sum(0)}


def _exact_logp(case, s, cut, rows):
    x, target = cut("x"), s["target"][rows]
    V, scale, k = case["V"], case["scale"], case["k"]
    lse = torch.logsumexp(x * scale, 1, keepdim=True)
    log = x * scale - lse
    plogp = torch.special.entr(log.exp())                                 # -p log p, 0 where p is
    entropy = plogp.sum(1)
    if case["dir"] == "bwd":
        p = log.exp()
        one = (torch.arange(V, device=DEV) == target.unsqueeze(1)).double()
        gl = cut("g_logp") * (target >= 0)
        d = gl.unsqueeze(1) * (one - p) + cut("g_entropy").unsqueeze(1) * (plogp - p * entropy.unsqueeze(1))
        return d * scale
    at = torch.arange(len(x), device=DEV)
    out = {"logp": torch.where(target >= 0, log[at, target], 0.0), "entropy": entropy, "top_index": None, "top_logp": None}
    if k:
        out["top_index"] = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
        out["top_logp"] = log.gather(1, out["top_index"])
    return out


def _exact_distill(case, s, cut, rows):
    scale, index = case["scale"], s["index"][rows]
    x, t = cut("x"), cut("teacher") * scale
    listed_ = torch.zeros(x.shape, dtype=torch.bool, device=DEV).scatter_(1, index, True)
    log = torch.log_softmax(x * scale, 1)
    if case["rest"]:
        rest = cut("rest").unsqueeze(1)
        lse = torch.logaddexp(torch.logsumexp(t, 1, keepdim=True), rest)
        log_r, log_pr = rest - lse, torch.logsumexp(log.masked_fill(listed_, -math.inf), 1, keepdim=True)
    else:
        lse = torch.logsumexp(t, 1, keepdim=True)
    log_q = t - lse
    loss = (log_q.exp() * (log_q - log.gather(1, index))).sum(1)
    if case["rest"]:
        loss = loss + (log_r.exp() * (log_r - log_pr))[:, 0]
    if case["dir"] == "fwd":
        return {"loss": loss, "dx": None}
    p = log.exp()
    want = torch.zeros_like(x).scatter_(1, index, log_q.exp())            # the distribution that the student is drawn to
    if case["rest"]:
        want = torch.where(listed_, want, p * (log_r - log_pr).exp())
    return {"loss": loss, "dx": (p - want) * (cut("w").unsqueeze(1) * scale)}
