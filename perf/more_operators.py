"""Timed cases of dropout, layer norm and the log probabilities of given tokens:
the calls a trainer or a server makes of the library (``own`` true), and the
same results from elementary torch operations (``own`` false).

- ``dropout``: out = add + x kept / (1 - p), the mask a function of the seed and
  a value's place, stored nowhere. Its gradient is the same call on dout.
- ``norm``: h = add + dropout(x), y = (h - mean) / sqrt(var + eps) * w + b of
  every row; with neither add nor p, h is x.
- ``norm_grad``: the gradients of x, of h's other summand, and of w and b.
- ``logp``: each row's log probability of its target, entropy, largest logit
  (``peak``), log of the sum of exp(scale (logit - peak)), and likeliest words.
- ``logp_grad``: the gradient of the log probability and of the entropy.

Random words. Row i, column j of x with D columns belongs to word number
i * ceil(D / 2) + j // 2, its low half where j is even, its high half where j is
odd. The value is kept where that half is at least round(65536 p), and divided
by the share that is kept, 1 - round(65536 p) / 65536.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
IGNORE = -100
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # Between two recurrent layers: a batch of 20 sequences of 35 words, half of 650 cells dropped.
        {"name": "drop_hidden_650", "op": "dropout", "rows": 700, "D": 650, "dtype": "f32",
         "p": 0.5, "add": False},
        # Behind a large batch's projections, added to the residual stream.
        {"name": "drop_residual_2048", "op": "dropout", "rows": 65536, "D": 2048, "dtype": "bf16",
         "p": 0.1, "add": True},
        # One new token: the norm behind a sublayer, latency is all there is.
        {"name": "norm_token_2048", "op": "norm", "rows": 1, "D": 2048, "dtype": "bf16", "p": 0.0,
         "add": True},
        # Rows of odd length, in fp32, that no 16-byte vector divides.
        {"name": "norm_odd_517", "op": "norm", "rows": 4099, "D": 517, "dtype": "f32", "p": 0.0,
         "add": False},
        # A large training batch: dropout, residual sum and norm in one pass.
        {"name": "norm_residual_2048", "op": "norm", "rows": 65536, "D": 2048, "dtype": "bf16",
         "p": 0.1, "add": True},
        # A recurrent highway's 1792 cells: 128 sequences, 10 steps of the recurrence.
        {"name": "norm_grad_1792", "op": "norm_grad", "rows": 1280, "D": 1792, "dtype": "f32",
         "p": 0.0, "add": False},
        # The gradient of the large batch, with the gradient that comes along the residual stream.
        {"name": "norm_grad_2048", "op": "norm_grad", "rows": 65536, "D": 2048, "dtype": "bf16",
         "p": 0.1, "add": True},
        # One new token of a 100K vocabulary: its 20 likeliest words at a temperature of 0.7.
        {"name": "logp_token_100k", "op": "logp", "N": 1, "V": 100_000, "dtype": "bf16",
         "scale": 1 / 0.7, "top": 20, "masked": 0.0, "pad": 0},
        # A served batch over 800K words, a third of them not allowed.
        {"name": "logp_batch_800k", "op": "logp", "N": 64, "V": 800_000, "dtype": "bf16",
         "scale": 1.0, "top": 8, "masked": 0.33, "pad": 0},
        # The loss of a training batch, some of its places without a target.
        {"name": "logp_train_100k", "op": "logp", "N": 8192, "V": 100_000, "dtype": "bf16",
         "scale": 1.0, "top": 0, "masked": 0.0, "pad": 0},
        # The full softmax over 20K characters, 31 columns of padding, an odd row length.
        {"name": "logp_grad_char", "op": "logp_grad", "N": 2560, "V": 20_001, "dtype": "f32",
         "scale": 1.0, "masked": 0.0, "pad": 31, "entropy": True},
        # The gradient of the training batch.
        {"name": "logp_grad_100k", "op": "logp_grad", "N": 8192, "V": 100_000, "dtype": "bf16",
         "scale": 1.0, "masked": 0.0, "pad": 0, "entropy": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("dropout", "norm", "norm_grad", "logp", "logp_grad"))
    dtype = rng.choice(("f32", "bf16"))
    if op in ("dropout", "norm", "norm_grad"):
        D = _log(rng, 17, 8192)
        if rng.random() < 0.3:
            D = -(-D // 64) * 64
        rows = _log(rng, 1, min(65536, 120_000_000 // D))
        return {"op": op, "rows": rows, "D": D, "dtype": dtype,
                "p": rng.choice((0.1, 0.25, 0.5)) if op == "dropout" else
                rng.choice((0.0, 0.1, 0.3)), "add": rng.random() < 0.5}
    V = _log(rng, 100, 800_000)
    N = _log(rng, 1, max(1, min(8192, (300_000_000 if dtype == "f32" else 700_000_000) // V)))
    case = {"op": op, "N": N, "V": V, "dtype": dtype, "scale": rng.choice((1.0, 1 / 0.7, 0.5)),
            "masked": rng.choice((0.0, 0.0, 0.33)), "pad": rng.choice((0, 0, 7, 31))}
    if op == "logp":
        case["top"] = rng.choice((0, 1, 5, 20))
        if case["top"] and N * V > 100_000_000:
            case["N"] = max(1, 100_000_000 // V)
    else:
        case["entropy"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _randn(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEV).mul_(std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case, "op": case["op"], "seed": 1_000_003 * seed + 17}
    dt = TYPES[case["dtype"]]
    if case["op"] in ("logp", "logp_grad"):
        _prepare_logp(s, case, gen, dt)
        return s
    rows, D = case["rows"], case["D"]
    if case["op"] == "dropout":
        s["x"] = _randn(gen, rows, D, dtype=dt)
        s["add"] = _randn(gen, rows, D, std=2.0, dtype=dt) if case["add"] else None
        return s
    # Scales near 1 and small shifts, as training leaves them.
    s["w"] = _randn(gen, D, std=0.2) + 1
    s["b"] = _randn(gen, D, std=0.1)
    # A residual stream: rows of different sizes, off zero.
    size = torch.exp(_randn(gen, rows, 1, std=0.4))
    if case["op"] == "norm":
        s["x"] = (_randn(gen, rows, D) * size + 0.1).to(dt)
        s["add"] = _randn(gen, rows, D, std=2.0, dtype=dt) if case["add"] else None
        return s
    s["h"] = (_randn(gen, rows, D) * size + 0.1).to(dt)
    s["dy"] = _randn(gen, rows, D, std=1e-2, dtype=dt)
    s["add"] = _randn(gen, rows, D, std=1e-2, dtype=dt) if case["add"] else None
    wide = s["h"].double()
    mean = wide.mean(1)
    s["mean"] = mean.float()
    s["rstd"] = (wide.var(1, correction=0) + EPS).rsqrt().float()
    return s


def _prepare_logp(s, case, gen, dt):
    N, V = case["N"], case["V"]
    # Frequent words have the low ids and the larger logits.
    lean = -0.4 * torch.log1p(torch.arange(V, device=DEV, dtype=torch.float32))
    z = torch.empty(N, V, dtype=dt, device=DEV)
    for i in range(0, N, 1024):
        z[i:i + 1024] = _randn(gen, min(1024, N - i), V, std=2.0).add_(lean).to(dt)
    if case["masked"]:
        z[:, torch.rand(V, generator=gen, device=DEV) < case["masked"]] = -math.inf
    live = V - min(case["pad"], V // 2)
    z[:, live:] = -math.inf
    z[:, 0] = torch.where(torch.isinf(z[:, 0]), 0.0, z[:, 0].float()).to(dt)
    # Targets as Zipf's law draws them; one place in eight has none.
    u = torch.rand(N, generator=gen, device=DEV)
    t = (torch.exp(u * math.log(live + 1)) - 1).long().clamp_(0, live - 1)
    t = torch.where(torch.isinf(z[torch.arange(N, device=DEV), t]), 0, t)
    t[torch.arange(N, device=DEV) % 8 == 5] = IGNORE
    s.update(logits=z, targets=t)
    if case["op"] == "logp_grad":
        log_sum, ent = (torch.empty(N, device=DEV) for _ in range(2))
        for i in range(0, N, 256):
            y = z[i:i + 256].double()
            y = (y - y.amax(1, keepdim=True)) * _f32(case["scale"])
            a = torch.logsumexp(y, 1, keepdim=True)
            log_sum[i:i + 256] = a[:, 0]
            ent[i:i + 256] = -((y - a).exp() * (y - a).clamp(min=-1e30)).sum(1)
        s.update(peak=z.amax(1).float(), log_sum=log_sum, entropy=ent)
        s["dlogp"] = -torch.rand(N, generator=gen, device=DEV) / N
        s["dentropy"] = _randn(gen, N, std=0.1 / N) if case["entropy"] else None


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return {"dropout": _dropout, "norm": _norm, "norm_grad": _norm_grad, "logp": _logp,
            "logp_grad": _logp_grad}[s["op"]](s)


def _f32(x):
    """What the fp32 argument of a call holds of x."""
    return float(torch.tensor(x, dtype=torch.float32))


M32 = 0xFFFFFFFF


def _keys(seed):
    """Two 32-bit words from the 64-bit seed."""
    z = (seed * 0x9E3779B97F4A7C15 + 0x632BE59BD9B4E019) & (2 ** 64 - 1)
    z = ((z ^ (z >> 29)) * 0xD6E8FEB86659FD93) & (2 ** 64 - 1)
    z ^= z >> 32
    return z & M32, z >> 32


def _words(e, seed):
    """The 32-bit word of each number in `e` (int64)."""
    k0, k1 = _keys(seed)
    h = (((e & M32) ^ k0) * 0x9E3779B1) & M32
    h = h ^ (h >> 15)
    h = ((h + k1 + (e >> 32) * 0x85EBCA77) & M32) * 0xC2B2AE3D & M32
    return h ^ (h >> 16)


def _kept(rows, D, p, seed):
    """Which values a dropout of p keeps, and what they are multiplied by."""
    T = round(65536 * p)
    pairs = -(-D // 2)
    w = _words(torch.arange(rows * pairs, device=DEV), seed).view(rows, pairs)
    halves = torch.stack((w & 0xFFFF, w >> 16), 2).view(rows, 2 * pairs)[:, :D]
    return halves >= T, 65536 / (65536 - T)


def _dropped(x, p, seed):
    """dropout(x) in 32 bits."""
    if not p:
        return x.float()
    keep, scale = _kept(*x.shape, p, seed)
    return torch.where(keep, x.float() * scale, 0.0)


def _dropout(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        return lz.dropout(s["x"], c["p"], s["seed"], add=s["add"])
    y = _dropped(s["x"], c["p"], s["seed"])
    return (y if s["add"] is None else s["add"].float() + y).to(s["x"].dtype)


def _norm(s):
    c = s["case"]
    changed = s["add"] is not None or c["p"] > 0
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        r = lz.layer_norm(s["x"], s["w"], s["b"], eps=EPS, add=s["add"], p=c["p"], seed=s["seed"])
        out = {"y": r.y, "mean": r.mean, "rstd": r.rstd}
        if changed:
            out["h"] = r.h
        return out
    h = _dropped(s["x"], c["p"], s["seed"])
    if s["add"] is not None:
        h = s["add"].float() + h
    mean = h.mean(1)
    d = h - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + EPS)
    out = {"y": (d * rstd[:, None] * s["w"] + s["b"]).to(s["x"].dtype), "mean": mean,
           "rstd": rstd}
    if changed:
        out["h"] = h.to(s["x"].dtype)
    return out


def _norm_grad(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        r = lz.layer_norm_grad(s["dy"], s["h"], s["mean"], s["rstd"], s["w"], add=s["add"],
                               p=c["p"], seed=s["seed"])
        out = {"dh": r.dh, "dweight": r.dweight, "dbias": r.dbias}
        if c["p"] > 0:
            out["dx"] = r.dx
        return out
    dy = s["dy"].float()
    n = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["w"]
    dh = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    if s["add"] is not None:
        dh = s["add"].float() + dh
    out = {"dh": dh.to(s["h"].dtype), "dweight": (dy * n).sum(0), "dbias": dy.sum(0)}
    if c["p"] > 0:
        out["dx"] = _dropped(dh, c["p"], s["seed"]).to(s["h"].dtype)
    return out


def _logp(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        r = lz.token_logprobs(s["logits"], s["targets"], scale=c["scale"], top=c["top"],
                              ignore=IGNORE)
        out = {"logp": r.logp, "entropy": r.entropy, "peak": r.peak, "log_sum": r.log_sum}
        if c["top"]:
            out.update(top_logp=r.top_logp, top_ids=r.top_ids)
        return out
    z = s["logits"].float()
    peak = z.amax(1)
    d = (z - peak[:, None]) * c["scale"]
    e = torch.exp(d)
    total = e.sum(1)
    logs = torch.log(total)
    entropy = logs - torch.where(e > 0, e * d, 0.0).sum(1) / total
    t = s["targets"]
    at = d[torch.arange(c["N"], device=DEV), t.clamp(min=0)] - logs
    out = {"logp": torch.where(t == IGNORE, 0.0, at), "entropy": entropy, "peak": peak,
           "log_sum": logs}
    if c["top"]:
        # One number orders the logits, equal ones by their ids.
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2 ** 32
        key += c["V"] - 1 - torch.arange(c["V"], device=DEV)
        ids = c["V"] - 1 - (key.topk(c["top"], 1).values & M32)
        out["top_logp"] = torch.gather(d, 1, ids) - logs[:, None]
        out["top_ids"] = ids.int()
    return out


def _logp_grad(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        return lz.token_logprobs_grad(s["logits"], s["targets"], s["peak"], s["log_sum"],
                                      dlogp=s["dlogp"], entropy=s["entropy"],
                                      dentropy=s["dentropy"], scale=c["scale"], ignore=IGNORE)
    t = s["targets"]
    l = (s["logits"].float() - s["peak"][:, None]) * c["scale"] - s["log_sum"][:, None]
    prob = torch.exp(l)
    dlogp = torch.where(t == IGNORE, 0.0, s["dlogp"])
    d = -dlogp[:, None] * prob
    if s["dentropy"] is not None:
        more = prob * (l.clamp(min=-1e30) + s["entropy"][:, None])
        d = d - s["dentropy"][:, None] * more
    row = torch.arange(c["N"], device=DEV)
    d[row, t.clamp(min=0)] += dlogp
    return (d * c["scale"]).to(s["logits"].dtype)


# ---------------------------------------------------------------------------
# What a pass has to move and compute
# ---------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("logp", "logp_grad"):
        N, V = case["N"], case["V"]
        if case["op"] == "logp":
            return {"bytes": N * V * size + N * (8 + 16 + 8 * case["top"]), "flops": 6 * N * V}
        return {"bytes": 2 * N * V * size + N * (8 + 4 + 8 + (8 if case["entropy"] else 0)),
                "flops": (8 if case["entropy"] else 5) * N * V}
    rows, D, add, p = (case[k] for k in ("rows", "D", "add", "p"))
    n = rows * D
    if case["op"] == "dropout":
        return {"bytes": n * size * (3 if add else 2), "flops": n * (2 if add else 1)}
    if case["op"] == "norm":
        return {"bytes": n * size * (2 + add + (add or p > 0)) + 8 * (D + rows), "flops": 8 * n}
    return {"bytes": n * size * (3 + add + (p > 0)) + 12 * D + 8 * rows, "flops": 14 * n}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, written apart from the plain forms
# ---------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"dropout": _exact_dropout, "norm": _exact_norm, "norm_grad": _exact_norm_grad,
            "logp": _exact_logp, "logp_grad": _exact_logp_grad}[case["op"]](s)


def _exact_word(number, seed):
    """The word of each number, in 32-bit arithmetic that wraps around."""
    def wrap(k):
        return k - 2 ** 32 if k >= 2 ** 31 else k

    def right(a, n):
        return (a >> n) & ((1 << (32 - n)) - 1)
    z = (seed * 0x9E3779B97F4A7C15 + 0x632BE59BD9B4E019) % 2 ** 64
    z = (z ^ (z // 2 ** 29)) * 0xD6E8FEB86659FD93 % 2 ** 64
    z ^= z // 2 ** 32
    high = (number // 2 ** 32).int()
    a = (number - high * 2 ** 32 - 2 ** 31).int().bitwise_xor(-2 ** 31)
    a = (a ^ wrap(z % 2 ** 32)) * wrap(0x9E3779B1)
    a = a ^ right(a, 15)
    a = (a + wrap(z // 2 ** 32) + high * wrap(0x85EBCA77)) * wrap(0xC2B2AE3D)
    return a ^ right(a, 16)


def _exact_dropped(x, p, seed):
    """What dropout makes of x, in 64 bits: row by row, the even and the odd columns."""
    x = x.double()
    least = round(65536 * p)
    if least == 0:
        return x
    out = torch.zeros_like(x)
    half = (x.shape[1] + 1) // 2
    step = max(1, 2 ** 25 // half)
    for i in range(0, x.shape[0], step):
        n = min(step, x.shape[0] - i)
        word = _exact_word(torch.arange(i * half, (i + n) * half, device=DEV), seed).view(n, half)
        for odd in (0, 1):
            part = x[i:i + n, odd::2]
            r = word.div(65536, rounding_mode="floor") + 65536 if odd else word
            r = r.remainder(65536)[:, :part.shape[1]]
            out[i:i + n, odd::2] = torch.where(r >= least, part / (1 - least / 65536), 0.0)
    return out


def _exact_dropout(s):
    y = _exact_dropped(s["x"], s["case"]["p"], s["seed"])
    return y if s["add"] is None else y.add_(s["add"])


def _exact_norm(s):
    h = _exact_dropped(s["x"], s["case"]["p"], s["seed"])
    if s["add"] is not None:
        h = h + s["add"]
    var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
    root = torch.sqrt(var + EPS)
    out = {"y": s["w"] * ((h - mean) / root) + s["b"], "mean": mean[:, 0], "rstd": 1 / root[:, 0]}
    if s["add"] is not None or s["case"]["p"] > 0:
        out["h"] = h
    return out


def _exact_norm_grad(s):
    dy, mean, rstd = s["dy"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None]
    unit = rstd * (s["h"] - mean)
    D = unit.shape[1]
    out = {"dweight": (unit * dy).sum(0), "dbias": dy.sum(0)}
    g = dy.mul_(s["w"])
    dh = rstd * (g - g.sum(1, keepdim=True) / D - unit * (g * unit).sum(1, keepdim=True) / D)
    if s["add"] is not None:
        dh += s["add"]
    out["dh"] = dh
    if s["case"]["p"] > 0:
        out["dx"] = _exact_dropped(dh, s["case"]["p"], s["seed"])
    return out


def _exact_logp(s):
    c, z = s["case"], s["logits"]
    scale = _f32(c["scale"])
    out = {k: torch.empty(c["N"], device=DEV, dtype=torch.float64)
           for k in ("logp", "entropy", "peak", "log_sum")}
    if c["top"]:
        out["top_logp"] = torch.empty(c["N"], c["top"], device=DEV, dtype=torch.float64)
        out["top_ids"] = torch.empty(c["N"], c["top"], device=DEV, dtype=torch.int32)
    for i in range(0, c["N"], 256):
        y = z[i:i + 256].double()
        l = torch.log_softmax(y * scale, 1)
        part = slice(i, i + len(l))
        out["peak"][part] = y.max(1).values
        out["log_sum"][part] = -l.max(1).values
        out["entropy"][part] = torch.special.entr(l.exp()).sum(1)
        t = s["targets"][part]
        out["logp"][part] = torch.where(t < 0, 0.0, l.gather(1, t.clamp(min=0)[:, None])[:, 0])
        if c["top"]:
            ids = torch.sort(y, dim=1, descending=True, stable=True).indices[:, :c["top"]]
            out["top_ids"][part] = ids.int()
            out["top_logp"][part] = l.gather(1, ids)
    return out


def _exact_logp_grad(s):
    c = s["case"]
    out = torch.empty(c["N"], c["V"], device=DEV, dtype=torch.float64)
    words = torch.arange(c["V"], device=DEV)
    scale = _f32(c["scale"])
    for i in range(0, c["N"], 256):
        part = slice(i, i + 256)
        l = scale * s["logits"][part].double() - scale * s["peak"][part, None].double()
        l -= s["log_sum"][part, None]
        prob = l.exp()
        hit = (s["targets"][part, None] == words).double()
        dlogp = torch.where(s["targets"][part] < 0, 0.0, s["dlogp"][part].double())
        d = (hit - prob) * dlogp[:, None]
        if s["dentropy"] is not None:
            inside = torch.special.entr(prob) - prob * s["entropy"][part, None]
            d = d + inside * s["dentropy"][part, None]
        out[part] = scale * d
    return out
