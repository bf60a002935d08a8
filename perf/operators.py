"""Timed cases of the dense and the 8-bit AdamW step and of the relative
position bias: the calls a trainer makes of the library (``own`` true), and
the same results from elementary torch operations (``own`` false).

- ``adamw``: one AdamW step over a list of parameter tensors, moments in fp32
  or in 8 bits (e4m3 codes with one power-of-two scale per 32 values).
- ``rows``: the lazy AdamW step of the touched rows of an embedding table
  with 8-bit moments.
- ``bias``: the learned relative position bias of every head, written out or
  added to the attention scores.
- ``bias_grad``: the gradient of the bias table.

8-bit state. A block of 32 consecutive values (of one tensor, or of one row
of a table) has a scale 2^k, k the smallest integer with max|x| <= 448 2^k,
kept as the byte k + 127. A value is x = code * 2^k. The first moment is kept
as it is, the second as its square root. Rounding is stochastic, from the
32-bit word h of the element's number: with ulp the step of the e4m3 grid at
|x| 2^-k, the code is ulp * floor(|x| 2^-k / ulp + R / 2^20), R = the high
20 bits of h for the first moment and the low 20 for the second; a second
moment that is not zero never gets the code zero. An element whose new second
moment is not finite keeps its parameter and moments.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
BETA1, BETA2, EPS, WD = 0.9, 0.999, 1e-8, 0.01
GRADS = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # A small recurrent model's tensors: launch latency is all there is.
        {"name": "adamw32_tiny", "op": "adamw", "states": 32, "grad": "f32", "copy": False,
         "layers": 1, "width": 64, "rows": 0, "odd": False},
        # Two layers of the width of the paper's projection, with odd and empty tensors between.
        {"name": "adamw32_odd_512", "op": "adamw", "states": 32, "grad": "f32", "copy": False,
         "layers": 2, "width": 512, "rows": 98, "odd": True},
        # 12 layers and an output table: mixed precision, fp32 masters with bf16 copies.
        {"name": "adamw32_large", "op": "adamw", "states": 32, "grad": "bf16", "copy": True,
         "layers": 12, "width": 1024, "rows": 50_000, "odd": False},
        # The same two widths with 8-bit moments.
        {"name": "adamw8_odd_512", "op": "adamw", "states": 8, "grad": "f32", "copy": False,
         "layers": 2, "width": 512, "rows": 98, "odd": True},
        {"name": "adamw8_large", "op": "adamw", "states": 8, "grad": "bf16", "copy": True,
         "layers": 12, "width": 1024, "rows": 50_000, "odd": False},
        # The touched rows of an 8K-token step, and of a 256K-token step over 2M words.
        {"name": "rows8_word_8k", "op": "rows", "V": 100_000, "D": 512, "U": 3_629, "cap": 8_192,
         "ids": 32},
        {"name": "rows8_vocab2m", "op": "rows", "V": 2_000_000, "D": 1024, "U": 129_362,
         "cap": 262_144, "ids": 64},
        # One new token against a cache (its length is odd), for all heads.
        {"name": "bias_token_4097", "op": "bias", "B": 1, "H": 16, "Lq": 1, "Lk": 4097,
         "mode": "past", "buckets": 32, "distance": 128, "dtype": "bf16", "add": True},
        # A batch's attention scores with the bias and the causal mask added in one pass.
        {"name": "bias_scores_2048", "op": "bias", "B": 8, "H": 16, "Lq": 2048, "Lk": 2048,
         "mode": "causal", "buckets": 32, "distance": 128, "dtype": "bf16", "add": True},
        # The table's gradient: short odd sequences, a causal batch, a large batch of encoders.
        {"name": "grad_short_odd", "op": "bias_grad", "B": 2, "H": 8, "Lq": 151, "Lk": 151,
         "mode": "both", "buckets": 32, "distance": 128, "dtype": "f32"},
        {"name": "grad_causal_1024", "op": "bias_grad", "B": 4, "H": 12, "Lq": 1024, "Lk": 1024,
         "mode": "causal", "buckets": 32, "distance": 128, "dtype": "bf16"},
        {"name": "grad_large", "op": "bias_grad", "B": 16, "H": 16, "Lq": 2048, "Lk": 2048,
         "mode": "both", "buckets": 32, "distance": 128, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("adamw", "adamw", "rows", "bias", "bias_grad"))
    if op == "adamw":
        width = _log(rng, 33, 1280)
        layers = _log(rng, 1, 12)
        rows = rng.choice((0, _log(rng, 50, 50_000)))
        if layers * 12 * width * width + rows * width > 190_000_000:
            layers, rows = 6, min(rows, 20_000)
        return {"op": op, "states": rng.choice((32, 8)), "grad": rng.choice(("f32", "bf16")),
                "copy": rng.random() < 0.5, "layers": layers, "width": width, "rows": rows,
                "odd": rng.random() < 0.5}
    if op == "rows":
        V, D = _log(rng, 1000, 1_000_000), _log(rng, 17, 2048)
        V = min(V, 1_000_000_000 // D)
        cap = min(V, _log(rng, 100, 130_000), 130_000_000 // D)
        return {"op": op, "V": V, "D": D, "U": _log(rng, max(1, cap // 20), cap), "cap": cap,
                "ids": rng.choice((32, 64))}
    case = {"op": op, "B": _log(rng, 1, 16), "H": rng.choice((4, 8, 12, 16, 24)),
            "Lq": _log(rng, 1, 2048), "Lk": _log(rng, 1, 4096),
            "mode": rng.choice(("both", "past", "causal")), "buckets": rng.choice((16, 32, 64)),
            "distance": rng.choice((100, 128, 256, 777)), "dtype": rng.choice(("f32", "bf16"))}
    while case["B"] * case["H"] * case["Lq"] * case["Lk"] > 500_000_000:
        case["B"] = 1
        case["Lq"] = (case["Lq"] + 1) // 2
    if op == "bias":
        case["add"] = rng.random() < 0.5
        if not case["add"]:
            case["B"] = 1
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _shapes(case):
    """(elements, decays) of every tensor: matrices decay, vectors do not."""
    w, got = case["width"], []
    for _ in range(case["layers"]):
        got += [(w * w, True)] * 4 + [(4 * w * w, True)] * 2 + [(w, False)] * 3 + [(4 * w, False)]
        if case["odd"]:
            got += [(1, False), (w * (w + 1) + 1, True), (0, False), (33, True)]
    if case["rows"]:
        got.append((case["rows"] * w, True))
    return got


def _starts(sizes, step, odd):
    """Where each tensor starts in the flat buffer: on whole steps, or (odd) right behind the last."""
    at, got = 0, []
    for n in sizes:
        got.append(at)
        at += n if odd else -(-n // step) * step
    return got, max(at, 1)


def _views(flat, starts, sizes):
    return [flat[a:a + n] for a, n in zip(starts, sizes)]


def _randn(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype).mul_(std)


def _moments(gen, n):
    """First and second moments as a run leaves them: the gradients' size varies from block to
    block, the second moment's root stays near it, and some values have never had a gradient."""
    size = torch.exp(_randn(gen, -(-n // 256), std=1.5) - 7.0).repeat_interleave(256)[:n]
    m = _randn(gen, n, std=0.3).mul_(size)
    r = _randn(gen, n, std=0.3).abs_().add_(0.5).mul_(size)
    none = torch.rand(n, generator=gen, device=DEV) < 0.01
    m[none] = 0
    r[none] = 0
    return m, r


def _random_codes(gen, shape, signed):
    """Codes as a run leaves them: any e4m3 number but NaN, the small ones seldom."""
    c = torch.randint(0x20, 0x7F, shape, generator=gen, device=DEV, dtype=torch.uint8)
    if signed:
        c ^= torch.randint(0, 2, shape, generator=gen, device=DEV, dtype=torch.uint8) << 7
    return c.view(CODES)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case, "op": case["op"]}
    if case["op"] == "adamw":
        sizes, decays = [n for n, _ in _shapes(case)], [d for _, d in _shapes(case)]
        starts, total = _starts(sizes, 64, case["odd"])
        blocks = [-(-n // BLOCK) for n in sizes]
        bstarts, btotal = _starts(blocks, 1, True)
        flat = {"p": _randn(gen, total, std=0.02),
                "g": (_randn(gen, total, std=1.0) *
                      torch.exp(_randn(gen, -(-total // 256), std=1.5) - 7.0)
                      .repeat_interleave(256)[:total]).to(GRADS[case["grad"]])}
        if case["copy"]:
            flat["copy"] = flat["p"].to(torch.bfloat16)
        if case["states"] == 32:
            flat["m"], flat["v"] = _moments(gen, total)
            flat["v"].square_()
        else:
            flat["m"] = _random_codes(gen, (total,), True)
            flat["v"] = _random_codes(gen, (total,), False)
            size = torch.randint(-26, -15, (btotal,), generator=gen, device=DEV)
            flat["m_scale"] = (size + 126).to(torch.uint8)
            flat["v_scale"] = (size + 127).to(torch.uint8)
        s.update(flat=flat, sizes=sizes, decay=decays, step=100,
                 grad_scale=torch.full((1,), 0.5, device=DEV))
        for k, x in flat.items():
            s[k] = _views(x, bstarts, blocks) if k.endswith("_scale") else _views(x, starts, sizes)
        if own:
            from paper_1810_10045_amd import lmzipf as lz
            s["plan"] = lz.adamw_plan(s["p"], s["g"], s["m"], s["v"], m_scale=s.get("m_scale"),
                                      v_scale=s.get("v_scale"), copies=s.get("copy"),
                                      decay=decays)
    elif case["op"] == "rows":
        V, D, U, cap = case["V"], case["D"], case["U"], case["cap"]
        nb = -(-D // BLOCK)
        idt = torch.int32 if case["ids"] == 32 else torch.int64
        rows = torch.zeros(cap, dtype=idt, device=DEV)
        rows[:U] = torch.randperm(V, generator=gen, device=DEV)[:U].sort().values.to(idt)
        size = torch.randint(-26, -15, (V, 1), generator=gen, device=DEV)
        s.update(table=_randn(gen, V, D, std=0.02), rows=rows, n=U,
                 n_rows=torch.tensor([U], dtype=torch.int64, device=DEV),
                 vals=_randn(gen, cap, D, std=1e-3), step=100,
                 m=_random_codes(gen, (V, D), True), v=_random_codes(gen, (V, D), False),
                 m_scale=(size + 126).to(torch.uint8).expand(V, nb).contiguous(),
                 v_scale=(size + 127).to(torch.uint8).expand(V, nb).contiguous())
    else:
        B, H, Lq, Lk = (case[k] for k in ("B", "H", "Lq", "Lk"))
        dt = GRADS[case["dtype"]]
        s["q_start"] = Lk - Lq if case["mode"] != "both" else 0
        if case["op"] == "bias":
            s["table"] = _randn(gen, case["buckets"], H)
            s["add"] = _randn(gen, B, H, Lq, Lk, std=3.0).to(dt) if case["add"] else None
        else:
            s["dout"] = _randn(gen, B, H, Lq, Lk, std=1e-3).to(dt)
        if own:
            from paper_1810_10045_amd import lmzipf as lz
            s["buckets"] = lz.rel_buckets(case["buckets"], case["distance"], case["mode"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return {"adamw": _adamw, "rows": _rows, "bias": _bias, "bias_grad": _bias_grad}[s["op"]](s)


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


_B1, _B2 = _f32(BETA1), _f32(BETA2)  # the step's parameters are fp32 numbers
_LR, _EPS, _WD = _f32(1e-3), _f32(EPS), _f32(WD)


def _adamw(s):
    step = s["step"]
    s["step"] += 1
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        lz.adamw(s["plan"], lr=_LR, beta1=_B1, beta2=_B2, eps=_EPS, weight_decay=_WD, step=step,
                 grad_scale=s["grad_scale"], seed=step)
    elif s["case"]["states"] == 32:
        _adamw_plain32(s, step)
    else:
        first = _numbers(s["sizes"])
        for_each = zip(s["p"], s["g"], s["m"], s["v"], s["m_scale"], s["v_scale"], s["decay"],
                       first)
        new = [(p, m, v, ms, vs) + _step8(p, g.float() * s["grad_scale"], m, v, ms, vs,
                                          _WD if d else 0.0, step, step,
                                          e0 + torch.arange(p.numel(), device=DEV))
               for p, g, m, v, ms, vs, d, e0 in for_each if p.numel()]
        [old.copy_(x) for a in new for old, x in zip(a[:5], a[5:])]
        if s["case"]["copy"]:
            torch._foreach_copy_(s["copy"], s["p"])
    out = {k: x for k, x in s["flat"].items() if k != "g"}
    out.update({k: x.view(SCALES) for k, x in out.items() if k.endswith("_scale")})
    return out


def _numbers(sizes):
    """The number of each tensor's first element: every tensor starts on a whole block."""
    got, at = [], 0
    for n in sizes:
        got.append(at)
        at += -(-n // BLOCK) * BLOCK
    return got


def _adamw_plain32(s, step):
    live = [i for i, n in enumerate(s["sizes"]) if n]
    p, m, v, g = ([s[k][i] for i in live] for k in "pmvg")
    wd = [_WD if s["decay"][i] else 0.0 for i in live]
    g = torch._foreach_mul([x.float() for x in g], s["grad_scale"][0])
    torch._foreach_mul_(m, _B1)
    torch._foreach_add_(m, torch._foreach_mul(g, 1 - _B1))
    torch._foreach_mul_(v, _B2)
    torch._foreach_add_(v, torch._foreach_mul(torch._foreach_mul(g, g), 1 - _B2))
    d = torch._foreach_sqrt(torch._foreach_mul(v, 1 / (1 - _B2 ** step)))
    torch._foreach_add_(d, _EPS)
    u = torch._foreach_div(torch._foreach_mul(m, 1 / (1 - _B1 ** step)), d)
    torch._foreach_add_(u, torch._foreach_mul(p, wd))
    torch._foreach_add_(p, torch._foreach_mul(u, -_LR))
    if s["case"]["copy"]:
        torch._foreach_copy_([s["copy"][i] for i in live], p)


M32 = 0xFFFFFFFF


def _keys(seed):
    """Two 32-bit words from the 64-bit seed."""
    z = (seed * 0x9E3779B97F4A7C15 + 0x632BE59BD9B4E019) & (2 ** 64 - 1)
    z = ((z ^ (z >> 29)) * 0xD6E8FEB86659FD93) & (2 ** 64 - 1)
    z ^= z >> 32
    return z & M32, z >> 32


def _words(e, seed):
    """The 32-bit word of each element number in `e` (int64)."""
    k0, k1 = _keys(seed)
    h = (((e & M32) ^ k0) * 0x9E3779B1) & M32
    h = h ^ (h >> 15)
    h = ((h + k1 + (e >> 32) * 0x85EBCA77) & M32) * 0xC2B2AE3D & M32
    return h ^ (h >> 16)


def _decode(codes, scale, shape):
    """code * 2^k of [.., n] codes with [.., ceil(n / 32)] scale bytes."""
    k = (scale.to(torch.int32) - 127).repeat_interleave(BLOCK, -1)[..., :shape[-1]]
    return torch.ldexp(codes.float(), k)


def _encode(x, R, keep):
    """Codes and scale bytes of x [.., n]; `keep`: no code zero for a value that is not."""
    n = x.shape[-1]
    pad = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK))
    top = pad.view(*x.shape[:-1], -1, BLOCK).amax(-1)
    f, e = torch.frexp(top)
    k = (e - 9 + (f > 0.875)).clamp_(min=-127).masked_fill_(top == 0, -127)
    y = torch.ldexp(x.abs(), -k.repeat_interleave(BLOCK, -1)[..., :n]).double()
    exp = torch.frexp(y)[1].clamp_(min=-5) - 1
    ulp = torch.ldexp(torch.ones_like(y), exp - 3)
    q = torch.floor(y / ulp + R * 2.0 ** -20) * ulp
    q = torch.where((q == 0) & (x != 0), 2.0 ** -9, q) if keep else q
    return torch.copysign(q, x.double()).float().to(CODES), (k + 127).to(torch.uint8)


def _step8(p, g, m8, v8, ms, vs, wd, step, seed, e):
    """The new parameter, codes and scales of values [.., n] with the element numbers e."""
    h = _words(e, seed)
    m, r = _decode(m8, ms, p.shape), _decode(v8, vs, p.shape)
    m1 = m * _B1 + g * (1 - _B1)
    v1 = (r * r) * _B2 + (g * (1 - _B2)) * g
    r1 = torch.sqrt(v1)
    mhat = m1 * (1 / (1 - _B1 ** step))
    d = r1 * math.sqrt(1 / (1 - _B2 ** step)) + _EPS
    p1 = p - _LR * (mhat / d + wd * p)
    ok = torch.isfinite(v1)
    p1, m1, r1 = torch.where(ok, p1, p), torch.where(ok, m1, m), torch.where(ok, r1, r)
    m8, ms = _encode(m1, h >> 12, False)
    v8, vs = _encode(r1, h & 0xFFFFF, True)
    return p1, m8, v8, ms, vs


def _rows(s):
    step = s["step"]
    s["step"] += 1
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        lz.sparse_apply_q8(s["table"], s["rows"], s["n_rows"], s["vals"], s["m"], s["v"],
                           s["m_scale"], s["v_scale"], lr=_LR, beta1=_B1, beta2=_B2, eps=_EPS,
                           weight_decay=_WD, step=step, seed=step)
    else:
        at = s["rows"][:s["n"]].long()
        m8, v8 = s["m"].view(torch.uint8), s["v"].view(torch.uint8)
        e = at[:, None] * s["table"].shape[1] + torch.arange(s["table"].shape[1], device=DEV)
        p, m, v, ms, vs = _step8(s["table"][at], s["vals"][:s["n"]], m8[at].view(CODES),
                                 v8[at].view(CODES), s["m_scale"][at], s["v_scale"][at], _WD,
                                 step, step, e)
        s["table"][at] = p
        m8[at], v8[at] = m.view(torch.uint8), v.view(torch.uint8)
        s["m_scale"][at], s["v_scale"][at] = ms, vs
    return {"table": s["table"], "m": s["m"], "v": s["v"], "m_scale": s["m_scale"].view(SCALES),
            "v_scale": s["v_scale"].view(SCALES)}


def _bucket(rel, buckets, distance, mode):
    """The bucket of each distance rel = key position - query position: one for each distance up
    to half of a side's buckets, then growing with the distance's logarithm up to `distance`."""
    n = buckets // 2 if mode == "both" else buckets
    d = rel.abs() if mode == "both" else (-rel).clamp(min=0)
    near = n // 2
    far = torch.log(d.double().clamp(min=1) / near) / math.log(distance / near) * (n - near)
    far = (near + torch.floor(far + 1e-9).long()).clamp(max=n - 1)  # 1e-9: borders are reached
    b = torch.where(d < near, d, far)
    return b + n * (rel > 0) if mode == "both" else b


def _bias(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        return lz.rel_bias(s["table"], s["buckets"], c["Lq"], c["Lk"], q_start=s["q_start"],
                           add=s["add"], dtype=GRADS[c["dtype"]])
    k = torch.arange(c["Lk"], device=DEV)
    rel = k - torch.arange(s["q_start"], s["q_start"] + c["Lq"], device=DEV)[:, None]
    out = s["table"][_bucket(rel, c["buckets"], c["distance"], c["mode"])].permute(2, 0, 1)
    if s["add"] is not None:
        out = s["add"].float() + out
    if c["mode"] == "causal":
        out = out.masked_fill(rel > 0, -math.inf)
    out = out.to(GRADS[c["dtype"]])
    return out.contiguous()


def _bias_grad(s):
    c = s["case"]
    if own:
        from paper_1810_10045_amd import lmzipf as lz
        return lz.rel_bias_grad(s["dout"], s["buckets"], q_start=s["q_start"])
    Lq, Lk, H = c["Lq"], c["Lk"], c["H"]
    d = s["dout"].sum(0, dtype=torch.float32)
    # Rows of Lq + Lk - 1, read as rows of one more: a diagonal becomes a column.
    d = torch.nn.functional.pad(d, (0, Lq - 1)).reshape(H, -1)
    d = torch.nn.functional.pad(d, (Lq - 1, 1)).reshape(H, Lq, Lq + Lk).sum(1)[:, :-1]
    rel = torch.arange(Lq + Lk - 1, device=DEV) - (Lq - 1) - s["q_start"]
    if c["mode"] == "causal":
        d = d.masked_fill(rel > 0, 0.0)
    b = _bucket(rel, c["buckets"], c["distance"], c["mode"])
    hit = (b == torch.arange(c["buckets"], device=DEV)[:, None]).float()
    return (d * hit[:, None]).sum(-1)


# ---------------------------------------------------------------------------
# What a pass has to move and compute
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "adamw":
        n = sum(n for n, _ in _shapes(case))
        per = 8 + (4 if case["grad"] == "f32" else 2) + (2 if case["copy"] else 0)
        per += 16 if case["states"] == 32 else 4 + 4 / BLOCK
        return {"bytes": per * n, "flops": 20 * n}
    if case["op"] == "rows":
        n = case["U"] * case["D"]
        return {"bytes": n * (8 + 4 + 4) + 4 * case["U"] * -(-case["D"] // BLOCK) +
                case["U"] * case["ids"] // 8, "flops": 20 * n}
    B, H, Lq, Lk = (case[k] for k in ("B", "H", "Lq", "Lk"))
    size = 4 if case["dtype"] == "f32" else 2
    q0 = Lk - Lq if case["mode"] != "both" else 0
    seen = Lq * Lk
    if case["mode"] == "causal":
        seen = sum(min(max(q0 + i + 1, 0), Lk) for i in range(Lq))
    if case["op"] == "bias":
        return {"bytes": size * B * H * (Lq * Lk + (seen if case["add"] else 0)) +
                4 * H * case["buckets"], "flops": B * H * seen if case["add"] else 0}
    return {"bytes": size * B * H * seen + 4 * H * case["buckets"], "flops": B * H * seen}


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
    return {"adamw": _exact_adamw, "rows": _exact_rows, "bias": _exact_bias,
            "bias_grad": _exact_bias_grad}[case["op"]](s)


def _exact_values(p, g, m, root, wd, step):
    """(p, m, root of v) after the step, in 64 bits."""
    g = g.double()
    m = _B1 * m + (1 - _B1) * g
    v = _B2 * root ** 2 + (1 - _B2) * g ** 2
    hat = (v / (1 - _B2 ** step)).sqrt_().add_(_EPS)
    return p.double() * (1 - _LR * wd) - _LR * (m / (1 - _B1 ** step)) / hat, m, v.sqrt_()


def _grid():
    """The e4m3 numbers from 0 to 448 in ascending order: their bits count them."""
    return torch.arange(0x7F, dtype=torch.uint8, device=DEV).view(CODES).double()


def _exact_codes(x, number, seed, first):
    """Codes (as values) and scales (as powers of two) of rows x [n, D] of values."""
    grid, n = _grid(), x.shape[-1]
    spread = [torch.nn.functional.pad(t, (0, -n % BLOCK)).view(*t.shape[:-1], -1, BLOCK)
              for t in (x, number)]
    top = spread[0].abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -127)))
    y = spread[0].abs() / torch.exp2(k)
    below = torch.searchsorted(grid, y, right=True) - 1
    low, high = grid[below], grid[(below + 1).clamp(max=0x7E)]
    word = _exact_words(spread[1], seed)
    part = (word // 4096 if first else word % 2 ** 20).double() / 2 ** 20
    step = torch.where(high > low, high - low, 32.0)
    up = (y - low) / step + part >= 1
    q = torch.where(up, high, low)
    if not first:
        q = torch.where((q == 0) & (y > 0), grid[1], q)
    q = q * torch.sign(spread[0])
    return q.flatten(-2)[..., :n], torch.exp2(k.squeeze(-1))


def _exact_words(number, seed):
    k0, k1 = _keys(seed)
    a = number.remainder(2 ** 32).bitwise_xor(k0).mul(0x9E3779B1).remainder(2 ** 32)
    a = a.bitwise_xor(a.div(2 ** 15, rounding_mode="floor"))
    a = a.add(k1).add(number.div(2 ** 32, rounding_mode="floor").mul(0x85EBCA77))
    a = a.remainder(2 ** 32).mul(0xC2B2AE3D).remainder(2 ** 32)
    return a.bitwise_xor(a.div(2 ** 16, rounding_mode="floor"))


def _exact_adamw(s):
    step, out = s["step"], {k: x.double() for k, x in s["flat"].items() if k not in ("g", "copy")}
    eight = s["case"]["states"] == 8
    if eight:
        for k in ("m_scale", "v_scale"):
            out[k] = torch.exp2(out[k] - 127)
    number = 0
    where = {k: (s["flat"][k].data_ptr(), s["flat"][k].element_size()) for k in out}
    for i, n in enumerate(s["sizes"]):
        if not n:
            continue

        def part(k):
            a = (s[k][i].data_ptr() - where[k][0]) // where[k][1]
            return out[k][a:a + s[k][i].numel()]
        p, m, v = part("p"), part("m"), part("v")
        wd = _WD if s["decay"][i] else 0.0
        g = s["g"][i].double() * s["grad_scale"].double()
        if eight:
            ms, vs = part("m_scale"), part("v_scale")
            at = torch.arange(n, device=DEV) // BLOCK
            new_p, new_m, root = _exact_values(p, g, m * ms[at], v * vs[at], wd, step)
            e = number + torch.arange(n, device=DEV)
            m[:], ms[:] = _exact_codes(new_m, e, step, True)
            v[:], vs[:] = _exact_codes(root, e, step, False)
            number += -(-n // BLOCK) * BLOCK
        else:
            new_p, new_m, root = _exact_values(p, g, m, v.sqrt(), wd, step)
            m[:], v[:] = new_m, root.square()
        p[:] = new_p
    if s["case"]["copy"]:
        copy = s["flat"]["copy"].double()
        for i, n in enumerate(s["sizes"]):
            a = (s["p"][i].data_ptr() - where["p"][0]) // 4
            copy[a:a + n] = out["p"][a:a + n]
        out["copy"] = copy
    return out


def _exact_rows(s):
    at, step = s["rows"][:s["n"]].long(), s["step"]
    D = s["table"].shape[1]
    out = {"table": s["table"].double()}
    old = {k: s[k].view(torch.uint8)[at].view(CODES).double() for k in "mv"}
    scale = {k: torch.exp2(s[k + "_scale"][at].double() - 127).repeat_interleave(BLOCK, 1)[:, :D]
             for k in "mv"}
    p, m, root = _exact_values(out["table"][at], s["vals"][:s["n"]], old["m"] * scale["m"],
                               old["v"] * scale["v"], _WD, step)
    out["table"][at] = p
    e = at[:, None] * D + torch.arange(D, device=DEV)
    for k, x, first in (("m", m, True), ("v", root, False)):
        q, sc = _exact_codes(x, e, step, first)
        # e4m3 numbers and powers of two: fp32 holds them
        out[k], out[k + "_scale"] = s[k].float(), torch.exp2(s[k + "_scale"].float() - 127)
        out[k][at], out[k + "_scale"][at] = q.float(), sc.float()
    return out


def _exact_table(c, lo, hi):
    """The bucket of each distance in [lo, hi), by whole numbers: a far distance d is in bucket
    near + t or above where d^N >= near^(N - t) distance^t, N the number of far buckets."""
    n = c["buckets"] // 2 if c["mode"] == "both" else c["buckets"]
    near = n // 2
    N = n - near
    first = [next(d for d in range(near, c["distance"] + 1)
                  if d ** N >= near ** (N - t) * c["distance"] ** t) for t in range(N)]
    got = []
    for rel in range(lo, hi):
        d = abs(rel) if c["mode"] == "both" else max(-rel, 0)
        b = d if d < near else near - 1 + sum(d >= f for f in first)
        got.append(b + (n if c["mode"] == "both" and rel > 0 else 0))
    return torch.tensor(got, device=DEV)


def _exact_bias(s):
    c = s["case"]
    lo = 1 - c["Lq"] - s["q_start"]
    line = s["table"].double()[_exact_table(c, lo, c["Lk"] - s["q_start"])]
    if c["mode"] == "causal":
        line[max(0, 1 - lo):] = -math.inf
    # row i of a head is the line from key 0 at query i on
    out = line.T.unfold(1, c["Lk"], 1).flip(1)
    return (out if s["add"] is None else s["add"].double() + out).contiguous()


def _exact_bias_grad(s):
    c = s["case"]
    lo, hi = 1 - c["Lq"] - s["q_start"], c["Lk"] - s["q_start"]
    of, out = _exact_table(c, lo, hi), torch.zeros(c["buckets"], c["H"], device=DEV,
                                                    dtype=torch.float64)
    d = s["dout"].sum(0, dtype=torch.float64)
    sums = torch.stack([d.diagonal(r + s["q_start"], 1, 2).sum(-1) for r in range(lo, hi)])
    if c["mode"] == "causal":
        sums[max(0, 1 - lo):] = 0
    return out.index_add_(0, of, sums)
