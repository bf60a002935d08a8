"""Dropout, layer norm and token log probabilities in 64 bits on the CPU (no test
functions here), each with how far fp32 arithmetic may be off.

U = 2^-24 is half a step of fp32 relative to the value. A sum of n fp32 numbers in any
order is off by at most (n's depth of additions) U times the sum of their magnitudes; DEPTH
bounds the additions that one number takes part in inside a row (a lane adds at most 32
numbers of its own row or batch, lanes and waves add 6 + 16 more)."""
from __future__ import annotations

import numpy as np
import torch

import moments_ref as M

U = 2.0 ** -24
DEPTH = 64
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 1e-37  # fp32 numbers below 2^-126 may be flushed to zero


def rounded(ref, dtype):
    """How far the rounding to `dtype` may move ref."""
    return HALF[dtype] * np.abs(ref) * 1.01 + TINY


def keep(rows, D, p, seed):
    """(which elements are kept, their factor)."""
    T = round(65536 * float(np.float32(p)))
    half = (D + 1) // 2
    w = M.words(np.arange(rows * half, dtype=np.uint64), seed).reshape(rows, half)
    bits = np.empty((rows, 2 * half), np.uint32)
    bits[:, 0::2], bits[:, 1::2] = w & np.uint32(0xFFFF), w >> np.uint32(16)
    return bits[:, :D] >= T, (65536 / (65536 - T) if T < 65536 else 0.0)


def dropout(x, p, seed, add=None):
    """(value, tolerance before the last rounding) of float64 arrays."""
    k, c = keep(*x.shape, p, seed)
    y = np.where(k, np.where(k, x, 0.0) * c, 0.0)
    tol = 2 * U * np.abs(y)  # c is rounded, and the product
    if add is not None:
        y = add + y
        tol = tol + U * np.abs(y)
    return y, tol


def norm(x, weight, bias, eps, p=0.0, seed=0, add=None):
    """{name: (value, tolerance before the last rounding)}."""
    h, dh = dropout(x, p, seed, add) if p > 0 or add is not None else (x, np.zeros_like(x))
    D = x.shape[1]
    w = np.ones(D) if weight is None else weight
    b = np.zeros(D) if bias is None else bias
    mean = h.mean(1, keepdims=True)
    size = np.abs(h).mean(1, keepdims=True)
    d_mean = dh.mean(1, keepdims=True) + (DEPTH + 2) * U * size
    d = h - mean
    d_d = dh + d_mean + U * (np.abs(d) + d_mean)
    var = (d * d).mean(1, keepdims=True)
    d_var = (2 * np.abs(d) * d_d + d_d ** 2).mean(1, keepdims=True) + (DEPTH + 4) * U * var
    rstd = 1 / np.sqrt(var + eps)
    d_rstd = rstd * (0.51 * (d_var + U * (var + eps)) / (var + eps) + 3 * U)
    n = d * rstd
    d_n = d_d * rstd + np.abs(d) * d_rstd + U * np.abs(n)
    y = n * w + b
    return {"h": (h, dh), "mean": (mean[:, 0], d_mean[:, 0]), "rstd": (rstd[:, 0], d_rstd[:, 0]),
            "y": (y, 1.01 * (d_n * np.abs(w) + U * (np.abs(n * w) + np.abs(y))))}


def norm_grad(dy, h, mean, rstd, weight, add=None, p=0.0, seed=0):
    """The gradients' {name: (value, tolerance before the last rounding)}."""
    rows, D = dy.shape
    w = np.ones(D) if weight is None else weight
    m, r = mean[:, None], rstd[:, None]
    n = (h - m) * r
    d_n = 2 * U * np.abs(n) + U * np.abs(h - m) * r
    g = dy * w
    size = np.abs(g)
    e0, e1 = g.mean(1, keepdims=True), (g * n).mean(1, keepdims=True)
    d_e0 = (DEPTH + 4) * U * size.mean(1, keepdims=True)
    d_e1 = (size * d_n).mean(1, keepdims=True) + (DEPTH + 4) * U * (size * np.abs(n)).mean(1, keepdims=True)
    inner = g - e0 - n * e1
    d_inner = (4 * U * (size + np.abs(e0) + np.abs(n * e1)) + d_e0 + np.abs(n) * d_e1 +
               d_n * np.abs(e1))
    dh = r * inner + (0.0 if add is None else add)
    d_dh = r * d_inner + 2 * U * (np.abs(r * inner) + np.abs(dh))
    depth = DEPTH + 40 + rows // 256
    out = {"dh": (dh, d_dh),
           "dweight": ((dy * n).sum(0), (np.abs(dy) * d_n).sum(0) + depth * U * np.abs(dy * n).sum(0)),
           "dbias": (dy.sum(0), depth * U * np.abs(dy).sum(0))}
    if p > 0:
        k, c = keep(rows, D, p, seed)
        dx = np.where(k, dh * c, 0.0)
        out["dx"] = (dx, np.where(k, d_dh * c, 0.0) + 2 * U * np.abs(dx))
    return out


def logprobs(x, targets, scale, top=0, ignore=-100):
    """{name: (value, tolerance)} of float64 logits [N, V]; targets int64 or None. ids exact."""
    N, V = x.shape
    peak = x.max(1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = (x - np.where(np.isinf(peak), 0.0, peak)[:, None]) * scale
        e = np.exp(d)
        S = e.sum(1)
        q = np.where(S[:, None] > 0, e / S[:, None], 0.0)
        size = np.where(q > 0, np.abs(d), 0.0)
        first, second = (q * size).sum(1), (q * size ** 2).sum(1)
        log_sum = np.log(S)
        entropy = np.where(S > 0, log_sum + first, 0.0)
        # a logit's exponent is off by 5 U of itself (a difference, a product, the rounded
        # scale, log2 e and their product), its power by two units; sums have the depth of a
        # row's lanes and of its batches of 32
        depth = DEPTH + V // 4096
        d_log = 5 * U * first + (depth + 4) * U + 2 * U * np.abs(np.where(S > 0, log_sum, 0))
        d_ent = d_log + U * (5 * (second + first) + (2 * depth + 12) * first + 2 * np.abs(entropy))
        out = {"peak": (peak, 0 * peak), "log_sum": (log_sum, d_log), "entropy": (entropy, d_ent)}

        def at(ids):
            row = np.arange(N).reshape(-1, *[1] * (ids.ndim - 1))
            ls, dl = (v.reshape(-1, *[1] * (ids.ndim - 1)) for v in (log_sum, d_log))
            y = d[row, ids]
            z = y - ls
            return (np.where(np.isinf(x[row, ids]), -np.inf, z),
                    3 * U * np.where(np.isinf(y), 0, np.abs(y)) + dl + U * np.where(np.isinf(z), 0, np.abs(z)))
        if targets is not None:
            t = np.where(targets == ignore, 0, targets)
            y, tol = at(t)
            out["logp"] = (np.where(targets == ignore, 0.0, y), np.where(targets == ignore, 0.0, tol))
        if top:
            pad = np.full((N, max(0, top - V)), -np.inf)
            ids = np.argsort(-np.concatenate([x, pad], 1), axis=1, kind="stable")[:, :top]
            there = np.isfinite(np.take_along_axis(np.concatenate([x, pad], 1), ids, 1))
            y, tol = at(np.minimum(ids, V - 1))
            out["top_ids"] = (np.where(there, ids, -1), None)
            out["top_logp"] = (np.where(there, y, -np.inf), np.where(there, tol, 0.0))
    return out


def logprobs_grad(x, targets, peak, log_sum, scale, dlogp=None, entropy=None, dentropy=None,
                  ignore=-100):
    """(value, tolerance before the last rounding); peak and log_sum as the call gets them."""
    N, V = x.shape
    none = np.isinf(peak)
    with np.errstate(invalid="ignore", over="ignore"):
        d = (x - np.where(none, 0.0, peak)[:, None]) * scale
        l = d - np.where(none, 0.0, log_sum)[:, None]
        q = np.exp(l)
        l = np.where(q > 0, l, 0.0)
        d = np.where(q > 0, np.abs(d), 0.0)
    # l is a difference, a product of a rounded scale and a sum; 2^x is off by two units and
    # its argument by two roundings
    rel = U * (4 * np.abs(l) + 3 * d + np.abs(np.where(none, 0, log_sum))[:, None] + 4)
    a = np.zeros(N) if dlogp is None else np.where(targets == ignore, 0.0, dlogp)
    hit = np.zeros((N, V))
    if targets is not None:
        hit[np.arange(N), np.where(targets == ignore, 0, targets)] = 1
    a = a[:, None]
    y = a * (hit - q)
    tol = np.abs(a) * (q * rel + 4 * U * (q + hit))
    if dentropy is not None:
        b, H = dentropy[:, None], entropy[:, None]
        y = y - b * q * (l + H)
        tol = tol + np.abs(b) * q * (rel * (1 + np.abs(l + H)) + 5 * U * (np.abs(l) + np.abs(H)))
    # a power below 2^-126 may come out as 0, and each term that it is a factor of with it (a
    # term holds q |l + H|, up to 88 and more times the 2^-126 that TINY allows for)
    gone = q < 2.0 ** -125
    tol = tol + np.where(gone, np.abs(a) * q, 0.0)
    if dentropy is not None:
        tol = tol + np.where(gone, np.abs(b) * q * np.abs(l + H), 0.0)
    tol = scale * (tol + 3 * U * np.abs(y))
    y = np.where(none[:, None], 0.0, scale * y)
    return y, np.where(none[:, None], 0.0, tol)
