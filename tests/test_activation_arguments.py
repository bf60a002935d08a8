"""Host-side checks of dropout, layer norm and the token log probabilities (no GPU): calls
that are refused return before anything is launched; the mask's words have the shares and
the independence that dropout asks of them; the definitions' gradients agree with differences."""
import ctypes
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import activations_ref as A  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")
OK, INVAL, WORKSPACE, UNSUPPORTED = 0, 1, 3, 5
F32, BF16 = 0, 1
FAR = 1 << 20  # operands are this far apart unless a test says otherwise


@pytest.fixture(scope="module")
def lz():
    if not os.path.exists(LIB):
        from paper_1810_10045_amd import build
        build.build()
    from paper_1810_10045_amd import lmzipf
    return lmzipf


class Calls:
    """The entry points on made-up addresses (the host reads none of them)."""

    def __init__(self, lz):
        self.lib = lz.lib()

    def dropout(self, x=1 * FAR, ld_x=8, add=None, ld_add=0, out=2 * FAR, ld_out=8, rows=4, D=8,
                dtype=F32, p=0.5, seed_at=None):
        return self.lib.lm_dropout(x, ld_x, add, ld_add, out, ld_out, rows, D, dtype, p, 1, seed_at,
                                   None)

    def norm(self, x=1 * FAR, ld_x=8, add=None, ld_add=0, rows=4, D=8, dtype=F32, weight=3 * FAR,
             bias=4 * FAR, eps=1e-5, p=0.0, seed_at=None, y=5 * FAR, ld_y=8, h=None, ld_h=0,
             mean=6 * FAR, rstd=7 * FAR):
        return self.lib.lm_layer_norm(x, ld_x, add, ld_add, rows, D, dtype, weight, bias, eps, p, 1,
                                      seed_at, y, ld_y, h, ld_h, mean, rstd, None)

    def norm_grad(self, dy=1 * FAR, ld_dy=8, h=2 * FAR, ld_h=8, add=None, ld_add=0, rows=4000, D=8,
                  dtype=F32, mean=3 * FAR, rstd=4 * FAR, weight=5 * FAR, p=0.0, dh=6 * FAR, ld_dh=8,
                  dx=None, ld_dx=0, dw=7 * FAR, db=8 * FAR, ws=9 * FAR, ws_bytes=1 << 18):
        return self.lib.lm_layer_norm_grad(dy, ld_dy, h, ld_h, add, ld_add, rows, D, dtype, mean,
                                           rstd, weight, p, 1, None, dh, ld_dh, dx, ld_dx, dw, db, 0,
                                           ws, ws_bytes, None)

    def logprobs(self, logits=1 * FAR, ld=100, N=4, V=100, dtype=F32, targets=2 * FAR, idtype=1,
                 scale=1.0, top=0, logp=3 * FAR, entropy=4 * FAR, peak=5 * FAR, log_sum=6 * FAR,
                 top_logp=None, top_ids=None, dev_err=None, ws=None, ws_bytes=0):
        return self.lib.lm_token_logprobs(logits, ld, N, V, dtype, targets, idtype, -100, scale, top,
                                          logp, entropy, peak, log_sum, top_logp, top_ids, dev_err,
                                          ws, ws_bytes, None)

    def logprobs_grad(self, logits=1 * FAR, ld=100, N=4, V=100, dtype=F32, targets=2 * FAR, idtype=1,
                      scale=1.0, peak=3 * FAR, log_sum=4 * FAR, dlogp=5 * FAR, entropy=6 * FAR,
                      dentropy=None, out=7 * FAR, ld_out=100):
        return self.lib.lm_token_logprobs_grad(logits, ld, N, V, dtype, targets, idtype, -100, scale,
                                               peak, log_sum, dlogp, entropy, dentropy, out, ld_out,
                                               None)


@pytest.fixture(scope="module")
def c(lz):
    return Calls(lz)


NAN = float("nan")


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(rows=-1), INVAL), (dict(D=-1), INVAL),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(D=1 << 31, ld_x=1 << 31, ld_out=1 << 31), UNSUPPORTED),
    (dict(p=-0.1), INVAL), (dict(p=1.01), INVAL), (dict(p=NAN), INVAL), (dict(x=None), INVAL),
    (dict(out=None), INVAL), (dict(ld_x=7), INVAL), (dict(ld_out=7), INVAL),
    (dict(ld_x=(1 << 40) + 1), INVAL), (dict(add=3 * FAR, ld_add=7), INVAL),
    (dict(x=FAR + 2), INVAL), (dict(out=2 * FAR + 1), INVAL), (dict(dtype=BF16, x=FAR + 1), INVAL),
    (dict(seed_at=4 * FAR + 4), INVAL), (dict(seed_at=2 * FAR), INVAL),  # the seed in the output
    (dict(out=FAR + 4), INVAL), (dict(out=FAR, ld_out=9), INVAL), (dict(out=FAR + 32), INVAL),
    (dict(add=2 * FAR + 4, ld_add=8), INVAL), (dict(add=2 * FAR, ld_add=9), INVAL),
    (dict(rows=0), OK), (dict(D=0), OK), (dict(rows=0, x=None, out=None), OK)])
def test_dropout_refusals(c, kw, code):
    assert c.dropout(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(rows=-1), INVAL), (dict(D=0), INVAL),
    (dict(D=16385, ld_x=16385, ld_y=16385), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(eps=-1e-9), INVAL), (dict(eps=NAN), INVAL), (dict(eps=float("inf")), INVAL),
    (dict(p=2.0), INVAL), (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(mean=None), INVAL),
    (dict(rstd=None), INVAL), (dict(ld_x=7), INVAL), (dict(ld_y=7), INVAL),
    (dict(h=2 * FAR, ld_h=7), INVAL), (dict(h=2 * FAR + 2, ld_h=8), INVAL),
    (dict(h=5 * FAR, ld_h=8), INVAL),               # y and h in one place
    (dict(h=5 * FAR + 16, ld_h=8), INVAL),
    (dict(y=FAR + 4), INVAL),                       # y beside x by an element
    (dict(y=6 * FAR - 4), INVAL),                   # y over the means
    (dict(mean=7 * FAR - 4), INVAL),                # the means over rstd
    (dict(weight=5 * FAR + 8), INVAL), (dict(bias=7 * FAR), INVAL), (dict(weight=3 * FAR + 1), INVAL),
    (dict(rows=0), OK)])
def test_layer_norm_refusals(c, kw, code):
    assert c.norm(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(D=0), INVAL), (dict(rows=-1), INVAL),
    (dict(D=16385, ld_dy=16385, ld_h=16385, ld_dh=16385), UNSUPPORTED), (dict(p=-1.0), INVAL),
    (dict(dy=None), INVAL), (dict(h=None), INVAL), (dict(mean=None), INVAL), (dict(rstd=None), INVAL),
    (dict(dh=None), INVAL), (dict(ws=None), INVAL), (dict(ws_bytes=8), WORKSPACE),
    (dict(ws=9 * FAR + 2), INVAL), (dict(ld_dy=7), INVAL), (dict(ld_dh=7), INVAL),
    (dict(dx=6 * FAR, ld_dx=8), INVAL),             # dx and dh in one place
    (dict(dx=2 * FAR, ld_dx=9), INVAL),             # over h, at other rows
    (dict(dw=8 * FAR - 4), INVAL), (dict(dw=5 * FAR), INVAL), (dict(dw=3 * FAR), INVAL), (dict(ws=7 * FAR - 60), INVAL),
    (dict(dh=3 * FAR - 4), INVAL), (dict(add=6 * FAR + 4, ld_add=8), INVAL)])
def test_layer_norm_grad_refusals(c, kw, code):
    assert c.norm_grad(**kw) == code


def test_layer_norm_grad_of_few_rows_needs_no_workspace(c):
    """(refused for another reason, so that nothing is launched)"""
    assert c.norm_grad(rows=4, ws=None, ws_bytes=0, dw=5 * FAR) == INVAL
    assert c.norm_grad(rows=4, ws=None, ws_bytes=0, dw=8 * FAR - 4) == INVAL


def test_layer_norm_grad_workspace(lz):
    f = lz.lib().lm_layer_norm_grad_workspace_bytes
    assert f(0, 8, F32) == 0 and f(-1, 8, F32) == 0 and f(4, 0, F32) == 0 and f(4, 8, 3) == 0
    assert f(4, 16385, F32) == 0 and f(1 << 31, 8, F32) == 0
    for rows in (1, 100, 5000, 1 << 20):
        for D in (1, 8, 517, 2048, 16384):
            for t in (F32, BF16):
                assert f(rows, D, t) % (8 * D) == 0 and f(rows, D, t) <= 512 * 8 * D
    assert f(1 << 20, 2048, BF16) >= f(100, 2048, BF16) > 0
    assert f(1, 2048, BF16) == 0  # one workgroup writes the results itself


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(idtype=2), UNSUPPORTED), (dict(N=-1), INVAL), (dict(V=0), INVAL),
    (dict(top=-1), INVAL), (dict(top=65, top_logp=8 * FAR, top_ids=9 * FAR), UNSUPPORTED),
    (dict(V=(1 << 30) + 1, ld=1 << 31), UNSUPPORTED), (dict(N=1 << 31), UNSUPPORTED),
    (dict(scale=0.0), INVAL), (dict(scale=-1.0), INVAL), (dict(scale=NAN), INVAL),
    (dict(scale=float("inf")), INVAL), (dict(scale=2e38), INVAL), (dict(logits=None), INVAL),
    (dict(logp=None), INVAL), (dict(entropy=None), INVAL), (dict(peak=None), INVAL),
    (dict(log_sum=None), INVAL), (dict(top=3), INVAL), (dict(top=3, top_logp=8 * FAR), INVAL),
    (dict(ld=99), INVAL), (dict(logits=FAR + 2), INVAL), (dict(targets=2 * FAR + 4), INVAL),
    (dict(V=50_000, ld=50_000), INVAL),             # rows cut into parts: no workspace
    (dict(V=50_000, ld=50_000, ws=10 * FAR, ws_bytes=64), WORKSPACE),
    (dict(V=50_000, ld=50_000, ws=10 * FAR + 8, ws_bytes=1 << 18), INVAL),
    (dict(logp=FAR + 40), INVAL), (dict(entropy=3 * FAR + 4), INVAL), (dict(peak=2 * FAR), INVAL),
    (dict(dev_err=6 * FAR), INVAL), (dict(N=0), OK), (dict(N=0, logits=None), OK)])
def test_token_logprobs_refusals(c, kw, code):
    assert c.logprobs(**kw) == code


def test_token_logprobs_workspace(lz):
    f = lz.lib().lm_token_logprobs_workspace_bytes
    for bad in ((-1, 10, F32, 0), (1, 0, F32, 0), (1, 10, 2, 0), (1, 10, F32, 65), (1, 10, F32, -1)):
        assert f(*bad) == 0
    assert f(4096, 100_000, BF16, 20) == 0 and f(1, 2000, F32, 20) == 0  # many rows, short rows
    assert 0 < f(1, 100_000, BF16, 0) < f(1, 100_000, BF16, 20) < 1 << 16
    for N in (1, 2, 3, 100, 1000):
        for V in (9000, 50_000, 800_000, 1 << 30):
            assert f(N, V, BF16, 64) <= N * 128 * (12 + 4 * 64) + 16


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(idtype=3), UNSUPPORTED), (dict(N=-1), INVAL), (dict(V=0), INVAL),
    (dict(scale=0.0), INVAL), (dict(scale=NAN), INVAL), (dict(logits=None), INVAL),
    (dict(peak=None), INVAL), (dict(log_sum=None), INVAL), (dict(out=None), INVAL),
    (dict(targets=None), INVAL), (dict(dentropy=8 * FAR, entropy=None), INVAL),
    (dict(ld=99), INVAL), (dict(ld_out=99), INVAL), (dict(out=FAR, ld_out=101), INVAL),
    (dict(out=FAR + 4), INVAL), (dict(out=5 * FAR - 8), INVAL), (dict(dlogp=5 * FAR + 2), INVAL),
    (dict(N=(1 << 31) - 1, V=1 << 30, ld=1 << 31, ld_out=1 << 31, out=1 << 63), UNSUPPORTED), (dict(V=(1 << 30) + 1, ld=1 << 31, ld_out=1 << 31), UNSUPPORTED),
    (dict(N=0), OK)])
def test_token_logprobs_grad_refusals(c, kw, code):
    assert c.logprobs_grad(**kw) == code


def test_tensors_on_the_cpu_are_refused(lz):
    import torch
    x, v = torch.zeros(4, 8), torch.zeros(4)
    for f in (lambda: lz.dropout(x, 0.5, 1), lambda: lz.layer_norm(x), lambda: lz.token_logprobs(x),
              lambda: lz.layer_norm_grad(x, x, v, v), lambda: lz.token_logprobs_grad(x, None, v, v)):
        with pytest.raises(lz.LmError):
            f()


def test_tensors_that_require_grad_are_refused(lz):
    import torch
    x = torch.zeros(4, 8, requires_grad=True)
    for f in (lambda: lz.dropout(x, 0.5, 1), lambda: lz.layer_norm(x), lambda: lz.token_logprobs(x)):
        with pytest.raises(lz.LmError, match="autograd"):
            f()


def test_rows_of_tensors(lz):
    import torch
    x = torch.zeros(2, 3, 4, 10)
    assert lz._matrix(x, "x") == (24, 10, 10) and lz._matrix(x[0, 0, 0], "x") == (1, 10, 10)
    assert lz._matrix(x[..., :7], "x") == (24, 7, 10) and lz._matrix(x[:, :, ::2, :3], "x") == (12, 3, 20)
    assert lz._matrix(x[1:, 1:2, :, 2:], "x") == (4, 8, 10) and lz._matrix(x[:0], "x")[0] == 0
    assert lz._matrix(x[..., :1], "x") == (24, 1, 10)
    for bad in (x[:, :2], x.transpose(1, 2), x.transpose(2, 3), x[..., ::2], torch.zeros(())):
        with pytest.raises(lz.LmError):
            lz._matrix(bad, "x")


def test_mask_words():
    """A quarter dropped: the share in all, in every column and every row, and no correlation
    between neighbours, between seeds, or between the halves of a word."""
    rows, D, p, z = 2048, 512, 0.25, 6.0
    k = [A.keep(rows, D, p, s)[0].astype(np.float64) - (1 - p) for s in (0, 1, 2, 3, 1 << 33)]
    var = p * (1 - p)
    for m in k:
        assert abs(m.mean()) < z * (var / m.size) ** 0.5
        assert np.abs(m.mean(0)).max() < z * (var / rows) ** 0.5
        assert np.abs(m.mean(1)).max() < z * (var / D) ** 0.5
    pairs = [(a, b) for i, a in enumerate(k) for b in k[:i]]
    for dr, dc in ((0, 1), (0, 2), (0, 4), (0, 8), (0, 64), (1, 0), (2, 0), (1, 1), (64, 0), (1024, 0)):
        pairs.append((k[0][dr:, dc:], k[0][:rows - dr, :D - dc]))
    for i, (a, b) in enumerate(pairs):
        assert abs((a * b).mean()) < z * var / a.size ** 0.5, i
    for q in (0.0, 1.0):
        kept, c = A.keep(3, 5, q, 1)
        assert kept.all() == (q == 0) and kept.any() == (q == 0) and c == (1.0 if q == 0 else 0.0)


def test_reference_gradients_by_differences():
    """The 64-bit gradients that the GPU tests compare with, against differences of the 64-bit
    forward forms."""
    rng = np.random.default_rng(5)
    rows, D, step = 4, 13, 1e-5
    x, add, dy = (rng.standard_normal((rows, D)) for _ in range(3))
    w, b = rng.standard_normal(D), rng.standard_normal(D)

    def forward(x, add, w, b):
        r = A.norm(x, w, b, 1e-5, 0.25, 3, add)
        return (r["y"][0] * dy).sum()
    r = A.norm(x, w, b, 1e-5, 0.25, 3, add)
    g = A.norm_grad(dy, r["h"][0], r["mean"][0], r["rstd"][0], w, None, 0.25, 3)
    for k, name in enumerate(("dx", "dh", "dweight", "dbias")):
        args = [x, add, w, b]
        v = rng.standard_normal(args[k].shape)
        ends = [forward(*[a + s * step * v if i == k else a for i, a in enumerate(args)])
                for s in (1, -1)]
        d = (ends[0] - ends[1]) / (2 * step)
        assert abs(d - (g[name][0] * v).sum()) < 1e-7 * max(1.0, abs(d)), name
    z, t = rng.standard_normal((rows, D)) * 2, rng.integers(0, D, rows)
    t[1] = -100
    a, e = rng.standard_normal(rows), rng.standard_normal(rows)

    def value(z):
        r = A.logprobs(z, t, 1.3)
        return (r["logp"][0] * a).sum() + (r["entropy"][0] * e).sum()
    r = A.logprobs(z, t, 1.3)
    dz, _ = A.logprobs_grad(z, t, r["peak"][0], r["log_sum"][0], 1.3, a, r["entropy"][0], e)
    v = rng.standard_normal(z.shape)
    d = (value(z + step * v) - value(z - step * v)) / (2 * step)
    assert abs(d - (dz * v).sum()) < 1e-7 * max(1.0, abs(d))
