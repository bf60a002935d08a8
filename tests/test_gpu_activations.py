"""Dropout, layer norm and token log probabilities on the GPU against their definitions
in 64 bits, at the sizes, strides and masks where they can go wrong."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import activations_ref as A  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lmzipf


def wide(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, tol, what, dtype=None):
    """got within tol of ref (and of its rounding to dtype); infinities and NaN alike."""
    got = wide(got) if isinstance(got, torch.Tensor) else got
    with np.errstate(invalid="ignore"):
        tol = tol + (A.rounded(ref, dtype) if dtype is not None else A.TINY)
        same = (got == ref) | (np.isnan(got) & np.isnan(ref))
        ok = same | (np.abs(got - ref) <= tol)
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError(f"{what}: {(~ok).sum()} of {ok.size} off, at {i} got {got[i]!r},"
                             f" not {ref[i]!r} within {np.broadcast_to(tol, ok.shape)[i]:.3g}")


def rows_of(gen, rows, D, dtype, std=1.0, shift=0.0, gap=0, off=0):
    """rows x D values, `gap` elements between rows, the first `off` elements into its memory."""
    ld = D + gap
    flat = torch.full((off + rows * ld + 8,), NAN, dtype=dtype, device=DEV)
    t = flat[off:off + rows * ld].view(rows, ld)[:, :D]
    t.copy_(torch.randn(rows, D, generator=gen, device=DEV) * std + shift)
    return t


def gen_of(*key):
    seed = 1
    for k in key:
        seed = (seed * 1_000_003 + hash(str(k)) % 1 + sum(map(ord, str(k)))) % (2 ** 31)
    return torch.Generator(device=DEV).manual_seed(seed)


# rows, D, gap, off: from one value to the widest row; odd sizes, gaps and starts
SHAPES = [(1, 1, 0, 0), (3, 2, 1, 1), (5, 3, 0, 0), (2, 7, 2, 3), (9, 8, 0, 0), (1, 9, 0, 1),
          (33, 31, 0, 0), (70, 64, 1, 0), (6, 65, 0, 5), (4, 127, 3, 0), (131, 130, 0, 0),
          (17, 517, 0, 0), (20, 650, 6, 2), (7, 1025, 0, 1), (5, 2048, 0, 0), (3, 2049, 1, 0),
          (1, 4100, 0, 0), (2, 8191, 0, 0), (3, 16384, 8, 0), (700, 96, 0, 0)]


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("rows,D,gap,off", SHAPES + [(2, 40_001, 0, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout(lz, rows, D, gap, off, dtype):
    gen = gen_of("dropout", rows, D, dtype)
    x = rows_of(gen, rows, D, dtype, gap=gap, off=off)
    add = rows_of(gen, rows, D, dtype, 2.0, gap=2 * gap, off=off)
    for p, seed, a in ((0.0, 1, None), (0.1, 2, None), (0.5, 3, add), (0.3, -5, add), (1.0, 7, add),
                       (0.75, 2 ** 63 + 9, None)):
        got = lz.dropout(x, p, seed, add=a)
        ref, tol = A.dropout(wide(x), p, seed % 2 ** 64, None if a is None else wide(a))
        close(got, ref, tol, f"p {p}", dtype)
        assert got.shape == x.shape and got.dtype == dtype and got.is_contiguous()


def test_dropout_shares_and_independence(lz):
    """What is kept is the share that is asked for, in every column and row, and the masks of
    two seeds, neighbouring columns and neighbouring rows have nothing to do with each other."""
    rows, D, p = 4096, 1024, 0.25
    x = torch.ones(rows, D, device=DEV)
    k = [(lz.dropout(x, p, s) != 0).double() for s in (1, 2, 2 ** 40 + 1)]
    n = rows * D
    z = 6.0  # standard deviations
    for m in k:
        assert abs(float(m.mean()) - (1 - p)) < z * (p * (1 - p) / n) ** 0.5
        for line in (m.mean(0), m.mean(1)):
            assert float((line - (1 - p)).abs().max()) < z * (p * (1 - p) / 1024) ** 0.5
    def corr(a, b):
        return abs(float(((a - (1 - p)) * (b - (1 - p))).mean())) / (p * (1 - p))
    pairs = [(k[0], k[1]), (k[0], k[2]), (k[0][:, 1:], k[0][:, :-1]), (k[0][:, 2:], k[0][:, :-2]),
             (k[0][1:], k[0][:-1]), (k[0][1:, 1:], k[0][:-1, :-1]), (k[0][:, 4:], k[0][:, :-4])]
    for i, (a, b) in enumerate(pairs):
        assert corr(a, b) < z / a.numel() ** 0.5, i


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropped_values_are_zero(lz, dtype):
    """Infinities and NaN in dropped places are zeros, in kept ones they stay."""
    x = torch.full((64, 33), NAN, dtype=dtype, device=DEV)
    x[::2] = INF
    kept, _ = A.keep(64, 33, 0.5, 11)
    got = wide(lz.dropout(x, 0.5, 11))
    assert (got[~kept] == 0).all()
    assert np.isinf(got[::2][kept[::2]]).all() and np.isnan(got[1::2][kept[1::2]]).all()
    assert (wide(lz.dropout(x, 1.0, 11)) == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [3, 8, 65, 650, 2049])
def test_dropout_in_place(lz, dtype, D):
    gen = gen_of("in place", D, dtype)
    x, add = (rows_of(gen, 37, D, dtype, gap=3, off=1) for _ in range(2))
    want, plain = lz.dropout(x, 0.3, 5, add=add), lz.dropout(x, 0.3, 5)
    a, b = rows_of(gen, 37, D, dtype, gap=3, off=1), rows_of(gen, 37, D, dtype, gap=3, off=1)
    a.copy_(x)
    b.copy_(add)
    assert lz.dropout(x, 0.3, 5, add=b, out=b) is b and torch.equal(b, want)
    assert torch.equal(lz.dropout(a, 0.3, 5, out=a), plain)
    base = x._base if x._base is not None else x
    assert torch.isnan(base[-8:]).all()


def test_dropout_views_and_words_past_32_bits(lz):
    """Halves of one matrix; more than 2^32 words: the last rows' mask is that of their numbers."""
    both = torch.randn(50, 128, device=DEV)
    left, right = both[:, :64], both[:, 64:]
    want = lz.dropout(left.clone(), 0.5, 1)
    lz.dropout(left, 0.5, 1, out=right)
    assert torch.equal(right, want)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    rows, D = (1 << 23) + 7, 1026  # 513 words a row
    x = torch.ones(rows, D, dtype=BF16, device=DEV)
    lz.dropout(x, 0.5, 3, out=x)
    import moments_ref as M
    for r in (0, (1 << 23) - 50_000, (1 << 32) // 513, (1 << 32) // 513 + 1, rows - 1):
        w = M.words(np.arange(r * 513, (r + 1) * 513, dtype=np.uint64), 3)
        bits = np.stack((w & np.uint32(0xFFFF), w >> np.uint32(16)), 1).reshape(-1)
        assert np.array_equal(wide(x[r]), np.where(bits >= 32768, 2.0, 0.0)), r


def test_dropout_gradient_by_differences(lz):
    """The same call on dout is the gradient: the forward is linear, so a difference of two
    outputs is the gradient's product with the step, up to the roundings of powers of two."""
    gen = gen_of("differences")
    x, dout = (rows_of(gen, 9, 33, F32) for _ in range(2))
    dx = lz.dropout(dout, 0.5, 21)
    for i, j in ((0, 0), (3, 32), (8, 17), (5, 5)):
        up, down = x.clone(), x.clone()
        up[i, j] += 0.5
        down[i, j] -= 0.5
        step = wide(up[i, j] - down[i, j])
        d = ((wide(lz.dropout(up, 0.5, 21)) - wide(lz.dropout(down, 0.5, 21))) * wide(dout)).sum()
        assert abs(d - step * wide(dx)[i, j]) <= 8 * A.U * abs(wide(dout)[i, j]) * 8


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
def params(gen, D):
    return (torch.randn(D, generator=gen, device=DEV) * 0.3 + 1,
            torch.randn(D, generator=gen, device=DEV) * 0.2)


@pytest.mark.parametrize("rows,D,gap,off", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm(lz, rows, D, gap, off, dtype):
    gen = gen_of("norm", rows, D, dtype)
    x = rows_of(gen, rows, D, dtype, 1.5, 0.7, gap, off)
    add = rows_of(gen, rows, D, dtype, 2.0, -3.0, 2 * gap, off)
    w, b = params(gen, D)
    for weight, bias, a, p, eps in ((w, b, None, 0.0, 1e-5), (None, None, add, 0.0, 1e-6),
                                    (w, None, add, 0.2, 1e-5), (None, b, None, 0.5, 1e-3)):
        r = lz.layer_norm(x, weight, bias, eps=eps, add=a, p=p, seed=9)
        none = lambda t: None if t is None else wide(t)  # noqa: E731
        ref = A.norm(wide(x), none(weight), none(bias), eps, p, 9, none(a))
        for name in ("mean", "rstd"):
            close(getattr(r, name), *ref[name], name)
        close(r.y, *ref["y"], "y", dtype)
        if a is None and p == 0:
            assert r.h is x
        else:
            close(r.h, *ref["h"], "h", dtype)
        assert r.mean.shape == (rows,) and r.y.shape == x.shape


@pytest.mark.parametrize("rows,D,gap,off", SHAPES + [(5003, 40, 0, 0), (1500, 300, 0, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_grad(lz, rows, D, gap, off, dtype):
    gen = gen_of("norm grad", rows, D, dtype)
    h = rows_of(gen, rows, D, dtype, 1.5, 0.7, gap, off)
    dy = rows_of(gen, rows, D, dtype, 1.0, 0.1, 0, off)
    add = rows_of(gen, rows, D, dtype, 1.0, 0.0, gap, 0)
    w, _ = params(gen, D)
    s = lz.layer_norm(h, eps=1e-3)
    for weight, a, p in ((w, None, 0.0), (None, add, 0.0), (w, add, 0.3)):
        r = lz.layer_norm_grad(dy, h, s.mean, s.rstd, weight, add=a, p=p, seed=5, bias=True)
        none = lambda t: None if t is None else wide(t)  # noqa: E731
        ref = A.norm_grad(wide(dy), wide(h), wide(s.mean), wide(s.rstd), none(weight), none(a), p, 5)
        close(r.dh, *ref["dh"], "dh", dtype)
        close(r.dbias, *ref["dbias"], "dbias")
        if weight is None:
            assert r.dweight is None
        else:
            close(r.dweight, *ref["dweight"], "dweight")
        if p > 0:
            close(r.dx, *ref["dx"], "dx", dtype)
        else:
            assert r.dx is r.dh


# Rows enough for a wave of their own each, and for every workgroup to have several turns
MANY = [(70_001, 40), (8300, 300), (4200, 517), (2100, 1025), (2100, 2048), (1100, 4100),
        (1030, 8191), (1026, 16384)]
# Rows between few and many: on both sides of where the forms of both passes change
BETWEEN = [(1024, 30), (1025, 30), (20_000, 3), (33_000, 3), (70_001, 3), (1024, 300), (3492, 300),
           (3493, 300), (1014, 517), (1015, 517), (255, 1025), (256, 1025), (1024, 1025),
           (128, 2048), (129, 2048), (1, 2048), (63, 4100), (64, 4100), (33, 8191), (16, 16384),
           (17, 16384), (600, 16384), (257, 2048), (511, 1025), (128, 4096), (32, 16384),
           (33, 16384), (260, 9001)]


@pytest.mark.parametrize("rows,D", MANY + BETWEEN)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_of_many_rows(lz, rows, D, dtype):
    gen = gen_of("many", rows, D, dtype)
    x, add = rows_of(gen, rows, D, dtype, 1.5, 0.7), rows_of(gen, rows, D, dtype, 2.0, -1.0)
    w, b = params(gen, D)
    r = lz.layer_norm(x, w, b, add=add, p=0.2, seed=9)
    ref = A.norm(wide(x), wide(w), wide(b), 1e-5, 0.2, 9, wide(add))
    for name, dt in (("mean", None), ("rstd", None), ("y", dtype), ("h", dtype)):
        close(getattr(r, name), *ref[name], name, dt)
    g = lz.layer_norm_grad(add, r.h, r.mean, r.rstd, w, add=x, p=0.2, seed=9)
    ref = A.norm_grad(wide(add), wide(r.h), wide(r.mean), wide(r.rstd), wide(w), wide(x), 0.2, 9)
    for name, dt in (("dh", dtype), ("dx", dtype), ("dweight", None), ("dbias", None)):
        close(getattr(g, name), *ref[name], name, dt)


def test_results_of_tens_of_megabytes(lz):
    """Results that the caches hold in part (32 to 256 MiB): the same numbers."""
    rows, D = 8300, 1025
    gen = gen_of("cached")
    x, dy = rows_of(gen, rows, D, F32), rows_of(gen, rows, D, F32)
    ref, tol = A.dropout(wide(x), 0.3, 2)
    close(lz.dropout(x, 0.3, 2), ref, tol, "dropout")
    r = lz.layer_norm(x)
    ref = A.norm(wide(x), None, None, 1e-5)
    close(r.y, *ref["y"], "y")
    g = lz.layer_norm_grad(dy, x, r.mean, r.rstd)
    close(g.dh, *A.norm_grad(wide(dy), wide(x), wide(r.mean), wide(r.rstd), None)["dh"], "dh")
    t = torch.randint(0, D, (rows,), generator=gen, device=DEV)
    s = lz.token_logprobs(x, t)
    ref, tol = A.logprobs_grad(wide(x), t.cpu().numpy(), wide(s.peak), wide(s.log_sum), 1.0,
                               wide(s.logp))
    close(lz.token_logprobs_grad(x, t, s.peak, s.log_sum, s.logp), ref, tol, "dlogits")


def test_layer_norm_grad_against_autograd_and_differences(lz):
    """fp32 against torch's autograd of the definition in 64 bits, and against differences of
    it: both through dropout, the residual sum and the norm."""
    rows, D, p, seed, eps = 6, 37, 0.25, 3, 1e-5
    gen = gen_of("autograd")
    x, add, dy, past = (rows_of(gen, rows, D, F32) for _ in range(4))
    w, b = params(gen, D)
    kept, c = A.keep(rows, D, p, seed)
    factor = torch.from_numpy(kept * c)
    leaf = [t.detach().double().cpu().requires_grad_() for t in (x, add, w, b)]

    def loss(x, add, w, b):
        h = add + x * factor
        d = h - h.mean(1, keepdim=True)
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + eps) * w + b
        return (y * dy.double().cpu()).sum() + (h * past.double().cpu()).sum()
    want = torch.autograd.grad(loss(*leaf), leaf)
    f = lz.layer_norm(x, w, b, eps=eps, add=add, p=p, seed=seed)
    r = lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, w, add=past, p=p, seed=seed)
    ref = A.norm_grad(wide(dy), wide(f.h), wide(f.mean), wide(f.rstd), wide(w), wide(past), p, seed)
    # the statistics' and h's roundings reach the gradient: U of each, times what it is worth
    slack = 2.0 ** -18
    got = (r.dx, r.dh, r.dweight, r.dbias)
    for g, t, name in zip(got, want, ("dx", "dh", "dweight", "dbias")):
        close(g, t.numpy(), ref[name][1] + slack * max(1.0, float(t.abs().max())), name)
    step = 1e-4
    for k, (g, name) in enumerate(zip(got, ("dx", "dh", "dweight", "dbias"))):
        v = torch.randn(leaf[k].shape, generator=torch.Generator().manual_seed(k), dtype=torch.float64)
        with torch.no_grad():
            ends = [loss(*[t + s * step * v if i == k else t for i, t in enumerate(leaf)])
                    for s in (1, -1)]
        d = float(ends[0] - ends[1]) / (2 * step)
        assert abs(d - float((torch.from_numpy(wide(g)) * v).sum())) < 1e-3 * max(1.0, abs(d)), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_rows_of_all_kinds(lz, dtype):
    """Equal values (the variance is 0), values far from zero, infinities and NaN: every row
    has its own result, and those that are not numbers stay in their row."""
    D = 300
    x = torch.randn(9, D, generator=gen_of("kinds"), device=DEV).to(dtype)
    x[0] = 5.0
    x[1] = 0.0
    x[2] += 256.0
    x[3, 7] = NAN
    x[4, 100] = INF
    x[5, 5] = -INF
    x[6] = x[6] * 1e-20
    w, b = params(gen_of("kinds2"), D)
    r = lz.layer_norm(x, w, b, eps=1e-5)
    with np.errstate(invalid="ignore"):
        ref = A.norm(wide(x), wide(w), wide(b), 1e-5)
    live = [0, 1, 2, 6, 7, 8]
    for name, dt in (("y", dtype), ("mean", None), ("rstd", None)):
        close(wide(getattr(r, name))[live], ref[name][0][live], ref[name][1][live], name, dt)
    assert torch.isnan(r.y[3:6]).all() and torch.isfinite(r.y[live]).all()
    assert torch.equal(r.y[1], b.to(dtype))
    g = lz.layer_norm_grad(x, x, r.mean, r.rstd, w)
    assert torch.isfinite(g.dh[live]).all() and torch.isnan(g.dh[3:6]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [5, 64, 517, 2048, 5000])
def test_layer_norm_in_place(lz, dtype, D):
    """The residual stream updated in place, y over x; the gradients over their sources."""
    gen = gen_of("norm in place", D, dtype)
    x, add, dy = (rows_of(gen, 41, D, dtype, gap=2, off=3) for _ in range(3))
    w, b = params(gen, D)
    want = lz.layer_norm(x, w, b, add=add, p=0.2, seed=4)
    grads = lz.layer_norm_grad(dy, want.h, want.mean, want.rstd, w, add=add, p=0.2, seed=4)
    x2, add2, dy2, past = (rows_of(gen, 41, D, dtype, gap=2, off=3) for _ in range(4))
    for t, s in ((x2, x), (add2, add), (dy2, dy), (past, add)):
        t.copy_(s)
    r = lz.layer_norm(x2, w, b, add=add2, p=0.2, seed=4, out=x2, sum_out=add2)
    assert r.y is x2 and r.h is add2
    for got, ref in zip(r, want):
        assert torch.equal(got, ref)
    g = lz.layer_norm_grad(dy2, add2, r.mean, r.rstd, w, add=past, p=0.2, seed=4, out=past, dx=dy2)
    assert g.dh is past and g.dx is dy2
    for got, ref in zip(g, grads):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("rows,D", [(1, 77), (5, 77), (130, 77), (300, 77), (5000, 77), (3, 5),
                                    (1, 2048), (2, 1025), (1, 9001), (40, 9001)])
def test_layer_norm_grad_accumulates(lz, rows, D):
    gen = gen_of("accumulate", rows)
    h, dy = (rows_of(gen, rows, D, BF16) for _ in range(2))
    w, _ = params(gen, D)
    s = lz.layer_norm(h)
    one = lz.layer_norm_grad(dy, h, s.mean, s.rstd, w)
    dw, db = torch.full((D,), 2.0, device=DEV), torch.full((D,), -1.0, device=DEV)
    two = lz.layer_norm_grad(dy, h, s.mean, s.rstd, w, dweight=dw, dbias=db, accumulate=True)
    assert two.dweight is dw and torch.equal(dw, one.dweight + 2.0)
    assert torch.equal(db, one.dbias - 1.0)
    none = lz.layer_norm_grad(dy[:0], h[:0], s.mean[:0], s.rstd[:0], w, dweight=dw, dbias=db)
    assert not dw.any() and not db.any() and none.dh.shape == (0, D)
    only = lz.layer_norm_grad(dy, h, s.mean, s.rstd, w, bias=False)
    assert only.dbias is None and torch.equal(only.dweight, one.dweight)


# ---------------------------------------------------------------------------
# Token log probabilities
# ---------------------------------------------------------------------------
def check_logprobs(lz, x, targets, scale, top, ws=None):
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = lz.token_logprobs(x, targets, scale=scale, top=top, dev_err=err, ws=ws)
    lz.check(err)
    s = float(np.float32(scale))
    ref = A.logprobs(wide(x), None if targets is None else targets.cpu().numpy().astype(np.int64), s,
                     top)
    for name in ("peak", "log_sum", "entropy") + (() if targets is None else ("logp",)):
        close(getattr(r, name), *ref[name], name)
    if top:
        assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"][0])
        close(r.top_logp, *ref["top_logp"], "top_logp")
    else:
        assert r.top_ids is None and r.top_logp is None
    return r, ref


LOGITS = [(1, 1, 0, 0), (3, 2, 0, 0), (5, 3, 1, 1), (2, 7, 0, 0), (4, 8, 0, 0), (9, 98, 0, 0),
          (3, 100, 5, 1), (2, 513, 0, 0), (7, 2047, 1, 0), (2, 2049, 0, 3), (1, 9999, 0, 0),
          (5, 20_001, 0, 0), (1, 100_000, 0, 0), (3, 70_003, 1, 1), (600, 333, 0, 0),
          (1030, 4099, 0, 0)]


@pytest.mark.parametrize("N,V,gap,off", LOGITS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs(lz, N, V, gap, off, dtype):
    gen = gen_of("logp", N, V, dtype)
    x = rows_of(gen, N, V, dtype, 2.5, -1.0, gap, off)
    t = torch.randint(0, V, (N,), generator=gen, device=DEV)
    if N > 2:
        t[1] = -100
    for targets, scale, top in ((t, 1.0, 0), (t.int(), 1 / 0.7, 5), (None, 0.25, 20), (t, 3.0, 64)):
        check_logprobs(lz, x, targets, scale, top)


@pytest.mark.parametrize("N,V,gap,off", LOGITS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_grad(lz, N, V, gap, off, dtype):
    gen = gen_of("logp grad", N, V, dtype)
    x = rows_of(gen, N, V, dtype, 2.5, -1.0, gap, off)
    t = torch.randint(0, V, (N,), generator=gen, device=DEV)
    if N > 2:
        t[1] = -100
    dlogp, dent = (torch.randn(N, generator=gen, device=DEV) for _ in range(2))
    r = lz.token_logprobs(x, t, scale=0.8)
    s = float(np.float32(0.8))
    for targets, a, b in ((t, dlogp, None), (None, None, dent), (t.int(), dlogp, dent)):
        got = lz.token_logprobs_grad(x, targets, r.peak, r.log_sum, dlogp=a, entropy=r.entropy,
                                     dentropy=b, scale=0.8)
        ref, tol = A.logprobs_grad(
            wide(x), None if targets is None else t.cpu().numpy(), wide(r.peak), wide(r.log_sum), s,
            None if a is None else wide(a), wide(r.entropy), None if b is None else wide(b))
        close(got, ref, tol, "dlogits", dtype)


def masked_rows(gen, V, dtype):
    """Rows whose masks leave everything, a third, one word, none; masks of the type's lowest
    value; equal logits; infinities and NaN."""
    x = torch.randn(12, V, generator=gen, device=DEV) * 2
    x[1, torch.rand(V, generator=gen, device=DEV) < 0.66] = -INF
    x[2] = -INF
    x[2, V // 2] = 3.0
    x[3] = -INF
    x = x.to(dtype)
    x[4] = torch.finfo(dtype).min
    x[5, : V // 2] = torch.finfo(dtype).min
    x[6] = 1.25
    x[7, V // 3] = NAN
    x[8, V - 1] = INF
    x[9] = -0.0
    x[9, V // 2:] = 0.0
    x[10] = torch.arange(V, device=DEV).to(dtype)  # ascending: every word beats those before it
    x[11, :-1] = torch.finfo(dtype).max
    return x


@pytest.mark.parametrize("V", [5, 98, 2500, 30_001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_masks(lz, V, dtype):
    x = masked_rows(gen_of("masks", V, dtype), V, dtype)
    N = len(x)
    t = torch.full((N,), V - 1, device=DEV)
    t[2] = V // 2
    live = [i for i in range(N) if i not in (7, 8)]
    for scale, top in ((1.0, 0), (1.0, 7), (0.5, 64)):
        r = lz.token_logprobs(x, t, scale=scale, top=top)
        ref = A.logprobs(wide(x[live]), t[live].cpu().numpy(), scale, top)
        for name in ("peak", "log_sum", "entropy", "logp") + (("top_logp",) if top else ()):
            close(wide(getattr(r, name))[live], *ref[name], name)
            assert torch.isnan(getattr(r, name)[7:9]).all(), name
        if top:
            assert np.array_equal(r.top_ids.cpu().numpy()[live], ref["top_ids"][0])
            assert (r.top_ids[7:9] == -1).all()
        # one call for each row: few rows are cut into parts
        for i in range(N):
            one = lz.token_logprobs(x[i:i + 1], t[i:i + 1], scale=scale, top=top)
            if i in live:
                ref1 = {k: (v[0][live.index(i)][None], None if v[1] is None else v[1][live.index(i)][None])
                        for k, v in ref.items()}
                for name in ("peak", "log_sum", "entropy", "logp") + (("top_logp",) if top else ()):
                    close(getattr(one, name), *ref1[name], (i, name))
                if top:
                    assert np.array_equal(one.top_ids.cpu().numpy(), ref1["top_ids"][0]), i
            else:
                assert torch.isnan(one.logp).all() and torch.isnan(one.log_sum).all()


@pytest.mark.parametrize("V", [5, 98, 2500])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_grad_masks(lz, V, dtype):
    """Masked words and empty rows get zeros; NaN stays in its row, and out of it where
    nothing depends on the row."""
    x = masked_rows(gen_of("grad masks", V, dtype), V, dtype)
    N = len(x)
    t = torch.full((N,), V - 1, device=DEV)
    t[2] = V // 2
    r = lz.token_logprobs(x, t)
    dlogp, dent = torch.linspace(-1, 1, N, device=DEV), torch.linspace(0.5, 2, N, device=DEV)
    live = [i for i in range(N) if i not in (7, 8)]
    for b in (None, dent):
        got = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, dlogp, r.entropy, b)
        ref, tol = A.logprobs_grad(wide(x[live]), t[live].cpu().numpy(), wide(r.peak)[live],
                                   wide(r.log_sum)[live], 1.0, wide(dlogp)[live],
                                   wide(r.entropy)[live], None if b is None else wide(b)[live])
        close(wide(got)[live], ref, tol, "dlogits", dtype)
        assert torch.isnan(got[7]).all()
        assert not got[3].any()
    t[7] = t[8] = -100
    dlogp[7] = dlogp[8] = NAN  # not used
    got = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, dlogp)
    assert not got[7:9].any() and torch.isfinite(got[live]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_far_from_zero(lz, dtype):
    """Rows 10,000 off zero: probabilities keep their digits."""
    gen = gen_of("far", dtype)
    x = (torch.randint(-8, 9, (4, 3000), generator=gen, device=DEV) * 64.0 + 16384.0).to(dtype)
    x[2:] -= 32768.0
    t = torch.randint(0, 3000, (4,), generator=gen, device=DEV)
    scale = 1 / 64
    r, _ = check_logprobs(lz, x, t, scale, 9)
    got = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, torch.ones(4, device=DEV), scale=scale)
    ref, tol = A.logprobs_grad(wide(x), t.cpu().numpy(), wide(r.peak), wide(r.log_sum), scale, np.ones(4))
    close(got, ref, tol, "dlogits", dtype)


@pytest.mark.parametrize("power", [0, 31, 100])
@pytest.mark.parametrize("size", [15, 19, 20, 22, 25, 31, 60])
@pytest.mark.parametrize("N,V", [(3, 500), (4, 9000), (2, 40_000)])
def test_token_logprobs_of_any_size(lz, power, size, N, V):
    """Rows around plus and minus 2^power whose exponents are around 2^size, and rows that hold
    both: neighbouring fp32 numbers count for what their difference is."""
    gen = gen_of("size", power, size, V)
    step = 2.0 ** (power - 23)
    x = torch.randint(-20, 21, (N, V), generator=gen, device=DEV) * step + 2.0 ** power
    x[1] *= -1
    if N > 2:
        x[2, ::2] *= -1
    x[0, : V // 2] -= 2.0 ** (power - 1)  # the first half is less, or nothing, beside the second
    t = torch.randint(V // 2, V, (N,), generator=gen, device=DEV)
    scale = 2.0 ** (size - power)
    r, _ = check_logprobs(lz, x, t, scale, 5)
    check_logprobs(lz, x, t, scale, 0)
    a = torch.ones(N, device=DEV)
    ref, tol = A.logprobs_grad(wide(x), t.cpu().numpy(), wide(r.peak), wide(r.log_sum), scale, wide(a),
                               wide(r.entropy), wide(a))
    close(lz.token_logprobs_grad(x, t, r.peak, r.log_sum, a, r.entropy, a, scale=scale), ref, tol,
          "dlogits")


def test_token_logprobs_ties(lz):
    """Equal logits: the lowest ids, also where more are equal than are kept as candidates, in
    rows that are cut into parts and rows that are not."""
    for N, V in ((1, 60_000), (1100, 3000), (2, 300)):
        x = torch.zeros(N, V, dtype=BF16, device=DEV)
        x[:, V // 2] = 1.0
        x[0, V - 1] = 2.0
        r = lz.token_logprobs(x, top=20)
        want = [V // 2] + list(range(19))
        if N > 1:
            assert r.top_ids[1].tolist() == want and (r.top_ids[1:] == r.top_ids[1]).all()
        assert r.top_ids[0].tolist() == [V - 1] + want[:-1]


def test_token_logprobs_grad_by_autograd_and_differences(lz):
    N, V, scale = 5, 41, 1.5
    gen = gen_of("logp autograd")
    x = rows_of(gen, N, V, F32, 2.0)
    t = torch.randint(0, V, (N,), generator=gen, device=DEV)
    dlogp, dent = (torch.randn(N, generator=gen, device=DEV) for _ in range(2))
    leaf = x.double().cpu().requires_grad_()

    def loss(z):
        l = torch.log_softmax(z * scale, 1)
        h = -(l.exp() * l).sum(1)
        return (l[torch.arange(N), t.cpu()] * dlogp.double().cpu() + h * dent.double().cpu()).sum()
    want, = torch.autograd.grad(loss(leaf), leaf)
    r = lz.token_logprobs(x, t, scale=scale)
    got = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, dlogp, r.entropy, dent, scale=scale)
    _, tol = A.logprobs_grad(wide(x), t.cpu().numpy(), wide(r.peak), wide(r.log_sum), scale, wide(dlogp),
                             wide(r.entropy), wide(dent))
    # log_sum's and the entropy's own roundings: a few U of each, times at most 2 scale |d|
    close(got, want.numpy(), tol + 64 * A.U * scale * 4, "dlogits")
    v = torch.randn(N, V, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    with torch.no_grad():
        d = float(loss(leaf + 1e-4 * v) - loss(leaf - 1e-4 * v)) / 2e-4
    assert abs(d - float((torch.from_numpy(wide(got)) * v).sum())) < 1e-4 * max(1.0, abs(d))


def test_token_logprobs_targets_out_of_range(lz):
    x = torch.randn(4, 50, device=DEV)
    t = torch.tensor([3, 50, -1, -100], device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = lz.token_logprobs(x, t, dev_err=err)
    assert int(err.item()) == lz.DEVERR_ID_RANGE
    assert torch.isnan(r.logp[1:3]).all() and float(r.logp[3]) == 0 and torch.isfinite(r.logp[0])
    g = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, torch.ones(4, device=DEV))
    assert torch.isnan(g[1:3]).all() and torch.isfinite(g[0]).all() and not g[3].any()
    other = lz.token_logprobs(x, t, ignore=-1)
    assert float(other.logp[2]) == 0 and torch.isnan(other.logp[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [6, 98, 2047, 20_001])
def test_token_logprobs_grad_in_place(lz, dtype, V):
    gen = gen_of("logp in place", V, dtype)
    x = rows_of(gen, 13, V, dtype, gap=1, off=1)
    t = torch.randint(0, V, (13,), generator=gen, device=DEV)
    r = lz.token_logprobs(x, t)
    a = torch.randn(13, generator=gen, device=DEV)
    want = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, a, r.entropy, a)
    assert lz.token_logprobs_grad(x, t, r.peak, r.log_sum, a, r.entropy, a, out=x) is x
    assert torch.equal(x, want)


def test_shapes_of_results(lz):
    """Leading dimensions are kept; empty batches are no error."""
    x = torch.randn(2, 3, 40, device=DEV)
    assert lz.dropout(x, 0.5, 1).shape == x.shape
    r = lz.layer_norm(x, add=x)
    assert r.y.shape == x.shape and r.mean.shape == (2, 3)
    t = torch.zeros(2, 3, dtype=torch.int64, device=DEV)
    s = lz.token_logprobs(x, t, top=4)
    assert s.logp.shape == s.entropy.shape == (2, 3) and s.top_ids.shape == (2, 3, 4)
    assert lz.token_logprobs_grad(x, t, s.peak, s.log_sum, s.logp).shape == x.shape
    part = x[:, :2]  # rows of 40, 40 and then 80 apart: not one distance
    for f in (lambda: lz.dropout(part, 0.5, 1), lambda: lz.layer_norm(part)):
        with pytest.raises(lz.LmError):
            f()
    one = x[0, 0]
    assert torch.equal(lz.layer_norm(one).y, r.y[0, 0] * 0 + lz.layer_norm(one[None]).y[0])
    for e in (x[:0], x[:, :0]):
        assert lz.dropout(e, 0.5, 1).shape == e.shape and lz.layer_norm(e).y.shape == e.shape
        assert lz.token_logprobs(e, top=3).top_ids.shape == (*e.shape[:-1], 3)
    assert lz.dropout(x[..., :0], 0.5, 1).numel() == 0


def test_repeated_calls_give_the_same_bits(lz):
    gen = gen_of("bits")
    h, dy = (rows_of(gen, 3000, 700, BF16) for _ in range(2))
    w, b = params(gen, 700)
    s = lz.layer_norm(h, w, b)
    x = rows_of(gen, 3, 50_000, F32)
    first = None
    for _ in range(3):
        g = lz.layer_norm_grad(dy, h, s.mean, s.rstd, w, p=0.1, seed=1)
        r = lz.token_logprobs(x, top=8)
        got = [*g, *r[1:], *lz.layer_norm(h, w, b)]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, got))
        first = got
