"""GPU parity of the relative position bias and its gradient. The bias is held to
torch's own fp32 sum rounded once, bit for bit; the gradient to 64 bits, and bit
for bit where the summands are small whole numbers (their sums are exact in fp32,
so a lost or doubled element shows at any length)."""
import math
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import relbias_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
U32 = 2.0 ** -24
SHAPES = [(1, 1, 1, 1), (2, 3, 1, 17), (1, 2, 5, 3), (2, 1, 64, 512), (1, 2, 63, 511),
          (3, 2, 65, 513), (1, 4, 130, 1030), (2, 2, 700, 40), (1, 1, 1, 4097), (1, 1, 4097, 1),
          (5, 1, 9, 250), (1, 3, 257, 257)]


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lmzipf


def _of(mode, Lq, Lk, q_start, nb=32, far=128):
    """The bucket of every place (-1: masked), from whole numbers."""
    lo = -(Lq - 1) - q_start
    line = torch.tensor([R.bucket(r, nb, far, mode) for r in range(lo, Lk - q_start)], device=DEV)
    i, j = torch.arange(Lq, device=DEV), torch.arange(Lk, device=DEV)
    return line[j - i[:, None] + Lq - 1]


def _want(table, add, of):
    bias = table[of.clamp(min=0)].permute(2, 0, 1)
    x = bias if add is None else add.float() + bias
    return x.masked_fill(of < 0, -math.inf)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["both", "past", "causal"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rel_bias(lz, dtype, mode, shape):
    B, H, Lq, Lk = shape
    gen = torch.Generator(device=DEV).manual_seed(Lq + Lk)
    table = torch.randn(32, H, generator=gen, device=DEV)
    buckets = lz.rel_buckets(32, 128, mode)
    for q_start in sorted({0, Lk - Lq, 5}):
        of = _of(mode, Lq, Lk, q_start)
        got = lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start, dtype=dtype)
        assert torch.equal(got, _want(table, None, of).to(dtype)), q_start
        add = (torch.randn(B, H, Lq, Lk, generator=gen, device=DEV) * 3).to(dtype)
        want = _want(table, add, of).to(dtype)
        assert torch.equal(lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start, add=add), want)
        lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start, add=add, out=add)
        assert torch.equal(add, want), "in place"


@pytest.mark.parametrize("nb,far,mode", [(4, 3, "both"), (2, 2, "past"), (33, 100, "past"),
                                         (64, 777, "both"), (256, 5000, "both"),
                                         (256, 100_000, "causal"), (255, 1000, "past")])
def test_rel_bias_other_buckets(lz, nb, far, mode):
    H, Lq, Lk = 3, 90, 1500
    table = torch.randn(nb, H, device=DEV)
    buckets = lz.rel_buckets(nb, far, mode)
    for q_start in (0, 1000):
        of = _of(mode, Lq, Lk, q_start, nb, far)
        got = lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start)
        assert torch.equal(got, _want(table, None, of))
        dout = torch.randint(-3, 4, (2, H, Lq, Lk), device=DEV).float()
        assert torch.equal(lz.rel_bias_grad(dout, buckets, q_start=q_start),
                           _grad(dout, of, nb).float())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("start", [0, 1, 3])
def test_rel_bias_strides_and_what_lies_between(lz, dtype, start):
    """Views with gaps in every dimension, at odd addresses: only their elements change."""
    B, H, Lq, Lk, pad = 2, 3, 70, 150, 5
    big = torch.full((start + B * (H + 1) * (Lq + 2) * (Lk + pad),), 7.0, dtype=dtype, device=DEV)
    strides = ((H + 1) * (Lq + 2) * (Lk + pad), (Lq + 2) * (Lk + pad), Lk + pad, 1)
    out = big.as_strided((B, H, Lq, Lk), strides, start)
    add = torch.randn(H, B, Lq, Lk, device=DEV).to(dtype).transpose(0, 1)
    wide = torch.randn(32, H + 2, device=DEV)
    table = wide[:, :H]
    buckets = lz.rel_buckets(32, 128, "both")
    want = _want(table, add, _of("both", Lq, Lk, 0)).to(dtype)
    lz.rel_bias(table, buckets, Lq, Lk, add=add, out=out)
    assert torch.equal(out, want)
    mark = torch.zeros_like(big, dtype=torch.bool)
    mark.as_strided((B, H, Lq, Lk), strides, start).fill_(True)
    assert bool((big[~mark] == 7).all()), "written outside the view"
    # a batch that repeats one matrix, and the gradient of it
    one = add[:1].expand(4, H, Lq, Lk)
    got = lz.rel_bias(table, buckets, Lq, Lk, add=one)
    assert torch.equal(got, want[:1].expand(4, H, Lq, Lk))
    whole = torch.randint(-3, 4, (H, B, Lq, Lk), device=DEV).to(dtype).transpose(0, 1)
    out.copy_(whole)
    for x in (whole, out, whole[:1].expand(3, H, Lq, Lk)):
        assert torch.equal(lz.rel_bias_grad(x, buckets), _grad(x, _of("both", Lq, Lk, 0), 32).float())


def test_rel_bias_special_values(lz):
    """Masks of the lowest value, infinities and NaN in the scores: as torch adds them;
    masked places are -infinity whatever the scores hold, rows without keys wholly."""
    for dtype in (torch.float32, torch.bfloat16):
        table = torch.randn(32, 2, device=DEV)
        add = torch.randn(1, 2, 40, 30, device=DEV).to(dtype)
        add[0, 0, 3] = torch.finfo(dtype).min
        add[0, 0, 4] = -math.inf
        add[0, 1, 5] = math.nan
        add[0, 1, 0, 1:] = math.nan
        add[0, 1, 1, 2:] = math.inf
        for mode, q_start in (("both", 0), ("causal", 0), ("causal", -10)):
            of = _of(mode, 40, 30, q_start)
            got = lz.rel_bias(table, lz.rel_buckets(32, 128, mode), 40, 30, q_start=q_start, add=add)
            want = _want(table, add, of).to(dtype)
            assert torch.equal(got.isnan(), want.isnan())
            assert torch.equal(got.nan_to_num(), want.nan_to_num())
        assert bool((got[:, :, :10] == -math.inf).all())


def _grad(dout, of, nb):
    d = dout.double().sum(0) if dout.dim() == 4 else dout.double()
    out = torch.zeros(nb + 1, d.shape[0], dtype=torch.float64, device=DEV)
    for h in range(d.shape[0]):
        keep = of >= 0
        out[:, h].scatter_add_(0, of[keep], d[h][keep])
    return out[:nb]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["both", "past", "causal"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rel_bias_grad(lz, dtype, mode, shape):
    B, H, Lq, Lk = shape
    gen = torch.Generator(device=DEV).manual_seed(Lq * Lk)
    buckets = lz.rel_buckets(32, 128, mode)
    for q_start in sorted({0, Lk - Lq, 5}):
        of = _of(mode, Lq, Lk, q_start)
        whole = torch.randint(-3, 4, shape, generator=gen, device=DEV).to(dtype)
        got = lz.rel_bias_grad(whole, buckets, q_start=q_start)
        assert torch.equal(got, _grad(whole, of, 32).float()), q_start
        if B == 1:
            assert torch.equal(lz.rel_bias_grad(whole[0], buckets, q_start=q_start), got)
        x = torch.randn(shape, generator=gen, device=DEV).to(dtype)
        old = torch.randn(32, H, generator=gen, device=DEV)
        got = lz.rel_bias_grad(x, buckets, q_start=q_start, out=old.clone(), accumulate=True)
        # any order of n sums is off by at most (n - 1) half steps of the magnitudes' sum; the
        # longest chain of additions here is under 1024
        n = min(1024, B * Lq * Lk + 2)
        most = n * U32 * (_grad(x.abs(), of, 32) + old.abs().double()) + 1e-45
        assert bool(((got.double() - (_grad(x, of, 32) + old.double())).abs() <= most).all())


@pytest.mark.parametrize("dtype,shape", [(torch.bfloat16, (4, 8, 1024, 1024)),
                                         (torch.float32, (2, 4, 1001, 2047)),
                                         (torch.bfloat16, (1, 1, 5000, 6001)),
                                         (torch.bfloat16, (40, 2, 128, 128))])
def test_rel_bias_grad_large(lz, dtype, shape):
    B, H, Lq, Lk = shape
    gen = torch.Generator(device=DEV).manual_seed(5)
    for mode in ("both", "causal"):
        of = _of(mode, Lq, Lk, Lk - Lq)
        buckets = lz.rel_buckets(32, 128, mode)
        # at most 2^24 ones in absolute sum: exact in any order
        x = torch.randint(-1, 2, shape, generator=gen, device=DEV)
        x = x * (torch.rand(shape, generator=gen, device=DEV) < 2.0 ** 23 / (B * Lq * Lk))
        got = lz.rel_bias_grad(x.to(dtype), buckets, q_start=Lk - Lq)
        assert torch.equal(got, _grad(x, of, 32).float()), mode
        again = lz.rel_bias_grad(x.to(dtype), buckets, q_start=Lk - Lq)
        assert torch.equal(got, again)


def test_rel_bias_grad_is_the_derivative(lz):
    """Against differences: the bias is linear in the table, so the sum of its product
    with w moves by the gradient's entry times the step, exactly but for rounding."""
    H, Lq, Lk = 2, 30, 45
    buckets = lz.rel_buckets(16, 20, "both")
    w = torch.randint(-2, 3, (1, H, Lq, Lk), device=DEV).float()
    grad = lz.rel_bias_grad(w, buckets, q_start=3)
    zero = torch.zeros(16, H, device=DEV)
    for n in range(16):
        for h in range(H):
            e = zero.clone()
            e[n, h] = 1.0
            moved = (lz.rel_bias(e, buckets, Lq, Lk, q_start=3).double() * w[0]).sum()
            assert float(moved) == float(grad[n, h]), (n, h)


def test_rel_bias_grad_masked_places_may_hold_anything(lz):
    H, L = 2, 300
    buckets = lz.rel_buckets(32, 128, "causal")
    of = _of("causal", L, L, 0)
    x = torch.randint(-3, 4, (1, H, L, L), device=DEV).float()
    want = lz.rel_bias_grad(x, buckets)
    for junk in (math.nan, math.inf, -math.inf):
        assert torch.equal(lz.rel_bias_grad(x.masked_fill(of < 0, junk), buckets), want)
    x[0, 0, 200, 100] = math.nan  # a visible one shows, in its bucket and head alone
    got = lz.rel_bias_grad(x, buckets)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[int(of[200, 100]), 0] = True
    assert torch.equal(got.isnan(), hit) and torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rel_bias_offsets_past_32_bits(lz, dtype):
    """Batch, head and row strides that put elements more than 2^32 apart."""
    need = 3 * (1 << 32)
    if torch.cuda.mem_get_info()[0] < need * 4 + (4 << 30):
        pytest.skip("needs 56 GB")
    big = torch.empty(need, dtype=dtype, device=DEV)
    buckets, table = lz.rel_buckets(32, 128, "both"), torch.randn(32, 2, device=DEV)
    for strides in (((1 << 32) + 64, 70_000, 128, 1), (9_000, (1 << 32) + 32, 128, 1),
                    (9_000_000, 128, (1 << 32) // 50 + 3, 1)):
        x = big.as_strided((2, 2, 60, 100), strides, 5)
        whole = torch.randint(-3, 4, x.shape, device=DEV).to(dtype)
        x.copy_(whole)
        of = _of("both", 60, 100, 7)
        assert torch.equal(lz.rel_bias_grad(x, buckets, q_start=7), _grad(whole, of, 32).float())
        lz.rel_bias(table, buckets, 60, 100, q_start=7, add=x, out=x)
        assert torch.equal(x, _want(table, whole, of).to(dtype))


@pytest.mark.parametrize("q_start", [-(1 << 30), 1 << 30])
@pytest.mark.parametrize("mode", ["both", "past", "causal"])
def test_rel_bias_far_starts(lz, mode, q_start):
    """Positions at the ends of the range: every key far before or far behind the query."""
    H, Lq, Lk = 2, 20, 70
    buckets, table = lz.rel_buckets(32, 128, mode), torch.randn(32, H, device=DEV)
    row = R.bucket(-q_start, 32, 128, mode)
    want = torch.full((H, Lq, Lk), -math.inf, device=DEV) if row < 0 else \
        table[row][:, None, None].expand(H, Lq, Lk)
    assert torch.equal(lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start), want)
    x = torch.randint(-3, 4, (1, H, Lq, Lk), device=DEV).float()
    grad = torch.zeros(32, H, device=DEV)
    if row >= 0:
        grad[row] = x.sum((0, 2, 3))
    assert torch.equal(lz.rel_bias_grad(x, buckets, q_start=q_start), grad)


def test_rel_bias_long_rows(lz):
    """One query against a long cache, and a long column of queries against one key."""
    buckets = lz.rel_buckets(32, 128, "past")
    table = torch.randn(32, 1, device=DEV)
    n = (1 << 20) + 3
    line = torch.arange(n, device=DEV)
    for Lq, Lk, q_start in ((1, n, n - 1), (n, 1, 0)):
        d = (n - 1 - line) if Lq == 1 else line
        small = torch.tensor([R.bucket(-i, 32, 128, "past") for i in range(200)], device=DEV)
        of = small[d.clamp(max=199)].view(Lq, Lk)
        got = lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start, dtype=torch.bfloat16)
        assert torch.equal(got, table[of].permute(2, 0, 1).bfloat16())
        x = torch.randint(-3, 4, (1, 1, Lq, Lk), device=DEV).bfloat16()
        assert torch.equal(lz.rel_bias_grad(x, buckets, q_start=q_start),
                           _grad(x, of, 32).float())


def test_rel_bias_grad_on_two_streams_at_once(lz):
    """Calls without a workspace of their own do not share one."""
    buckets = lz.rel_buckets(32, 128, "both")
    a, b = (torch.randint(-3, 4, (8, 8, 600, 600), device=DEV).bfloat16() for _ in range(2))
    want = [lz.rel_bias_grad(x, buckets) for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, x in enumerate((a, b)):
            got[i].append(lz.rel_bias_grad(x, buckets, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_rel_bias_custom_segments(lz):
    """Segments of a caller's own: rows in any order, one row twice, a row of none, a mask
    in the middle."""
    import ctypes
    starts = [-(1 << 31), -9, -2, 0, 1, 40, 300]
    ids = [3, -1, 0, 5, 3, -1, 1]
    pad = lambda x: (ctypes.c_int32 * lz.REL_MAX_SEGMENTS)(*x)  # noqa: E731
    buckets = lz.RelBuckets(pad(starts), pad(ids), len(ids), 7)
    H, Lq, Lk = 3, 100, 700
    rel = torch.arange(Lk, device=DEV) - torch.arange(Lq, device=DEV)[:, None]
    at = (rel[..., None] >= torch.tensor(starts, device=DEV)).sum(-1) - 1
    of = torch.tensor(ids, device=DEV)[at]
    table, add = torch.randn(7, H, device=DEV), torch.randn(2, H, Lq, Lk, device=DEV)
    assert torch.equal(lz.rel_bias(table, buckets, Lq, Lk, add=add), _want(table, add, of))
    x = torch.randint(-3, 4, (2, H, Lq, Lk), device=DEV).float()
    assert torch.equal(lz.rel_bias_grad(x, buckets), _grad(x, of, 7).float())
    x = x[..., :90, :80].masked_fill(of[:90, :80] < 0, math.nan)
    assert torch.equal(lz.rel_bias_grad(x, buckets), _grad(x, of[:90, :80], 7).float())


@pytest.mark.parametrize("q_start", [-(1 << 30), 0, 1 << 30])
def test_rel_bias_segments_at_the_ends_of_32_bits(lz, q_start):
    """Starts next to the largest and smallest 32-bit numbers, positions at both ends."""
    import ctypes
    starts = [-(1 << 31), -(1 << 31) + 1, -5, 2, (1 << 31) - 2, (1 << 31) - 1]
    ids = [0, 1, 2, 3, 4, -1]
    pad = lambda x: (ctypes.c_int32 * lz.REL_MAX_SEGMENTS)(*x)  # noqa: E731
    buckets = lz.RelBuckets(pad(starts), pad(ids), len(ids), 5)
    for Lq, Lk in ((100, 70), (600, 900)):
        rel = torch.arange(Lk, device=DEV) - torch.arange(Lq, device=DEV)[:, None] - q_start
        of = torch.tensor(ids, device=DEV)[(rel[..., None] >= torch.tensor(starts, device=DEV)).sum(-1) - 1]
        table = torch.randn(5, 2, device=DEV)
        assert torch.equal(lz.rel_bias(table, buckets, Lq, Lk, q_start=q_start), _want(table, None, of))
        x = torch.randint(-3, 4, (1, 2, Lq, Lk), device=DEV).float()
        assert torch.equal(lz.rel_bias_grad(x, buckets, q_start=q_start), _grad(x, of, 5).float())


def test_rel_bias_empty(lz):
    buckets = lz.rel_buckets(32, 128, "both")
    for shape in ((0, 2, 4, 4), (1, 2, 0, 4), (1, 2, 4, 0)):
        x = torch.zeros(shape, device=DEV)
        assert lz.rel_bias(torch.zeros(32, 2, device=DEV), buckets, *shape[2:], add=x).shape == shape
        assert not lz.rel_bias_grad(x, buckets).any()
        old = torch.ones(32, 2, device=DEV)
        assert bool((lz.rel_bias_grad(x, buckets, out=old, accumulate=True) == 1).all())


def test_rel_bias_in_a_graph_and_on_another_stream(lz):
    H, L = 4, 200
    buckets = lz.rel_buckets(32, 128, "causal")
    table, scores = torch.randn(32, H, device=DEV), torch.randn(2, H, L, L, device=DEV)
    out, grad = torch.empty_like(scores), torch.zeros(32, H, device=DEV)
    ws = lz.Workspace(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lz.rel_bias(table, buckets, L, L, add=scores, out=out)
        lz.rel_bias_grad(scores, buckets, out=grad)
    for i in range(4):
        table.normal_()
        scores.normal_()
        out.fill_(math.nan)
        grad.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        lz.rel_bias_grad(scores * 2, buckets, ws=ws)
        side.wait_stream(torch.cuda.current_stream())
        a = lz.rel_bias(table, buckets, L, L, add=scores, stream=side)
        b = lz.rel_bias_grad(scores, buckets, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(out, a) and torch.equal(grad, b), i


def test_rel_bias_refusals(lz):
    buckets = lz.rel_buckets(32, 128, "both")
    t = torch.zeros(32, 2, device=DEV)
    s = torch.zeros(1, 2, 8, 8, device=DEV)
    lz.rel_bias(t, buckets, 8, 8, add=s)
    z = lambda *n, d=torch.float32: torch.zeros(*n, dtype=d, device=DEV)  # noqa: E731
    for a, kw in (((z(31, 2), buckets, 8, 8), {}), ((t.bfloat16(), buckets, 8, 8), {}),
                  ((t.cpu(), buckets, 8, 8), {}), ((t, buckets, 8, 8), {"add": s[0]}),
                  ((t, buckets, 8, 8), {"add": z(1, 3, 8, 8)}),
                  ((t, buckets, 8, 8), {"add": z(1, 2, 8, 16)[..., ::2]}),
                  ((t, buckets, 8, 8), {"add": s.half()}), ((t, buckets, 8, 8), {"dtype": torch.half}),
                  ((t, buckets, 8, 8), {"add": s.cpu()}), ((t, buckets, 8, 8), {"out": z(2, 8, 9)}),
                  ((t, buckets, 8, 8), {"out": z(2, 8, 8, d=torch.bfloat16)}),
                  ((t, buckets, 8, 8), {"out": z(1, 8, 8).expand(2, 8, 8)}),
                  ((t, buckets, 8, 8), {"out": z(2, 8, 16)[..., ::2]}),
                  ((t, buckets, 8, 8), {"q_start": 1 << 31}),
                  ((z(2, 32).T, buckets, 8, 8), {})):
        with pytest.raises(lz.LmError):
            lz.rel_bias(*a, **kw)
    for x, kw in ((s.half(), {}), (s[0, 0], {}), (s.cpu(), {}), (z(1, 2, 8, 16)[..., ::2], {}),
                  (s, {"out": z(31, 2)}), (s, {"out": z(32, 2, d=torch.bfloat16)}),
                  (s, {"accumulate": True}), (s, {"out": z(2, 32).T}), (s, {"q_start": -(1 << 31)})):
        with pytest.raises(lz.LmError):
            lz.rel_bias_grad(x, buckets, **kw)
