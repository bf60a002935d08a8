"""What the results of dropout, layer norm and the token log probabilities keep to whatever
their inputs are: signs, and memory that is not theirs."""
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


# ---------------------------------------------------------------------------
# Log probabilities are at most 0
# ---------------------------------------------------------------------------
# Rows in some lanes, in a wave's, by a workgroup each, and cut into parts
@pytest.mark.parametrize("N,V", [(512, 3), (512, 98), (512, 1500), (1100, 3001), (24, 9000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [-INF, -30.0])
def test_log_probabilities_are_not_above_0(lz, N, V, dtype, rest):
    """One word left of each row, or one far above the others: it contributes e^0 to the sum, so
    the sum's logarithm is 0 or more and no probability is above 1."""
    top = torch.linspace(-32, 32, N, device=DEV) + torch.arange(N, device=DEV) % 7 * 0.013
    top = top.to(dtype).to(F32)
    at = torch.arange(N, device=DEV) * 31 % V
    for scale in (1.0, 1 / 0.7, 0.37, 3.0):
        x = (top[:, None] + rest / scale).expand(N, V).to(dtype).contiguous()
        x[torch.arange(N, device=DEV), at] = top.to(dtype)
        r = lz.token_logprobs(x, at, scale=scale, top=2)
        s = float(np.float32(scale))
        ref = A.logprobs(x.double().cpu().numpy(), at.cpu().numpy(), s, 2)
        assert bool((r.log_sum >= 0).all()) and bool((r.entropy >= 0).all())
        assert bool((r.logp <= 0).all()) and bool((r.top_logp <= 0).all())
        assert torch.equal(r.top_logp[:, 0], r.logp)
        for name in ("log_sum", "logp", "top_logp", "entropy"):
            want, tol = ref[name]
            got = getattr(r, name).double().cpu().numpy()
            same = got == want
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(got - want) <= tol + A.TINY)).all(), (scale, name)


# ---------------------------------------------------------------------------
# More logits at the border of the alternatives than are ranked at once
# ---------------------------------------------------------------------------
# Rows of no two equal logits: in lanes' registers (about half of them with 64 alternatives have
# more than 256 candidates, all of them where lanes are left without a logit), by a workgroup each
# and cut into parts
@pytest.mark.parametrize("N,V", [(300, 257), (300, 300), (300, 511), (300, 1000), (40, 2048),
                                 (1030, 2100), (3, 9000)])
@pytest.mark.parametrize("top", [60, 62, 63, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_candidates(lz, N, V, top, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + top)
    x = torch.stack([torch.randperm(V, generator=gen, device=DEV) for _ in range(N)])
    x = (x - V // 2).to(F32)
    # different bf16 numbers: each integer's own bits, its sign kept
    x = (x.sign() * 2.0 ** (x.abs() // 128 - 40) * (1 + x.abs() % 128 / 128)).to(dtype)
    assert int(torch.unique(x[0]).numel()) >= V - 1  # (0 and the smallest at most are one)
    r = lz.token_logprobs(x, top=top)
    ref = A.logprobs(x.double().cpu().numpy(), None, 1.0, top)
    assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"][0])
    want, tol = ref["top_logp"]
    assert (np.abs(r.top_logp.double().cpu().numpy() - want) <= tol + A.TINY).all()


@pytest.mark.parametrize("V", [1500, 4099, 80_001])
@pytest.mark.parametrize("live", [65, 300, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_alternatives_in_a_few_parts_of_a_row(lz, V, live, dtype):
    """Words left in a few stretches: parts of the row without any, so that every word left is a
    candidate."""
    gen = torch.Generator(device=DEV).manual_seed(V + live)
    for N in (5, 1040):
        x = torch.full((N, V), -INF, dtype=dtype, device=DEV)
        place = torch.arange(live, device=DEV)
        place = place // 8 % 3 * 8 * 64 + place % 8 + place // 24 * 8 * 64 * 3  # a lane's vectors
        place = place[place < V]
        x[:, place] = torch.randn(N, len(place), generator=gen, device=DEV).to(dtype)
        r = lz.token_logprobs(x, top=64)
        rows = [0, 1, N // 2, N - 1]
        ref = A.logprobs(x[rows].double().cpu().numpy(), None, 1.0, 64)
        assert np.array_equal(r.top_ids[rows].cpu().numpy(), ref["top_ids"][0])
        want, tol = ref["top_logp"]
        got = r.top_logp[rows].double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            assert ((got == want) | (np.abs(got - want) <= tol + A.TINY)).all()


# ---------------------------------------------------------------------------
# Memory around a result that has gaps
# ---------------------------------------------------------------------------
class Framed:
    """rows x D values to be written, `gap` elements between rows, in memory of NaN."""

    def __init__(self, rows, D, dtype, values=None, gap=5, off=3):
        ld = D + gap
        self.flat = torch.full((off + rows * ld + 64,), NAN, dtype=dtype, device=DEV)
        self.t = self.flat[off:off + rows * ld].view(rows, ld)[:, :D]
        self.around = torch.ones_like(self.flat, dtype=torch.bool)
        self.around[off:off + rows * ld].view(rows, ld)[:, :D] = False
        if values is not None:
            self.t.copy_(values)

    def check(self, what):
        assert bool(torch.isfinite(self.t).all()), f"{what}: not every value is written"
        n = int((~torch.isnan(self.flat[self.around])).sum())
        assert n == 0, f"{what}: {n} elements around the rows are written"


# On both sides of a vector's width (4 fp32, 8 bf16), of a wave's and of a workgroup's, one row,
# rows that fill a workgroup's groups and rows that do not
@pytest.mark.parametrize("rows", [1, 3, 41, 1100])
@pytest.mark.parametrize("D", [1, 3, 4, 5, 7, 8, 9, 63, 64, 65, 255, 257, 512, 517, 2047, 2049])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nothing_around_the_rows_is_written(lz, dtype, D, rows):
    gen = torch.Generator(device=DEV).manual_seed(rows * 10_000 + D)
    x, add, dy = (torch.randn(rows, D, generator=gen, device=DEV).to(dtype) for _ in range(3))
    new = lambda values=None: Framed(rows, D, dtype, values)  # noqa: E731

    def same(frame, want, what):
        frame.check(what)
        assert torch.equal(frame.t, want), what
    want = lz.dropout(x, 0.3, 5, add=add)
    a, b, c = new(), new(x), new(add)
    lz.dropout(x, 0.3, 5, add=add, out=a.t)
    same(a, want, "dropout")
    lz.dropout(b.t, 0.3, 5, add=c.t, out=b.t)
    same(b, want, "dropout in place")
    same(c, add, "dropout's addend")
    f = lz.layer_norm(x, add=add, p=0.2, seed=4)
    y, h, s = new(), new(), new(add)
    lz.layer_norm(x, add=add, p=0.2, seed=4, out=y.t, sum_out=h.t)
    same(y, f.y, "norm")
    same(h, f.h, "norm's sum")
    lz.layer_norm(x, add=s.t, p=0.2, seed=4, sum_out=s.t)
    same(s, f.h, "norm's sum in place")
    g = lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, add=add, p=0.2, seed=4, bias=True)
    dh, dx, past = new(), new(), new(add)
    db = Framed(1, D, F32, gap=0)
    lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, add=add, p=0.2, seed=4, out=dh.t, dx=dx.t,
                       dbias=db.t[0])
    same(dh, g.dh, "norm's gradient")
    same(dx, g.dx, "norm's gradient through dropout")
    same(db, g.dbias[None], "the bias's gradient")
    lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, add=past.t, p=0.2, seed=4, out=past.t)
    same(past, g.dh, "norm's gradient in place")
    t = torch.randint(0, D, (rows,), generator=gen, device=DEV)
    r = lz.token_logprobs(x, t)
    want = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, r.entropy + 1, r.entropy, r.entropy + 1)
    out, z = new(), new(x)
    for where, source in ((out, x), (z, z.t)):
        lz.token_logprobs_grad(source, t, r.peak, r.log_sum, r.entropy + 1, r.entropy, r.entropy + 1,
                               out=where.t)
        same(where, want, "the logits' gradient")


# ---------------------------------------------------------------------------
# A workspace that two graphs share
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("rows,D", [(900, 300), (4000, 40), (2000, 517), (100, 4100)])
def test_weights_gradients_of_two_graphs_with_one_workspace(lz, rows, D):
    """The results that pass through the workspace, whatever it holds before a replay."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    h, dy = ([torch.randn(rows, D, generator=gen, device=DEV) for _ in range(2)] for _ in range(2))
    w = torch.randn(D, generator=gen, device=DEV)
    m, r = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    need = lz.lib().lm_layer_norm_grad_workspace_bytes(rows, D, lz.F32)
    assert need > 0
    ws = lz.Workspace(DEV)
    ws.get(need)

    def run(i):
        return [*lz.layer_norm_grad(dy[i], h[i], m, r, w, ws=ws)]
    want = [run(i) for i in range(2)]
    for i in range(2):
        ref = A.norm_grad(*(t.double().cpu().numpy() for t in (dy[i], h[i], m, r, w)))
        for name in ("dweight", "dbias"):
            got = dict(zip(("dh", "dx", "dweight", "dbias"), want[i]))[name].double().cpu().numpy()
            assert (np.abs(got - ref[name][0]) <= ref[name][1] + A.TINY).all(), name
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g, stream=side):
            outs.append(run(i))
    for n in range(4):
        [t.zero_() for out in outs for t in out]
        ws.buf.view(torch.uint8).fill_(0xff)  # NaN
        for g in graphs if n % 2 else reversed(graphs):
            g.replay()
        torch.cuda.synchronize()
        run(n % 2)  # the program's own call with the same workspace
        for a, b in zip(outs, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b)), n


# ---------------------------------------------------------------------------
# The gradient of the longest rows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("V", [(1 << 29) + 3, 1 << 30])
def test_gradient_of_the_longest_rows(lz, V):
    """Every word's gradient, to the rounding of bf16 and what log_sum may be off."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    x = torch.full((1, V), -4.0, dtype=BF16, device=DEV)
    at = [V - 1, V // 2, 7, V - 2]
    x[0, at] = torch.tensor([9.0, 8.5, 8.0, 7.5], dtype=BF16, device=DEV)
    t = torch.tensor([V // 2], device=DEV)
    r = lz.token_logprobs(x, t)
    S = (V - 4) * np.exp(-13.0) + 1 + np.exp(-0.5) + np.exp(-1.0) + np.exp(-1.5)
    # a thread sums V / 2^15 logits in batches of 32, parts are joined
    off = (V // (1 << 15) // 32 + 200) * A.U
    g = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, torch.full((1,), 3.0, device=DEV), out=x)
    q = np.exp(np.array([0.0, -0.5, -1.0, -1.5, -13.0])) / S
    want = 3 * (np.array([0, 1.0, 0, 0, 0]) - q)
    got = g[0, [*at, 0]].double().cpu().numpy()
    # an exponent of up to 13 + log S is off by 16 of its half steps at most
    tol = 1.01 * A.HALF[BF16] * np.abs(want) + 3 * q * (1.01 * off + 16 * (13 + np.log(S)) * A.U)
    assert (np.abs(got - want) <= tol).all(), (got, want, tol)
    assert int((g == g[0, 0]).sum()) == V - 4
