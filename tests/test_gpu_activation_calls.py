"""Calls of dropout, layer norm and the token log probabilities that their documentation
allows at the edges: graphs, streams, autograd, sizes past 31 and 32 bits; and a training step
of them with the embedding's path, eager against 64 bits and captured against eager."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import activations_ref as A  # noqa: E402
import moments_ref as M  # noqa: E402
from paper_1810_10045_amd import synth  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
ONE_LAUNCH = (1 << 24) - 1  # workgroups of 256 threads


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lmzipf


def _room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB")


# ---------------------------------------------------------------------------
# Sizes past one launch, and offsets past 31 and 32 bits
# ---------------------------------------------------------------------------
def test_layer_norm_past_one_launch(lz):
    """Rows of one value: 64 of them a workgroup (32 groups of two), more than 2^24 workgroups."""
    _room(40)
    rows = ONE_LAUNCH * 64 + 130
    x = torch.zeros(rows, 1, dtype=BF16, device=DEV)
    at = sorted([0, 1 << 30, rows - 131, rows - 130, rows - 1])
    x[at] = 3.0
    bias = torch.full((1,), 0.5, device=DEV)
    r = lz.layer_norm(x, None, bias, out=x.clone())
    assert bool((r.y == 0.5).all())
    assert r.mean.nonzero().flatten().tolist() == at and bool((r.mean[at] == 3.0).all())


def test_token_logprobs_past_one_launch(lz):
    """Rows of one word: 16 of them a workgroup."""
    _room(24)
    N = ONE_LAUNCH * 16 + 40
    x = torch.zeros(N, 1, dtype=BF16, device=DEV)
    at = sorted([0, 1 << 28, N - 41, N - 1])
    x[at] = 2.0
    r = lz.token_logprobs(x)
    assert r.peak.nonzero().flatten().tolist() == at
    assert not r.log_sum.any() and not r.entropy.any()
    t = torch.zeros(N, dtype=torch.int32, device=DEV)
    g = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, torch.ones(N, device=DEV), out=x)
    assert not g.any()


def test_dropout_past_2_31_vectors(lz):
    """More vectors than 31 bits count: a second launch, whose mask goes on where the first's ends."""
    _room(48)
    D = 1 << 10  # 128 vectors a row
    rows = (1 << 24) + 3
    x = torch.ones(rows, D, dtype=BF16, device=DEV)
    lz.dropout(x, 0.5, 9, out=x)
    for r in (0, (1 << 24) - 9, (1 << 24) - 8, 1 << 24, rows - 1):
        w = M.words(np.arange(r * D // 2, (r + 1) * D // 2, dtype=np.uint64), 9)
        bits = np.stack((w & np.uint32(0xFFFF), w >> np.uint32(16)), 1).reshape(-1)
        assert np.array_equal(x[r].double().cpu().numpy(), np.where(bits >= 32768, 2.0, 0.0)), r


def _far_rows(n, D, dtype):
    """n rows of D values, more than 2^31 elements from one to the next."""
    ld = (1 << 31) + 9
    flat = torch.empty((n - 1) * ld + D, dtype=dtype, device=DEV)
    t = flat.as_strided((n, D), (ld, 1))
    t.copy_(torch.randn(n, D, generator=torch.Generator(device=DEV).manual_seed(n + D), device=DEV))
    return t


@pytest.mark.parametrize("dtype,D", [(BF16, 2049), (F32, 520)])
def test_rows_far_apart(lz, dtype, D):
    _room(40)
    x = _far_rows(3, D, dtype)
    near = x.clone()
    assert torch.equal(lz.dropout(x, 0.3, 1), lz.dropout(near, 0.3, 1))
    a, b = lz.layer_norm(x, add=x, p=0.1, seed=3), lz.layer_norm(near, add=near, p=0.1, seed=3)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    ga = lz.layer_norm_grad(x, x, a.mean, a.rstd, add=x, bias=True)
    gb = lz.layer_norm_grad(near, near, a.mean, a.rstd, add=near, bias=True)
    assert torch.equal(ga.dh, gb.dh) and torch.equal(ga.dbias, gb.dbias)
    t = torch.tensor([D - 1, 0, 5], device=DEV)
    p, q = lz.token_logprobs(x, t, top=5), lz.token_logprobs(near, t, top=5)
    assert all(torch.equal(u, v) for u, v in zip(p, q))
    want = lz.token_logprobs_grad(near, t, q.peak, q.log_sum, q.logp)
    assert torch.equal(lz.token_logprobs_grad(x, t, q.peak, q.log_sum, q.logp, out=x), want)


@pytest.mark.parametrize("V", [(1 << 29) + 3, 1 << 30])
def test_token_logprobs_of_the_largest_rows(lz, V):
    """A row of half a gigabyte's words and one of 2^30: the last ids are found."""
    _room(24)
    x = torch.full((1, V), -4.0, dtype=BF16, device=DEV)
    at = [V - 1, V // 2, 7, V - 2]
    x[0, at] = torch.tensor([9.0, 8.5, 8.0, 7.5], dtype=BF16, device=DEV)
    t = torch.tensor([V - 1], device=DEV)
    r = lz.token_logprobs(x, t, top=4)
    assert r.top_ids[0].tolist() == at
    # the sum: V - 4 equal terms and four more; fp32 sums of V / 2^15 terms in batches, and joins
    S = (V - 4) * np.exp(-13.0) + 1 + np.exp(-0.5) + np.exp(-1.0) + np.exp(-1.5)
    tol = (V // (1 << 15) // 32 + 200) * A.U
    assert abs(float(r.log_sum) - np.log(S)) < tol and abs(float(r.logp) + np.log(S)) < tol
    g = lz.token_logprobs_grad(x, t, r.peak, r.log_sum, torch.ones(1, device=DEV), out=x)
    want = np.exp(np.array([0.0, -0.5, -1.0, -1.5])) / S
    got = g[0, at].double().cpu().numpy()
    assert np.allclose(got, np.array([1.0, 0, 0, 0]) - want, rtol=2 ** -7, atol=2 ** -8)
    assert bool((g[0, 8:1000] == g[0, V // 2 + 1]).all())


# ---------------------------------------------------------------------------
# Graphs and streams
# ---------------------------------------------------------------------------
def test_graphs_read_their_seed_from_the_device(lz):
    """Captured calls, replayed with new seeds and inputs, eager calls in between: each replay is
    the eager call; a seed given as a number is repeated."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    rows, D, N, V = 77, 520, 3, 40_000
    x, add, dy = (torch.randn(rows, D, generator=gen, device=DEV).bfloat16() for _ in range(3))
    w, b = torch.randn(2, D, generator=gen, device=DEV).unbind()
    z = torch.randn(N, V, generator=gen, device=DEV)
    t = torch.randint(0, V, (N,), generator=gen, device=DEV)
    seed = torch.zeros(2, dtype=torch.int64, device=DEV)

    def step():
        f = lz.layer_norm(x, w, b, add=add, p=0.3, seed=seed[:1])
        g = lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, w, add=add, p=0.3, seed=seed[:1])
        r = lz.token_logprobs(z, t, top=6)
        return [*f, *g, *r, lz.dropout(x, 0.5, seed[1:], add=add), lz.dropout(x, 0.5, 12),
                lz.token_logprobs_grad(z, t, r.peak, r.log_sum, r.logp, r.entropy, r.entropy)]
    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g, stream=side):
            outs.append(step())
    for i in range(5):
        seed.copy_(torch.tensor([3 * i + 1, -i], device=DEV))
        x.normal_(generator=gen)
        z.normal_(generator=gen)
        torch.cuda.synchronize()
        want = [o.clone() for o in step()]
        for g, out in zip(graphs, outs):
            [o.zero_() for o in out]
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), i
    assert torch.equal(outs[0][-3], lz.dropout(x, 0.5, -4, add=add))


def test_a_workspace_of_the_callers_in_two_graphs(lz):
    """Two captured graphs with one workspace, replayed one after the other."""
    z = [torch.randn(2, 30_000, device=DEV) for _ in range(2)]
    h = [torch.randn(900, 300, device=DEV) for _ in range(2)]
    m, r = torch.zeros(900, device=DEV), torch.ones(900, device=DEV)
    ws = lz.Workspace(DEV)
    ws.get(1 << 22)

    def run(i):
        return [*lz.token_logprobs(z[i], top=3, ws=ws)[1:],
                *lz.layer_norm_grad(h[i], h[i], m, r, bias=True, ws=ws)[:1]]
    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g, stream=side):
            outs.append(run(i))
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_calls_on_two_streams_at_once(lz):
    """Calls that overlap on two streams, each with memory of its own."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    z = [torch.randn(2, 200_000, generator=gen, device=DEV) for _ in range(2)]
    h = [torch.randn(5000, 800, generator=gen, device=DEV) for _ in range(2)]
    w = torch.randn(800, generator=gen, device=DEV)
    m, r = torch.zeros(5000, device=DEV), torch.ones(5000, device=DEV)

    def run(i, stream):
        got = [*lz.token_logprobs(z[i], top=9, stream=stream)[1:]]
        got += lz.layer_norm_grad(h[i], h[i], m, r, w, stream=stream)
        got += lz.layer_norm(h[i], w, add=h[1 - i], stream=stream)
        return got + [lz.dropout(h[i], 0.1, i, stream=stream)]
    want = [run(i, None) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[run(i, s) for _ in range(3) for i, s in enumerate(streams)] for _ in range(2)]
    torch.cuda.synchronize()
    for turn in got:
        for k, out in enumerate(turn):
            assert all(torch.equal(a, b) for a, b in zip(out, want[k % 2]))


def test_memory_of_a_side_streams_results(lz):
    """Results made on a side stream come from its part of the allocator: what the current
    stream allocates meanwhile is not written."""
    side = torch.cuda.Stream()
    x = torch.randn(4000, 512, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    out = lz.layer_norm(x, add=x, p=0.5, seed=1, stream=side)
    del out
    new = [torch.full((4000, 512), 7.0, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((t == 7.0).all()) for t in new)


def test_plain_calls_are_the_other_calls(lz):
    """Calls that go through the extension module and the same calls that do not (an output, a
    workspace or a stream of the caller's): the same results, of the same shapes."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    here = torch.cuda.current_stream()
    ws = lz.Workspace(DEV)
    seed = torch.tensor([77], device=DEV)
    for dtype in (F32, BF16):
        x, add, dy = (torch.randn(2, 9, 130, generator=gen, device=DEV).to(dtype) for _ in range(3))
        w, b = torch.randn(2, 130, generator=gen, device=DEV).unbind()
        for s in (77, seed):
            for a in (None, add):
                got, want = lz.dropout(x, 0.3, s, add=a), torch.empty_like(x)
                lz.dropout(x, 0.3, 77, add=a, out=want)
                assert torch.equal(got, want)
                for p in (0.0, 0.3):
                    f = lz.layer_norm(x, w, b, add=a, p=p, seed=s)
                    g = lz.layer_norm(x, w, b, add=a, p=p, seed=s, stream=here)
                    assert all(torch.equal(u, v) and u.shape == v.shape for u, v in zip(f, g))
                    assert (f.h is x) == (g.h is x)
                    for bias in (None, True, False):
                        f2 = lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, w, a, p, s, bias=bias)
                        g2 = lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, w, a, p, s, bias=bias, ws=ws)
                        assert (f2.dbias is None) == (bias is False) == (g2.dbias is None)
                        for u, v in zip(f2, g2):
                            assert u is v is None or torch.equal(u, v)
                        assert (f2.dx is f2.dh) == (p == 0)
        for V in (130, 9000):
            z = torch.randn(3, V, generator=gen, device=DEV).to(dtype)
            t = torch.tensor([1, -100, V - 1], device=DEV)
            for targets in (None, t, t.int()):
                for top in (0, 4):
                    f = lz.token_logprobs(z, targets, 0.5, top)
                    g = lz.token_logprobs(z, targets, 0.5, top, stream=here)
                    for u, v in zip(f, g):
                        assert u is v is None or (torch.equal(u, v) and u.dtype == v.dtype)
            dl = torch.randn(3, generator=gen, device=DEV)
            f = lz.token_logprobs_grad(z, t, g.peak, g.log_sum, dl, g.entropy, dl, 0.5)
            assert torch.equal(f, lz.token_logprobs_grad(z, t, g.peak, g.log_sum, dl, g.entropy, dl,
                                                         0.5, out=torch.empty_like(z)))
    p = torch.nn.Parameter(torch.randn(4, 8, device=DEV))
    with torch.no_grad():
        assert not lz.dropout(p, 0.5, 1).requires_grad
        assert torch.equal(lz.layer_norm(p).y, lz.layer_norm(p.detach()).y)


# ---------------------------------------------------------------------------
# Autograd
# ---------------------------------------------------------------------------
def functions(lz):
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, add, w, b, p, seed):
            r = lz.layer_norm(x, w, b, add=add, p=p, seed=seed)
            ctx.save_for_backward(r.h, r.mean, r.rstd, w)
            ctx.p, ctx.seed = p, seed
            return r.y, r.h

        @staticmethod
        def backward(ctx, dy, dh):
            h, mean, rstd, w = ctx.saved_tensors
            g = lz.layer_norm_grad(dy.contiguous(), h, mean, rstd, w, add=dh.contiguous(), p=ctx.p,
                                   seed=ctx.seed)
            return g.dx, g.dh, g.dweight, g.dbias, None, None

    class Logp(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, t):
            r = lz.token_logprobs(z, t)
            ctx.save_for_backward(z, t, r.peak, r.log_sum, r.entropy)
            return r.logp, r.entropy

        @staticmethod
        def backward(ctx, dlogp, dentropy):
            z, t, peak, log_sum, entropy = ctx.saved_tensors
            return lz.token_logprobs_grad(z, t, peak, log_sum, dlogp.contiguous(), entropy,
                                          dentropy.contiguous()), None

    class Drop(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, seed):
            ctx.p, ctx.seed = p, seed
            return lz.dropout(x, p, seed)

        @staticmethod
        def backward(ctx, dy):
            return lz.dropout(dy.contiguous(), ctx.p, ctx.seed), None, None
    return Norm.apply, Logp.apply, Drop.apply


def test_in_autograd_functions(lz):
    """Dropout, norm, projection, loss with an entropy bonus: torch's autograd through them
    against torch's own in 64 bits."""
    norm, logp, drop = functions(lz)
    gen = torch.Generator(device=DEV).manual_seed(8)
    N, D, V = 12, 40, 90
    leaves = [torch.randn(*s, generator=gen, device=DEV) for s in ((N, D), (N, D), (D,), (D,), (D, V))]
    t = torch.randint(0, V, (N,), generator=gen, device=DEV)
    t[3] = -100
    k1, c1 = A.keep(N, D, 0.2, 5)
    k2, c2 = A.keep(N, D, 0.4, 6)
    own = [x.clone().requires_grad_() for x in leaves]
    y, h = norm(own[0], own[1], own[2], own[3], 0.2, 5)
    lp, ent = logp(drop(y + 0.1 * h, 0.4, 6) @ own[4], t)
    (-lp.sum() - 0.3 * ent.sum()).backward()
    ref = [x.double().cpu().requires_grad_() for x in leaves]
    h = ref[1] + ref[0] * torch.from_numpy(k1 * c1)
    d = h - h.mean(1, keepdim=True)
    y = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * ref[2] + ref[3]
    l = torch.log_softmax(((y + 0.1 * h) * torch.from_numpy(k2 * c2)) @ ref[4], 1)
    ent = -(l.exp() * l).sum(1)
    tc = t.cpu()
    lp = torch.where(tc < 0, 0.0, l[torch.arange(N), tc.clamp(min=0)])
    (-lp.sum() - 0.3 * ent.sum()).backward()
    # chains of sums of at most 90 terms, three roundings of everything between: the norm of the
    # difference is under 1000 half steps of the gradient's own norm
    for a, b in zip(own, ref):
        diff = float((a.grad.double().cpu() - b.grad).norm())
        assert diff <= 1000 * A.U * float(b.grad.norm())


def test_writes_in_place_are_seen_by_autograd(lz):
    x, add = torch.randn(4, 8, device=DEV), torch.randn(4, 8, device=DEV)
    v = torch.zeros(4, device=DEV)
    for f, t in ((lambda: lz.dropout(x, 0.5, 1, out=add), add),
                 (lambda: lz.layer_norm(x, add=add, sum_out=add), add),
                 (lambda: lz.layer_norm(x, out=add), add),
                 (lambda: lz.layer_norm_grad(x, x, v, v, out=add), add),
                 (lambda: lz.token_logprobs_grad(x, None, v, v, out=add), add)):
        before = t._version
        f()
        assert t._version > before
    w = torch.randn(4, 8, device=DEV, requires_grad=True)
    y = (w * x).sum()
    with torch.no_grad():
        lz.dropout(add, 0.5, 1, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


def test_refusals_of_tensors(lz):
    x = torch.randn(6, 8, device=DEV)
    v, w = torch.zeros(6, device=DEV), torch.zeros(8, device=DEV)
    t = torch.zeros(6, dtype=torch.int64, device=DEV)
    err = torch.zeros(2, device=DEV)
    for f in (lambda: lz.dropout(x.half(), 0.5, 1), lambda: lz.dropout(x, 0.5, 1, add=x.bfloat16()),
              lambda: lz.dropout(x, 0.5, 1, out=x[:5]), lambda: lz.dropout(x, 1.5, 1),
              lambda: lz.dropout(x, 0.5, torch.zeros(1, device=DEV)),
              lambda: lz.dropout(x, 0.5, torch.zeros(1, dtype=torch.int64)),
              lambda: lz.dropout(x.t(), 0.5, 1), lambda: lz.dropout(x[:, :4], 0.5, 1, out=x[:, 2:6]),
              lambda: lz.dropout(x[:1].expand(6, 8), 0.5, 1),
              lambda: lz.layer_norm(x, w.bfloat16()), lambda: lz.layer_norm(x, v),
              lambda: lz.layer_norm(x, w, torch.zeros(16, device=DEV)[::2]),
              lambda: lz.layer_norm(x, out=x, sum_out=x), lambda: lz.layer_norm(x, eps=-1.0),
              lambda: lz.layer_norm(torch.zeros(2, 16385, device=DEV)),
              lambda: lz.layer_norm_grad(x, x[:, :4], v, v), lambda: lz.layer_norm_grad(x, x, v, w),
              lambda: lz.layer_norm_grad(x, x, v, v, w, accumulate=True),
              lambda: lz.layer_norm_grad(x, x, v, v, w, dweight=w.clone(), accumulate=True),
              lambda: lz.layer_norm_grad(x, x, v, v, w, dweight=w),
              lambda: lz.token_logprobs(x, t[:5]), lambda: lz.token_logprobs(x, t.float()),
              lambda: lz.token_logprobs(x, top=65), lambda: lz.token_logprobs(x, scale=0.0),
              lambda: lz.token_logprobs(x, dev_err=err), lambda: lz.token_logprobs(x, t.cpu()),
              lambda: lz.token_logprobs_grad(x, None, v, v, dlogp=v),
              lambda: lz.token_logprobs_grad(x, t, v, v, dentropy=v),
              lambda: lz.token_logprobs_grad(x, t, v, w, dlogp=v),
              lambda: lz.token_logprobs_grad(x, t, v, v, dlogp=v, out=x.bfloat16())):
        with pytest.raises(lz.LmError):
            f()


# ---------------------------------------------------------------------------
# A training step
# ---------------------------------------------------------------------------
B, L, DM, VOC = 3, 50, 72, 700


class Model:
    """Embedding, dropout and norm behind it, a residual layer with its norm, the output's
    projection, and the loss of the next words; the embedding's rows by Unique and Seg-Sum."""

    def __init__(self, lz, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lz = lz
        r = lambda *n: torch.randn(*n, generator=gen, device=DEV) * 0.3  # noqa: E731
        self.embed = r(VOC, DM)
        self.w1, self.b1, self.w2, self.b2 = (r(DM) + 1, r(DM), r(DM) + 1, r(DM))
        self.inner, self.out = r(DM, DM), r(DM, VOC)
        self.params = [self.w1, self.b1, self.w2, self.b2, self.inner, self.out]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.m, self.v = ([torch.zeros_like(p) for p in self.params] for _ in range(2))
        self.plan = lz.adamw_plan(self.params, self.grads, self.m, self.v)
        self.ids = torch.zeros(B * L, dtype=torch.int32, device=DEV)
        self.next = torch.zeros(B * L, dtype=torch.int64, device=DEV)
        self.unique = lz.unique_buffers(B * L, VOC, torch.int32, torch.device(DEV))
        self.sums = torch.zeros(B * L, DM, device=DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.seeds = torch.zeros(2, dtype=torch.int64, device=DEV)
        self.ws = lz.Workspace(DEV)
        self.ws.get(1 << 20)

    def state(self):
        return [self.embed, *self.params, *self.m, *self.v]

    def step(self, n):
        lz, ws, (gw1, gb1, gw2, gb2, ginner, gout) = self.lz, self.ws, self.grads
        s1, s2 = self.seeds[:1], self.seeds[1:]
        x = self.embed[self.ids.long()]
        a = lz.layer_norm(x, self.w1, self.b1, p=0.1, seed=s1)
        branch = a.y @ self.inner
        c = lz.layer_norm(branch, self.w2, self.b2, add=a.h, p=0.2, seed=s2)
        logits = c.y @ self.out
        r = lz.token_logprobs(logits, self.next, dev_err=self.err, ws=ws)
        dlogp = torch.full_like(r.logp, -1.0 / (B * L))
        dlogits = lz.token_logprobs_grad(logits, self.next, r.peak, r.log_sum, dlogp, out=logits)
        gout.copy_(c.y.t().contiguous() @ dlogits)
        dy = dlogits @ self.out.t().contiguous()
        g = lz.layer_norm_grad(dy, c.h, c.mean, c.rstd, self.w2, p=0.2, seed=s2, dweight=gw2,
                               dbias=gb2, ws=ws)
        ginner.copy_(a.y.t().contiguous() @ g.dx)
        dy = g.dx @ self.inner.t().contiguous()
        g = lz.layer_norm_grad(dy, a.h, a.mean, a.rstd, self.w1, add=g.dh, p=0.1, seed=s1,
                               dweight=gw1, dbias=gb1, ws=ws)
        u = lz.unique(self.ids, VOC, out=self.unique, ws=ws)
        lz.segsum(g.dx, u.perm, u.inverse, u.offsets, u.num_unique, out=self.sums, dev_err=self.err,
                  ws=ws)
        lz.sparse_apply(self.embed, u.uniq, u.num_unique, self.sums, "sgd", lr=0.1, dev_err=self.err)
        lz.adamw(self.plan, lr=1e-2, weight_decay=0.1, step=n, dev_err=self.err)
        return r.logp

    def feed(self, seed):
        ids = synth.zipf_ids(B * L + 1, VOC, 1.0, seed, np.int32)
        self.ids.copy_(torch.from_numpy(ids[:-1]))
        self.next.copy_(torch.from_numpy(ids[1:].astype(np.int64)))
        self.next[5] = -100
        self.seeds.copy_(torch.tensor([2 * seed, 2 * seed + 1], device=DEV))


def _autograd(m):
    embed, w1, b1, w2, b2, inner, out = (t.double().cpu().requires_grad_()
                                         for t in (m.embed, *m.params))
    seeds = m.seeds.tolist()

    def keep(p, s):
        k, c = A.keep(B * L, DM, p, s)
        return torch.from_numpy(k * c)

    def norm(h, w, b):
        d = h - h.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * w + b
    h1 = embed[m.ids.long().cpu()] * keep(0.1, seeds[0])
    h2 = h1 + (norm(h1, w1, b1) @ inner) * keep(0.2, seeds[1])
    l = torch.log_softmax(norm(h2, w2, b2) @ out, 1)
    t = m.next.cpu()
    logp = torch.where(t < 0, 0.0, l[torch.arange(B * L), t.clamp(min=0)])
    loss = -logp.sum() / (B * L)
    return logp.detach(), torch.autograd.grad(loss, (embed, w1, b1, w2, b2, inner, out))


def test_training_step(lz):
    m = Model(lz, 1)
    for n in (1, 2, 3):
        m.feed(20 + n)
        want, (ge, *grads) = _autograd(m)
        logp = m.step(n)
        torch.cuda.synchronize()
        lz.check(m.err)
        lz.check(m.unique.dev_err)
        # fp32 chains of products and sums of at most 700 terms, two norms and a softmax between:
        # the norm of the difference is under 2000 half steps of the value's own norm
        near = lambda a, b: float((a - b).norm()) <= 2000 * A.U * float(b.norm())  # noqa: E731
        assert near(logp.double().cpu(), want)
        for g, w in zip(m.grads, grads):
            assert near(g.double().cpu(), w)
        U = int(m.unique.num_unique)
        assert near(m.sums[:U].double().cpu(), ge[m.unique.uniq[:U].long().cpu()])


def test_training_step_in_a_graph(lz):
    """The step captured and replayed on new ids, seeds and state, eager steps of another model
    between the replays: each replay is the eager step."""
    m, other = Model(lz, 2), Model(lz, 3)
    m.feed(1)
    m.step(5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.step(5)
    for i in range(4):
        m.feed(50 + i)
        other.feed(60 + i)
        before = [t.clone() for t in m.state()]
        torch.cuda.synchronize()
        graph.replay()
        other.step(i + 1)
        torch.cuda.synchronize()
        lz.check(m.err)
        after = [t.clone() for t in m.state()]
        [t.copy_(x) for t, x in zip(m.state(), before)]
        two = lz.segsum_two_launches(True)  # the form that a capture takes: the same order of sums
        m.step(5)
        lz.segsum_two_launches(two)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(m.state(), after)), i
