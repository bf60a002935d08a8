"""Calls of the AdamW and relative-bias entry points that their documentation allows at
the edges: grids past one launch, memory across streams, state that is kept, autograd."""
import ctypes
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as M  # noqa: E402
import relbias_ref as R  # noqa: E402
import test_gpu_adamw as adamw_tests  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
ONE_LAUNCH = (1 << 24) - 1  # workgroups of 256 threads


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    M.device_powers(torch)
    return lmzipf


def _room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB")


# ---------------------------------------------------------------------------
# More workgroups than one launch holds
# ---------------------------------------------------------------------------
def test_rel_bias_past_one_launch(lz):
    """One workgroup a head and batch entry, more than 2^24 of them."""
    _room(4)
    B, H, Lk = (1 << 23) + 3, 2, 3
    assert B * H > ONE_LAUNCH
    table = torch.randn(32, H, device=DEV)
    add = torch.randn(B, H, 1, Lk, device=DEV)
    got = lz.rel_bias(table, lz.rel_buckets(32, 128, "both"), 1, Lk, q_start=1, add=add)
    of = torch.tensor([R.bucket(j - 1, 32, 128, "both") for j in range(Lk)], device=DEV)
    assert torch.equal(got, add + table[of].T[None, :, None])


@pytest.mark.parametrize("B,H,Lk,threads", [(1, (1 << 22) + 5, 4, 1024),     # a head a workgroup
                                            (9, (1 << 22) + 5, 4, 1024),     # the join's
                                            (1, (1 << 23) + 1, 257, 256)])   # two a head
def test_rel_bias_grad_past_one_launch(lz, B, H, Lk, threads):
    _room(24)
    assert H * (2 if Lk > 256 else 1) * threads >= 1 << 32
    buckets = lz.rel_buckets(4, 3, "both")
    of = torch.tensor([R.bucket(j, 4, 3, "both") for j in range(Lk)], device=DEV)
    x = torch.randint(-3, 4, (B, H, 1, Lk), device=DEV, dtype=torch.int8).float()
    got = lz.rel_bias_grad(x, buckets)
    total = x.sum(0)[:, 0]
    del x
    for n in range(4):
        assert torch.equal(got[n], total[:, of == n].sum(1)), n


def test_rows8_past_one_launch(lz):
    """A capacity of 2^31 - 1 rows of one value, most of whose ids name no row."""
    _room(24)
    cap, V = (1 << 31) - 1, 50
    rows = torch.full((cap,), -1, dtype=torch.int32, device=DEV)
    vals = torch.zeros(cap, 1, device=DEV)
    at, ids = [0, 1 << 30, cap - 3, cap - 2, cap - 1], [4, 9, 20, 30, 49]
    rows[at] = torch.tensor(ids, dtype=torch.int32, device=DEV)
    vals[at] = 1.0
    table = torch.zeros(V, 1, device=DEV)
    m, v, ms, vs = (torch.zeros(V, 1, dtype=torch.uint8, device=DEV) for _ in range(4))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    lz.sparse_apply_q8(table, rows, torch.tensor([cap], device=DEV), vals, m, v, ms, vs, lr=0.5,
                       dev_err=err)
    assert int(err.item()) == lz.DEVERR_ID_RANGE
    for t in (table, m, v, ms, vs):
        assert t[:, 0].nonzero().flatten().tolist() == ids
    assert float((table[ids] + 0.5).abs().max()) < 1e-6


def test_adamw_past_one_launch(lz):
    """A list of more than 2^24 tensors of one value."""
    _room(8)
    n = ONE_LAUNCH + 4
    p, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    g = torch.ones(n, device=DEV)
    at = lambda t: np.uint64(t.data_ptr()) + 4 * np.arange(n, dtype=np.uint64)  # noqa: E731
    lists = [at(t) for t in (p, g, m, v)]
    sizes = np.ones(n, np.int64)
    ptr = lambda a: a.ctypes.data  # noqa: E731
    need = lz.lib().lm_adamw_plan_bytes(ptr(sizes), n)
    table = np.zeros(need // 8, np.uint64)
    chunks = ctypes.c_int64()
    assert lz.lib().lm_adamw_plan(*[ptr(a) for a in lists], None, None, None, ptr(sizes), None, n,
                                  lz.F32, 32, ptr(table), need, ctypes.byref(chunks)) == 0
    assert chunks.value == n
    plan = torch.from_numpy(table.view(np.int64)).to(DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert lz.lib().lm_adamw(plan.data_ptr(), need, n, lz.F32, 32, 0, 0.5, 0.0, 0.0, 1e-8, 0.0, 1,
                             None, 0, err.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    lz.check(err)
    assert bool((m == 1).all()) and bool((v == 1).all()) and float((p + 0.5).abs().max()) < 1e-6


# ---------------------------------------------------------------------------
# Memory across streams
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("states", [32, 8])
def test_adamw_plan_memory_outlives_a_late_side_stream(lz, states):
    """A step that waits on a side stream when the plan, the last owner of its tensors, goes
    away: their memory goes to no new tensor of the first stream before the step is over."""
    n = 300_000
    dt = torch.uint8 if states == 8 else torch.float32
    p, g = torch.zeros(n, device=DEV), torch.ones(n, device=DEV)
    m, v = (torch.zeros(n, dtype=dt, device=DEV) for _ in range(2))
    copy = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    scales = [[torch.zeros(M.blocks(n), dtype=torch.uint8, device=DEV)] for _ in range(2)]
    kw = dict(m_scale=scales[0], v_scale=scales[1]) if states == 8 else {}
    plan = lz.adamw_plan([p], [g], [m], [v], copies=[copy], **kw)
    sizes = [(t.numel(), t.dtype) for t in (g, m, v, copy, *scales[0], *scales[1])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # 10 to 200 ms by the clock it counts
    lz.adamw(plan, lr=0.5, beta1=0.0, beta2=0.0, stream=side)
    del plan, g, m, v, copy, scales, kw
    new = [torch.full((k,), 7, dtype=d, device=DEV) for k, d in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in new)
    assert float((p + 0.5).abs().max()) < 1e-6


# ---------------------------------------------------------------------------
# Values that a step leaves as they are
# ---------------------------------------------------------------------------
def _state_that_rounds_down(lz, shape):
    """8-bit moments whose blocks keep their scale (each holds 448), at scales whose power the
    device's math library gives half a unit low, and a seed for which some codes of both moments
    are rounded with the random part 0: scaled by such a power they would lose a step."""
    rng = np.random.default_rng(7)
    n = shape[0] * shape[1]
    bytes_ = np.arange(1, 255)
    low = bytes_[M.INVERSE[1:255] < np.exp2(127.0 - bytes_)]
    low = low if len(low) else bytes_
    m = rng.integers(1, 0x7F, shape).astype(np.uint8) | \
        (rng.integers(0, 2, shape).astype(np.uint8) << 7)
    v = rng.integers(1, 0x7F, shape).astype(np.uint8)
    m[:, ::32] = v[:, ::32] = 0x7E
    ms, vs = (rng.choice(low, (shape[0], M.blocks(shape[1]))).astype(np.uint8) for _ in range(2))
    for seed in range(100):
        w = M.words(np.arange(n, dtype=np.uint64), seed)
        if ((w >> np.uint32(12)) == 0).any() and ((w & np.uint32(0xFFFFF)) == 0).any():
            break
    else:
        raise AssertionError("no seed with a random part of 0")
    return seed, [torch.from_numpy(x).to(DEV) for x in (m, v, ms, vs)]


def test_adamw8_values_without_a_finite_moment_keep_their_codes(lz):
    seed, state = _state_that_rounds_down(lz, (1, 1 << 22))
    state = [x[0] for x in state]
    p = torch.randn(1 << 22, device=DEV)
    t = [x.clone() for x in (p, *state)]
    g = torch.full_like(p, float("nan"))
    plan = lz.adamw_plan([t[0]], [g], [t[1]], [t[2]], m_scale=[t[3]], v_scale=[t[4]])
    lz.adamw(plan, seed=seed, weight_decay=0.1)
    for got, was in zip(t, (p, *state)):
        assert torch.equal(got, was)


def test_rows8_values_without_a_finite_moment_keep_their_codes(lz):
    V, D = 4096, 1024
    seed, state = _state_that_rounds_down(lz, (V, D))
    p = torch.randn(V, D, device=DEV)
    t = [x.clone() for x in (p, *state)]
    rows = torch.arange(V, dtype=torch.int32, device=DEV)
    lz.sparse_apply_q8(t[0], rows, torch.tensor([V], device=DEV),
                       torch.full((V, D), float("inf"), device=DEV), *t[1:], seed=seed)
    for got, was in zip(t, (p, *state)):
        assert torch.equal(got, was)


@pytest.mark.parametrize("states_kept", [True, False])
def test_adamw8_kept_values_in_a_block_whose_scale_shrinks(lz, states_kept):
    """The block's largest value decays until its scale halves (its gradient is finite, and
    beta = 0); the others, kept, are the same numbers on the finer grid."""
    n = 1 << 20
    seed, state = _state_that_rounds_down(lz, (1, n))
    m, v, ms, vs = [x[0] for x in state]
    for c in (m, v):                     # the others: at most 224, so the scale can halve
        rest = c.view(-1, 32)[:, 1:]
        rest.copy_(torch.where((rest & 0x7F) > 0x76, (rest & 0x80) | 0x76, rest))
    ms.clamp_(60, 170)                   # (squares of the roots are finite)
    vs.clamp_(60, 170)
    before = [M.decode(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((m, ms), (v, vs))]
    g = torch.full((n,), float("nan"), device=DEV)
    if not states_kept:
        g[::32] = 0.0
    p = torch.randn(n, device=DEV)
    plan = lz.adamw_plan([p], [g], [m], [v], m_scale=[ms], v_scale=[vs])
    lz.adamw(plan, seed=seed, beta1=0.0, beta2=0.0)
    for was, c, s in zip(before, (m, v), (ms, vs)):
        got = M.decode(c.cpu().numpy(), s.cpu().numpy()).reshape(-1, 32)
        assert np.array_equal(got[:, 1:], was.reshape(-1, 32)[:, 1:])
        assert np.array_equal(got[:, 0], was[::32] if states_kept else np.zeros(n // 32))


# ---------------------------------------------------------------------------
# Scores and output in one buffer
# ---------------------------------------------------------------------------
def test_rel_bias_scores_beside_the_output(lz):
    """Halves of a buffer's columns and of its heads, and a view in another order beside the
    output: taken, and right."""
    B, H, L = 2, 4, 70
    table, buckets = torch.randn(32, H, device=DEV), lz.rel_buckets(32, 128, "both")
    of = torch.tensor([[R.bucket(j - i, 32, 128, "both") for j in range(L)] for i in range(L)],
                      device=DEV)
    wide, tall = torch.randn(B, H, L, 2 * L, device=DEV), torch.randn(B, 2 * H, L, L, device=DEV)
    both = torch.randn(2 * H, B, L, L, device=DEV)
    for add, out in ((wide[..., :L], wide[..., L:]), (wide[..., L:], wide[..., :L]),
                     (tall[:, H:], tall[:, :H]), (tall[:, ::2], tall[:, 1::2]),
                     (both[:H].transpose(0, 1), both[H:].view(B, H, L, L))):
        was = add.clone()
        lz.rel_bias(table, buckets, L, L, add=add, out=out)
        assert torch.equal(out, was + table[of].permute(2, 0, 1)) and torch.equal(add, was)
    with pytest.raises(lz.LmError):
        lz.rel_bias(table, buckets, L, L, add=wide[..., 1:L + 1], out=wide[..., :L])
    with pytest.raises(lz.LmError):
        lz.rel_bias(table, buckets, L, L, add=tall[:, 1:H + 1], out=tall[:, :H])


# ---------------------------------------------------------------------------
# Autograd
# ---------------------------------------------------------------------------
def test_rel_bias_refuses_to_drop_a_graph(lz):
    buckets = lz.rel_buckets(32, 128, "causal")
    table, add = torch.randn(32, 2, device=DEV), torch.randn(1, 2, 8, 8, device=DEV)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda: lz.rel_bias(leaf(table), buckets, 8, 8),
             lambda: lz.rel_bias(table, buckets, 8, 8, add=leaf(add)),
             lambda: lz.rel_bias(table, buckets, 8, 8, add=leaf(add) * 2),
             lambda: lz.rel_bias(table, buckets, 8, 8, add=add, out=leaf(add)),
             lambda: lz.rel_bias_grad(leaf(add), buckets),
             lambda: lz.rel_bias_grad(add, buckets, out=leaf(table))]
    for call in calls:
        with pytest.raises(lz.LmError, match="autograd"):
            call()
        with torch.no_grad():
            call()
        with torch.inference_mode():
            call()


def test_rel_bias_in_an_autograd_function(lz):
    """The way that the refusal names: the table's gradient is that of the formula."""
    H, L = 2, 50
    buckets = lz.rel_buckets(32, 128, "causal")

    class Bias(torch.autograd.Function):
        @staticmethod
        def forward(ctx, scores, table):
            return lz.rel_bias(table, buckets, L, L, add=scores)

        @staticmethod
        def backward(ctx, dout):
            # (softmax gives masked places no gradient)
            return dout, lz.rel_bias_grad(dout.contiguous(), buckets)
    table = torch.randn(32, H, device=DEV, requires_grad=True)
    scores = torch.randn(2, H, L, L, device=DEV, requires_grad=True)
    w = torch.randn(2, H, L, L, device=DEV)
    got = torch.autograd.grad((Bias.apply(scores, table).softmax(-1) * w).sum(), (scores, table))
    of = torch.tensor([[R.bucket(j - i, 32, 128, "causal") for j in range(L)] for i in range(L)],
                      device=DEV)
    s, t = scores.detach().double().requires_grad_(), table.detach().double().requires_grad_()
    x = (s + t[of.clamp(min=0)].permute(2, 0, 1)).masked_fill(of < 0, -float("inf"))
    want = torch.autograd.grad((x.softmax(-1) * w.double()).sum(), (s, t))
    for a, b in zip(got, want):
        # a softmax over at most 50 places and sums of under 5,000 terms: 1000 half steps
        assert float((a.double() - b).norm()) <= 1000 * 2.0 ** -24 * float(b.norm())


def test_writes_in_place_are_seen_by_autograd(lz):
    """A backward pass that saved a tensor which a call has written since raises."""
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8, device=DEV)  # noqa: E731
    f = lambda *n, d=torch.float32: torch.ones(*n, dtype=d, device=DEV)  # noqa: E731

    def raises(saved, write):
        x = f(*saved.shape, d=saved.dtype).requires_grad_()
        y = (x * saved).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    p = torch.nn.Parameter(f(50))
    copy = torch.nn.Parameter(f(50, d=torch.bfloat16))
    plan = lz.adamw_plan([p], [f(50)], [f(50)], [f(50)], copies=[copy])
    for t in (p, copy):
        raises(t, lambda: lz.adamw(plan))
    flat = f(100)
    plan = lz.adamw_plan([flat[:50], flat[50:90]], [f(50), f(40)], [f(50), f(40)], [f(50), f(40)])
    for t in (flat, flat[:50], flat[50:90], flat[90:]):
        raises(t, lambda: lz.adamw(plan))
    with torch.inference_mode():
        q = f(50)
    lz.adamw(lz.adamw_plan([q], [f(50)], [u8(50)], [u8(50)], m_scale=[u8(2)], v_scale=[u8(2)]))
    table = f(10, 40)
    raises(table, lambda: lz.sparse_apply_q8(
        table, u8(3).int(), torch.ones(1, dtype=torch.int64, device=DEV), f(3, 40), u8(10, 40),
        u8(10, 40), u8(10, 2), u8(10, 2)))
    buckets, scores, grad = lz.rel_buckets(32, 128, "both"), f(1, 2, 8, 8), f(32, 2)
    raises(scores, lambda: lz.rel_bias(f(32, 2), buckets, 8, 8, add=scores, out=scores))
    raises(grad, lambda: lz.rel_bias_grad(scores, buckets, out=grad))


@pytest.mark.parametrize("copies", [False, True])
def test_adamw_refuses_gradients_that_were_replaced(lz, copies):
    """After zero_grad() the parameters' (the bf16 copies') gradients are other memory: the plan
    would step the old ones. Gradients zeroed in place, and gradients of the caller's own, stay."""
    f = lambda n: torch.zeros(n, device=DEV)  # noqa: E731
    sizes = [50, 0, 70]
    p = [torch.nn.Parameter(f(n) + 1) for n in sizes]
    owners = [torch.nn.Parameter(t.detach().bfloat16()) for t in p] if copies else p

    def backward(x):
        sum((t * x).sum() for t in owners).backward()

    def plan():
        return lz.adamw_plan(p, [t.grad for t in owners], [f(n) for n in sizes],
                             [f(n) for n in sizes], copies=owners if copies else None)
    step = lambda a: lz.adamw(a, lr=0.5, beta1=0.0, beta2=0.0)  # noqa: E731
    mean = lambda: [float(t.detach().mean()) for t in p if t.numel()]  # noqa: E731
    backward(2.0)
    first = plan()
    step(first)
    assert mean() == pytest.approx([0.5, 0.5])
    for t in owners:
        t.grad.zero_()
    backward(-1.0)
    step(first)
    assert mean() == pytest.approx([1.0, 1.0])
    for t in owners:
        t.grad = None
    for _ in range(2):  # no gradients, then new ones
        with pytest.raises(lz.LmError, match="gradient"):
            step(first)
        assert mean() == pytest.approx([1.0, 1.0])
        backward(3.0)
    step(plan())
    assert mean() == pytest.approx([0.5, 0.5])
    owners[2].grad = None  # one of them is enough
    with pytest.raises(lz.LmError, match="gradient"):
        step(first)
    own = lz.adamw_plan(p, [f(n) - 1 for n in sizes], [f(n) for n in sizes], [f(n) for n in sizes])
    step(own)
    assert mean() == pytest.approx([1.0, 1.0])


# ---------------------------------------------------------------------------
# Every form of the 8-bit rows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("D", [2, 3, 4, 36, 40, 61, 96, 100, 127, 128, 129, 130, 255, 256, 257, 259,
                               260, 509, 512, 513, 516])
def test_rows8_widths(lz, idt, pad, D):
    """Rows of 8 to 64 lanes of 1 to 4 vectors, with ends inside a vector and lanes past the
    end: bit for bit, counts that are no multiple of a wave's or a workgroup's rows."""
    for V, U in ((400, 131), (9, 1), (60, 33)):
        adamw_tests.test_rows8(lz, idt, V, D, U, pad)


@pytest.mark.parametrize("D", [3, 40, 96, 130, 257, 513])
def test_rows8_from_blocks_of_one_large_value(lz, D):
    """The last value of each row far above its block: the lanes past the end, which hold values
    again, neither raise a block's scale nor lose it."""
    V, U = 50, 37
    rng = np.random.default_rng(D)
    p = rng.normal(0, 0.02, (V, D)).astype(np.float32)
    g = (rng.normal(0, 1, (U, D)) * 1e-6).astype(np.float32)
    g[:, -1] = 100.0
    g[::2, D // 2] = 3.0
    ids = np.sort(rng.permutation(V)[:U])
    z = [np.zeros((V, n), np.uint8) for n in (D, D, M.blocks(D), M.blocks(D))]
    t = [torch.from_numpy(x).to(DEV) for x in (p, *z)]
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    hyper = (1e-2, 0.9, 0.999, 1e-8, 0.1, 1)
    for turn in range(3):
        lz.sparse_apply_q8(t[0], torch.from_numpy(ids).to(DEV), torch.tensor([U], device=DEV),
                           torch.from_numpy(g).to(DEV), *t[1:], lr=1e-2, weight_decay=0.1,
                           step=1, seed=turn, dev_err=err)
        number = ids[:, None].astype(np.uint64) * np.uint64(D) + np.arange(D, dtype=np.uint64)
        ref, bound, *new, _ = M.step8(p[ids], g, *[x[ids] for x in z], hyper, number, turn)
        for got, old, want in zip(t[1:], z, new):
            old[ids] = want
            assert np.array_equal(got.cpu().numpy(), old), turn
        got = t[0].cpu().numpy()
        assert (np.abs(got[ids].astype(np.float64) - ref) <= bound).all(), turn
        p = got
    lz.check(err)
