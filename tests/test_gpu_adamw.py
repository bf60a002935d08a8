"""GPU parity of the AdamW step over many tensors and of the lazy step on table
rows with 8-bit moments. Codes and scale bytes are held to a numpy computation
bit for bit, parameters to 64 bits within the roundings of the fp32 step."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as R  # noqa: E402
from paper_1810_10045_amd import synth  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
HYPER = (1e-2, 0.9, 0.999, 1e-8, 0.1, 7)  # lr, beta1, beta2, eps, weight decay, step
SIZES = [0, 1, 2, 3, 4, 5, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 4093, 4096,
         4097, 12_345]


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.device_powers(torch)
    return lmzipf


def _kw(hyper=HYPER):
    return dict(zip(("lr", "beta1", "beta2", "eps", "weight_decay", "step"), hyper))


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


class Flat:
    """Tensors of given sizes in one buffer with `gap` filler elements before and
    behind each, which no call may change."""

    def __init__(self, sizes, gap, dtype, values):
        total = sum(sizes) + gap * (len(sizes) + 1)
        self.flat = torch.full((total,), 0x55, dtype=torch.uint8, device=DEV) \
            if dtype == torch.uint8 else torch.full((total,), 77.0, dtype=dtype, device=DEV)
        self.views, self.spans, at = [], [], gap
        for n, x in zip(sizes, values):
            view = self.flat[at:at + n]
            view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(DEV))
            self.views.append(view)
            self.spans.append((at, n))
            at += n + gap
        self.filler = torch.ones(total, dtype=torch.bool, device=DEV)
        for a, n in self.spans:
            self.filler[a:a + n] = False
        self.before = self.flat[self.filler].clone()

    def check_filler(self):
        assert torch.equal(self.flat[self.filler], self.before), "written outside the tensors"


def _inputs(sizes, seed, bf16):
    rng = np.random.default_rng(seed)
    p = [rng.normal(0, 0.02, n).astype(np.float32) for n in sizes]
    g = [(rng.normal(0, 1, n) * np.exp(rng.normal(-5, 2, n))).astype(np.float32) for n in sizes]
    if bf16:
        g = [torch.from_numpy(x).bfloat16().float().numpy() for x in g]
    return rng, p, g


def _codes(rng, shape, signed):
    c = rng.integers(0, 0x7F, shape).astype(np.uint8)
    return c | (rng.integers(0, 2, shape).astype(np.uint8) << 7) if signed else c


def _run8(lz, sizes, gap, bf16, copies, seed, grad_scale=None, decay=None, hyper=HYPER, spoil=None,
          dev_err=None):
    rng, p, g = _inputs(sizes, seed, bf16)
    if spoil is not None:
        spoil(g)
    m, v = [_codes(rng, n, True) for n in sizes], [_codes(rng, n, False) for n in sizes]
    ms = [rng.integers(98, 110, R.blocks(n)).astype(np.uint8) for n in sizes]
    vs = [rng.integers(98, 112, R.blocks(n)).astype(np.uint8) for n in sizes]
    nb = [R.blocks(n) for n in sizes]
    u8 = torch.uint8
    f = {"p": Flat(sizes, gap, torch.float32, p),
         "g": Flat(sizes, gap, torch.bfloat16 if bf16 else torch.float32, g),
         "m": Flat(sizes, gap, u8, m), "v": Flat(sizes, gap, u8, v),
         "ms": Flat(nb, gap, u8, ms), "vs": Flat(nb, gap, u8, vs)}
    if copies:
        f["c"] = Flat(sizes, gap, torch.bfloat16, [np.zeros(n, np.float32) for n in sizes])
    plan = lz.adamw_plan(f["p"].views, f["g"].views, f["m"].views, f["v"].views,
                         m_scale=f["ms"].views, v_scale=f["vs"].views,
                         copies=f["c"].views if copies else None, decay=decay)
    gs = None if grad_scale is None else torch.tensor([grad_scale], device=DEV)
    lz.adamw(plan, grad_scale=gs, seed=seed, dev_err=dev_err, **_kw(hyper))
    torch.cuda.synchronize()
    first = 0
    for i, n in enumerate(sizes):
        wd = hyper[4] if decay is None or decay[i] else 0.0
        gi = g[i] if grad_scale is None else g[i] * np.float32(grad_scale)
        number = first + np.arange(n)
        first += R.blocks(n) * 32
        if n == 0:
            continue
        ref, bound, m8, v8, ms8, vs8, left = R.step8(p[i], gi, m[i], v[i], ms[i], vs[i],
                                                     hyper[:4] + (wd,) + hyper[5:], number, seed)
        for name, want in (("ms", ms8), ("vs", vs8), ("m", m8), ("v", v8)):
            got = f[name].views[i].cpu().numpy()
            assert np.array_equal(got, want), (i, n, name, np.flatnonzero(got != want)[:5])
        got = f["p"].views[i].cpu().numpy()
        off = np.abs(got.astype(np.float64) - ref)
        assert (off <= bound).all(), (i, n, "p", (off / bound).max())
        assert np.array_equal(got[left], p[i][left])
        if copies:
            assert torch.equal(f["c"].views[i], f["p"].views[i].bfloat16())
    for x in f.values():
        x.check_filler()
    return f


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("gap", [1, 8])
def test_adamw8_list(lz, bf16, copies, gap):
    _run8(lz, SIZES, gap, bf16, copies, 11 + gap)


def test_adamw8_scale_decay_and_order(lz):
    """Gradient scale, weight decay for some tensors only, sizes in another order."""
    sizes = SIZES[::-1]
    _run8(lz, sizes, 3, False, True, 21, grad_scale=0.3, decay=[i % 3 > 0 for i in range(len(sizes))])
    _run8(lz, [70_001], 1, True, False, 22, grad_scale=2.0, decay=[False])


@pytest.mark.parametrize("hyper", [(1e-3, 0.0, 0.0, 1e-8, 0.0, 1), (0.0, 0.9, 0.95, 1e-6, 0.0, 1),
                                   (1e-3, 0.95, 0.999, 0.0, 0.01, 10 ** 9)])
def test_adamw8_hyper(lz, hyper):
    _run8(lz, [1000, 33], 2, False, False, 31, hyper=hyper)


def test_adamw8_from_zero_and_extremes(lz):
    """Zero state, zero gradients, blocks of zeros, tiny and huge values: still the numpy step."""
    n = 32 * 64
    rng = np.random.default_rng(41)
    p = rng.normal(0, 0.02, n).astype(np.float32)
    g = (rng.normal(0, 1, n) * np.exp2(np.repeat(rng.integers(-140, 60, n // 32), 32))
         ).astype(np.float32)
    g[:32] = 0
    g[64:96] = 1e-44
    g[96:128] = 1e18
    g[128] = 0
    m = np.zeros(n, np.uint8)
    v, ms, vs = m.copy(), np.zeros(n // 32, np.uint8), np.zeros(n // 32, np.uint8)
    t = [torch.from_numpy(x).to(DEV) for x in (p, g, m, v, ms, vs)]
    plan = lz.adamw_plan([t[0]], [t[1]], [t[2]], [t[3]], m_scale=[t[4]], v_scale=[t[5]])
    for step in (1, 2, 3):
        hyper = (1e-3, 0.9, 0.999, 1e-8, 0.0, step)
        lz.adamw(plan, seed=100 + step, **_kw(hyper))
        ref, bound, m, v, ms, vs, left = R.step8(p, g, m, v, ms, vs, hyper, np.arange(n), 100 + step)
        assert not left.any()
        for got, want in zip(t[2:], (m, v, ms, vs)):
            assert np.array_equal(got.cpu().numpy(), want), step
        p = t[0].cpu().numpy()
        assert (np.abs(p.astype(np.float64) - ref) <= bound).all(), step
    # a root is zero where the second moment is, also by underflow: (1 - b2) g^2 < 2^-150
    some = (np.float32(1) - np.float32(0.999)) * g * g > 0
    assert (v[some] > 0).all() and some.sum() > n // 4 and not v[:32].any() and not ms[0]


def test_adamw8_rounding_has_no_bias(lz):
    """The mean of many roundings of one value is the value: 2^20 uniform parts, each
    rounding within a step, so the mean of n of them is off by under 6 half steps / sqrt(n)."""
    n = 32 * 4096
    x = 1.0 + np.random.default_rng(5).random(n // 32).astype(np.float32) * 0.9
    g = np.full((n // 32, 32), 0, np.float32)
    g[:] = x[:, None]
    g[:, 0] = 448.0                 # the block's scale is 1: codes of g itself
    t = [torch.from_numpy(a).to(DEV) for a in
         (np.zeros(n, np.float32), g.reshape(-1), np.zeros(n, np.uint8), np.zeros(n, np.uint8),
          np.zeros(n // 32, np.uint8), np.zeros(n // 32, np.uint8))]
    plan = lz.adamw_plan([t[0]], [t[1]], [t[2]], [t[3]], m_scale=[t[4]], v_scale=[t[5]])
    total = {2: np.zeros((n // 32, 32)), 3: np.zeros((n // 32, 32))}
    rounds = 64
    for seed in range(rounds):
        for k in (2, 3, 4, 5):
            t[k].zero_()
        lz.adamw(plan, lr=0.0, beta1=0.0, beta2=0.0, step=1, seed=seed)
        for k in total:
            total[k] += R.decode(t[k].cpu().numpy(), t[k + 2].cpu().numpy()).reshape(-1, 32)
    for k, s in total.items():
        off = s[:, 1:] / rounds - x[:, None]
        each = np.abs(off.mean(1))     # 31 x 64 roundings of the same value
        assert each.max() <= 6 * 0.5 * 0.125 / np.sqrt(31 * rounds), (k, each.max())
        assert abs(off.mean()) <= 6 * 0.5 * 0.125 / np.sqrt(31 * rounds * n / 32), k
        assert off.std() > 0
    pair = np.corrcoef((total[2][:, 1:] / rounds - x[:, None]).ravel(),
                       (total[3][:, 1:] / rounds - x[:, None]).ravel())[0, 1]
    assert abs(pair) < 6 / np.sqrt(31 * n / 32), "the two moments' roundings go together"


@pytest.mark.parametrize("states", [32, 8])
def test_adamw_leaves_values_that_are_not_finite(lz, states):
    err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def spoil(g):
        g[0][[0, 3, 40]] = [np.nan, np.inf, -np.inf]
        g[1][:] = np.nan
        g[2][5] = 3e38  # its square overflows
    sizes = [100, 50, 64, 64]
    if states == 8:
        _run8(lz, sizes, 1, False, True, 51, spoil=spoil, dev_err=err)
    else:
        _run32(lz, sizes, 1, False, True, 51, spoil=spoil, dev_err=err)
    assert int(err.item()) == lz.DEVERR_NONFINITE
    with pytest.raises(lz.DeviceError):
        lz.check(err)


def test_adamw8_nothing_finite_changes_nothing(lz):
    n = 5000
    rng = np.random.default_rng(6)
    x = rng.normal(0, 1, n).astype(np.float32)
    m, ms = R.encode(x, rng.random(n), False)
    v, vs = R.encode(np.abs(x), rng.random(n), True)
    t = [torch.from_numpy(a).to(DEV) for a in (x, np.full(n, np.nan, np.float32), m, v, ms, vs)]
    plan = lz.adamw_plan([t[0]], [t[1]], [t[2]], [t[3]], m_scale=[t[4]], v_scale=[t[5]])
    lz.adamw(plan, seed=3, weight_decay=0.1)
    got = [a.cpu().numpy() for a in t]
    assert np.array_equal(got[0], x)
    # The values, not their codes: where a block's largest was rounded down to 224 = 448 / 2
    # the scale halves, and every code of the old grid, subnormals too, is a number of the new one.
    assert np.array_equal(R.decode(got[2], got[4]), R.decode(m, ms))
    assert np.array_equal(R.decode(got[3], got[5]), R.decode(v, vs))
    assert (got[4] <= ms).all() and (got[4].astype(int) >= ms.astype(int) - 1).all()


def _run32(lz, sizes, gap, bf16, copies, seed, grad_scale=None, decay=None, hyper=HYPER,
           spoil=None, dev_err=None):
    rng, p, g = _inputs(sizes, seed, bf16)
    if spoil is not None:
        spoil(g)
    m = [rng.normal(0, 1e-2, n).astype(np.float32) for n in sizes]
    v = [np.square(rng.normal(0, 1e-2, n)).astype(np.float32) for n in sizes]
    f = {"p": Flat(sizes, gap, torch.float32, p),
         "g": Flat(sizes, gap, torch.bfloat16 if bf16 else torch.float32, g),
         "m": Flat(sizes, gap, torch.float32, m), "v": Flat(sizes, gap, torch.float32, v)}
    if copies:
        f["c"] = Flat(sizes, gap, torch.bfloat16, [np.zeros(n, np.float32) for n in sizes])
    plan = lz.adamw_plan(f["p"].views, f["g"].views, f["m"].views, f["v"].views,
                         copies=f["c"].views if copies else None, decay=decay)
    gs = None if grad_scale is None else torch.tensor([grad_scale], device=DEV)
    lz.adamw(plan, grad_scale=gs, dev_err=dev_err, **_kw(hyper))
    torch.cuda.synchronize()
    for i, n in enumerate(sizes):
        if n == 0:
            continue
        wd = hyper[4] if decay is None or decay[i] else 0.0
        gi = g[i] if grad_scale is None else g[i] * np.float32(grad_scale)
        b1, b2 = (float(np.float32(b)) for b in hyper[1:3])
        with np.errstate(over="ignore", invalid="ignore"):
            left = ~np.isfinite((1 - np.float32(b2)) * gi * gi)
        gi = np.where(left, 0, gi).astype(np.float64)
        m1, v1 = b1 * m[i] + (1 - b1) * gi, b2 * v[i].astype(np.float64) + (1 - b2) * gi * gi
        ref, bound = R.parameter(p[i], gi, m[i], v1, m1, hyper[:4] + (wd,) + hyper[5:])
        got = {k: f[k].views[i].cpu().numpy() for k in "pmv"}
        for k, old in (("p", p[i]), ("m", m[i]), ("v", v[i])):
            assert np.array_equal(got[k][left], old[left]), (i, k)
        live = ~left
        # m: the product (1 - b1) g and the fused sum; v: its two products and the fused sum
        bm = 2.02 * R.U32 * (b1 * np.abs(m[i]) + (1 - b1) * np.abs(gi)) + 1e-45
        bv = 3.03 * R.U32 * v1 + 1e-45
        for k, want, most in (("p", ref, bound), ("m", m1, bm), ("v", v1, bv)):
            off = np.abs(got[k].astype(np.float64) - want)
            assert (off <= most)[live].all(), (i, n, k, (off / most)[live].max())
        if copies:
            assert torch.equal(f["c"].views[i], f["p"].views[i].bfloat16())
    for x in f.values():
        x.check_filler()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("gap", [1, 8])
def test_adamw32_list(lz, bf16, copies, gap):
    _run32(lz, SIZES, gap, bf16, copies, 61 + gap)


def test_adamw32_scale_and_decay(lz):
    _run32(lz, SIZES[::-1], 3, True, True, 71, grad_scale=0.25,
           decay=[i % 2 for i in range(len(SIZES))])


@pytest.mark.parametrize("D", [1024, 70])
def test_adamw32_is_sparse_apply_with_every_row(lz, D):
    V = 300
    t = [torch.randn(V, D, device=DEV) * s for s in (0.02, 1e-2, 1e-2)]
    t.append(t[2].square())
    p, g, m, v = t[0], t[1], t[2], t[3]
    q = [x.clone() for x in (p, m, v)]
    rows = torch.arange(V, dtype=torch.int32, device=DEV)
    n = torch.tensor([V], device=DEV)
    lz.sparse_apply(q[0], rows, n, g, "adam", m=q[1], v=q[2], **_kw())
    lz.adamw(lz.adamw_plan([p], [g], [m], [v]), **_kw())
    for a, b in zip((p, m, v), q):
        assert torch.equal(a, b)


def test_adamw_many_small_tensors(lz):
    rng = np.random.default_rng(81)
    _run8(lz, [int(x) for x in rng.integers(0, 200, 700)], 1, True, False, 82)


def test_adamw8_one_tensor_past_32_bits(lz):
    """A tensor of more than 2^32 values between two small ones: its last values, whose
    numbers and offsets pass 32 bits, and the tensor behind it."""
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    n, tail = (1 << 32) + 3 * 2048 + 37, 3 * 2048 + 37
    sizes = [33, n, 100]
    rng = np.random.default_rng(91)
    g = [rng.normal(0, 1e-2, k).astype(np.float32) for k in (33, tail, 100)]
    z = lambda k, d=torch.uint8: torch.zeros(k, dtype=d, device=DEV)  # noqa: E731
    p = [z(k, torch.float32) for k in sizes]
    grads = [z(k, torch.bfloat16) for k in sizes]
    for t, x in zip(grads, g):
        t[-len(x):] = torch.from_numpy(x).to(DEV)
    m, v = [z(k) for k in sizes], [z(k) for k in sizes]
    ms, vs = [z(R.blocks(k)) for k in sizes], [z(R.blocks(k)) for k in sizes]
    lz.adamw(lz.adamw_plan(p, grads, m, v, m_scale=ms, v_scale=vs), seed=4, **_kw())
    first = 0
    for i, k in enumerate(sizes):
        c = len(g[i])
        x = grads[i][-c:].float().cpu().numpy()
        zero, zb = np.zeros(c, np.uint8), np.zeros(R.blocks(c), np.uint8)
        number = np.arange(first + k - c, first + k, dtype=np.uint64)
        ref, bound, m8, v8, ms8, vs8, _ = R.step8(np.zeros(c, np.float32), x, zero, zero, zb, zb,
                                                  HYPER, number, 4)
        first += R.blocks(k) * 32
        for got, want in ((m, m8), (v, v8), (ms, ms8), (vs, vs8)):
            assert np.array_equal(got[i][-len(want):].cpu().numpy(), want), i
        off = np.abs(p[i][-c:].cpu().numpy().astype(np.float64) - ref)
        assert (off <= bound).all(), i
    assert not p[1][:-tail].any() and not v[1][:-tail].any()  # zero gradients move nothing


def test_adamw_refuses_another_list_with_the_plan(lz):
    """A plan used with other counts or types than it was made with steps nothing."""
    p, g, m, v = (torch.ones(5000, device=DEV) for _ in range(4))
    plan = lz.adamw_plan([p], [g], [m], [v])
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    for bad in (plan._replace(chunks=1), plan._replace(gtype=lz.BF16),
                plan._replace(states=8), plan._replace(copies=True)):
        err.zero_()
        lz.adamw(bad, dev_err=err)
        assert int(err.item()) == lz.DEVERR_CAPACITY
    assert all(bool((x == 1).all()) for x in (p, g, m, v))
    with pytest.raises(lz.LmError):  # more chunks than the plan holds
        lz.adamw(plan._replace(chunks=plan.chunks + 1), dev_err=err)


def test_adamw_plan_holds_its_memory(lz):
    """A parameter that is given other memory, and lists and plans that go away: a step
    goes to the memory the plan was made with, and nothing else is touched."""
    n = 300_000
    p = torch.nn.Parameter(torch.zeros(n, device=DEV))
    old = p.data
    g, m, v = (torch.ones(n, device=DEV) for _ in range(3))
    plan = lz.adamw_plan([p], [g], [m], [v])
    p.data = torch.full((n,), 5.0, device=DEV)
    del g, m, v
    rest = [torch.full((n,), 7.0, device=DEV) for _ in range(8)]  # would take freed memory
    lz.adamw(plan, lr=0.5, beta1=0.0, beta2=0.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lz.adamw(plan, lr=0.5, beta1=0.0, beta2=0.0, stream=side)
    with torch.cuda.stream(side):
        lz.adamw(plan, lr=0.5, beta1=0.0, beta2=0.0)
    del plan
    more = [torch.full((n,), 7.0, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    assert bool((p == 5).all()) and all(bool((x == 7).all()) for x in rest + more)
    assert float((old + 1.5).abs().max()) < 1e-6  # three updates of lr


def test_adamw_in_a_graph_and_on_another_stream(lz):
    """A captured step replayed between eager steps, the gradients rewritten in
    place: each equals the eager step from the same state."""
    sizes = [1000, 33, 4096 * 3 + 5]
    make = lambda s: [torch.randn(n, device=DEV) * s for n in sizes]  # noqa: E731
    p, g, m = make(0.02), make(1e-2), [torch.zeros(n, dtype=torch.uint8, device=DEV) for n in sizes]
    v = [x.clone() for x in m]
    ms = [torch.zeros(R.blocks(n), dtype=torch.uint8, device=DEV) for n in sizes]
    vs = [x.clone() for x in ms]
    state = [*p, *m, *v, *ms, *vs]
    plan = lz.adamw_plan(p, g, m, v, m_scale=ms, v_scale=vs)
    scale = torch.ones(1, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lz.adamw(plan, step=3, seed=9, grad_scale=scale, dev_err=err)
    for i in range(4):
        [x.normal_(0, 1e-2) for x in g]
        scale.fill_(1.0 + i)
        before = [x.clone() for x in state]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        after = [x.clone() for x in state]
        [x.copy_(y) for x, y in zip(state, before)]
        side.wait_stream(torch.cuda.current_stream())
        lz.adamw(plan, step=3, seed=9, grad_scale=scale, dev_err=err, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state, after)), i
    lz.check(err)


# ---------------------------------------------------------------------------
# Rows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("V,D,U,pad", [(500, 1024, 100, 0), (500, 512, 500, 0), (300, 70, 41, 3),
                                       (90, 1, 30, 1), (90, 31, 17, 5), (90, 32, 17, 0),
                                       (90, 33, 17, 0), (40, 1025, 13, 7), (9, 2500, 3, 0),
                                       (1, 5, 1, 0)])
def test_rows8(lz, idt, V, D, U, pad):
    seed = V + D
    rng = np.random.default_rng(seed)
    nb = R.blocks(D)
    wide = lambda a, n: torch.from_numpy(np.concatenate(  # noqa: E731
        [a, np.full((len(a), pad), 0x55, a.dtype)], 1)).to(DEV)[:, :n] if pad else \
        torch.from_numpy(a).to(DEV)
    p = rng.normal(0, 0.02, (V, D)).astype(np.float32)
    g = rng.normal(0, 1e-2, (U + 4, D)).astype(np.float32)
    m, v = _codes(rng, (V, D), True), _codes(rng, (V, D), False)
    ms = rng.integers(98, 110, (V, nb)).astype(np.uint8)
    vs = rng.integers(98, 112, (V, nb)).astype(np.uint8)
    ids = np.sort(rng.permutation(V)[:U])
    rows = torch.full((U + 4,), -5, dtype=idt, device=DEV)
    rows[:U] = torch.from_numpy(ids).to(DEV)
    t = [wide(p, D), wide(g, D), wide(m, D), wide(v, D), wide(ms, nb), wide(vs, nb)]
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    lz.sparse_apply_q8(t[0], rows, torch.tensor([U], device=DEV), t[1], t[2], t[3], t[4], t[5],
                       seed=seed, dev_err=err, **_kw())
    torch.cuda.synchronize()
    lz.check(err)
    number = ids[:, None].astype(np.uint64) * np.uint64(D) + np.arange(D, dtype=np.uint64)
    ref, bound, m8, v8, ms8, vs8, _ = R.step8(p[ids], g[:U], m[ids], v[ids], ms[ids], vs[ids],
                                              HYPER, number, seed)
    for got, old, want in ((t[4], ms, ms8), (t[5], vs, vs8), (t[2], m, m8), (t[3], v, v8)):
        old[ids] = want
        assert np.array_equal(got.cpu().numpy(), old)
    got = t[0].cpu().numpy()
    assert (np.abs(got[ids].astype(np.float64) - ref) <= bound).all()
    rest = np.setdiff1d(np.arange(V), ids)
    assert np.array_equal(got[rest], p[rest])
    if pad:
        for x in t:
            assert bool((x.as_strided((x.shape[0], pad), x.stride(), x.shape[1]) == 0x55).all())


def test_rows8_numbers_past_32_bits(lz):
    """Rows far down a wide table: their values' numbers pass 2^32."""
    V, D = 70_000, 65_536 + 32
    codes = torch.zeros(V, D, dtype=torch.uint8, device=DEV)
    free = torch.cuda.mem_get_info()[0]
    if free < 24 * V * D // 10 * 3:
        pytest.skip("needs 30 GB")
    table = torch.zeros(V, D, device=DEV)
    m, v = codes, torch.zeros_like(codes)
    ms = torch.zeros(V, R.blocks(D), dtype=torch.uint8, device=DEV)
    vs = torch.zeros_like(ms)
    ids = np.array([0, 65_470, 65_537, 69_999])
    g = np.random.default_rng(3).normal(0, 1e-2, (4, D)).astype(np.float32)
    lz.sparse_apply_q8(table, torch.from_numpy(ids).to(DEV), torch.tensor([4], device=DEV),
                       torch.from_numpy(g).to(DEV), m, v, ms, vs, seed=5, **_kw())
    z = np.zeros((4, D), np.uint8)
    zb = np.zeros((4, R.blocks(D)), np.uint8)
    number = ids[:, None].astype(np.uint64) * np.uint64(D) + np.arange(D, dtype=np.uint64)
    assert number.max() > 2 ** 32
    ref, bound, m8, v8, ms8, vs8, _ = R.step8(np.zeros((4, D), np.float32), g, z, z, zb, zb, HYPER,
                                              number, 5)
    at = torch.from_numpy(ids).to(DEV)
    for got, want in ((m, m8), (v, v8), (ms, ms8), (vs, vs8)):
        assert np.array_equal(got[at].cpu().numpy(), want)
    assert (np.abs(table[at].cpu().numpy().astype(np.float64) - ref) <= bound).all()


def test_rows8_data_errors(lz):
    """An id outside the table, a count above the capacity, values that are not finite."""
    V, D = 20, 40
    rng = np.random.default_rng(8)

    def run(ids, n, g):
        p = torch.ones(V, D, device=DEV)
        m, v = (torch.zeros(V, D, dtype=torch.uint8, device=DEV) for _ in range(2))
        ms, vs = (torch.zeros(V, 2, dtype=torch.uint8, device=DEV) for _ in range(2))
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        lz.sparse_apply_q8(p, torch.tensor(ids, device=DEV), torch.tensor([n], device=DEV),
                           torch.from_numpy(g).to(DEV), m, v, ms, vs, lr=0.1, dev_err=err)
        moved = (p != 1).any(1).nonzero().flatten().tolist()
        assert (v != 0).any(1).nonzero().flatten().tolist() == moved
        return int(err.item()), moved, p
    g = rng.normal(1, 0.1, (3, D)).astype(np.float32)
    assert run([2, 5, 9], 3, g)[:2] == (0, [2, 5, 9])
    assert run([2, 20, -1], 3, g)[:2] == (lz.DEVERR_ID_RANGE, [2])
    assert run([2, 5, 9], 7, g)[:2] == (lz.DEVERR_CAPACITY, [2, 5, 9])
    assert run([2, 5, 9], 0, g)[:2] == (0, [])
    assert run([2, 5, 9], -4, g)[:2] == (0, [])
    g[1] = np.inf
    g[2, 7] = np.nan
    err, moved, p = run([2, 5, 9], 3, g)
    assert err == lz.DEVERR_NONFINITE and moved == [2, 9] and float(p[9, 7]) == 1


def test_rows8_step_after_segsum(lz):
    """Unique, Seg-Sum and the 8-bit step on the same rows as the fp32 step: from zero
    moments the first update is lr * g / (|g| + eps) in both."""
    K, V, D = 5000, 3000, 96
    ids = torch.from_numpy(synth.zipf_ids(K, V, 1.0, 7, np.int32)).to(DEV)
    grad = torch.from_numpy(synth.normal_rows(K, D, 8)).to(DEV)
    p0 = torch.from_numpy(synth.normal_rows(V, D, 9, 0.02)).to(DEV)
    u = lz.unique(ids, V)
    s = lz.segsum(grad, u.perm, u.inverse, u.offsets, u.num_unique, dev_err=u.dev_err)
    a, b = p0.clone(), p0.clone()
    z = lambda *n: torch.zeros(*n, dtype=torch.uint8, device=DEV)  # noqa: E731
    m, v, ms, vs = z(V, D), z(V, D), z(V, 3), z(V, 3)
    lz.sparse_apply_q8(a, u.uniq, u.num_unique, s, m, v, ms, vs, lr=1e-3, step=1, seed=1,
                       dev_err=u.dev_err)
    lz.sparse_apply(b, u.uniq, u.num_unique, s, "adam", lr=1e-3, step=1, m=torch.zeros_like(b),
                    v=torch.zeros_like(b), dev_err=u.dev_err)
    lz.check(u.dev_err)
    # one update of size lr from the same gradient: under 16 half steps of it, and the sum's
    assert float((a - b).abs().max()) <= 2 * R.U32 * (16 * 1e-3 + float(b.abs().max()))
    assert torch.equal((a != p0).any(1), (b != p0).any(1))


# ---------------------------------------------------------------------------
# Refusals of the binding
# ---------------------------------------------------------------------------
def test_adamw_plan_refusals(lz):
    t = lambda n=8, d=torch.float32: torch.zeros(n, dtype=d, device=DEV)  # noqa: E731
    ok = [t()], [t()], [t()], [t()]
    lz.adamw_plan(*ok)
    u8, bf = torch.uint8, torch.bfloat16
    for bad, kw in (((([],) * 4), {}), (([t()], [t(), t()], [t()], [t()]), {}),
                    (([t(8, bf)], [t()], [t()], [t()]), {}),
                    (([t()], [t(8, torch.float16)], [t()], [t()]), {}),
                    (([t(), t()], [t(), t(8, bf)], [t(), t()], [t(), t()]), {}),
                    (([t()], [t(7)], [t()], [t()]), {}),
                    (([t()], [t()], [t(16)[::2]], [t()]), {}),
                    (([t()], [t()], [t(8, u8)], [t(8, u8)]), {}),
                    (([t()], [t()], [t(8, u8)], [t(8, u8)]), {"m_scale": [t(1, u8)]}),
                    (([t()], [t()], [t()], [t()]), {"m_scale": [t(1, u8)], "v_scale": [t(1, u8)]}),
                    (([t()], [t()], [t(8, u8)], [t(8, u8)]),
                     {"m_scale": [t(2, u8)], "v_scale": [t(2, u8)]}),
                    (([t()], [t()], [t()], [t()]), {"copies": [t()]}),
                    (([t()], [t()], [t()], [t()]), {"decay": [1, 0]}),
                    (([t()], [t().cpu()], [t()], [t()]), {})):
        with pytest.raises(lz.LmError):
            lz.adamw_plan(*bad, **kw)
    x = t(20)
    with pytest.raises(lz.LmError):  # the parameter and its moment share memory
        lz.adamw_plan([x[:8]], [t()], [x[7:15]], [t()])
    with pytest.raises(lz.LmError):  # the same tensor twice
        lz.adamw_plan([x[:8]] * 2, [t()] * 2, [t(), t()], [t(), t()])
    with pytest.raises(lz.LmError):  # a gradient inside a parameter
        lz.adamw_plan([x[:8]], [x[4:12]], [t()], [t()])
    lz.adamw_plan([t(), t()], [x[:8]] * 2, [t(), t()], [t(), t()])  # gradients may be shared
    plan = lz.adamw_plan(*ok)
    for kw in ({"step": 0}, {"beta1": 1.0}, {"beta2": -0.1}, {"grad_scale": torch.ones(1)},
               {"grad_scale": torch.ones(1, device=DEV, dtype=torch.float64)},
               {"dev_err": torch.zeros(1, device=DEV)}):
        with pytest.raises(lz.LmError):
            lz.adamw(plan, **kw)


def test_rows8_refusals(lz):
    V, D = 10, 40
    z = lambda *n, d=torch.uint8: torch.zeros(*n, dtype=d, device=DEV)  # noqa: E731
    ok = dict(table=z(V, D, d=torch.float32), rows=z(3, d=torch.int32), n_rows=z(1, d=torch.int64),
              vals=z(3, D, d=torch.float32), m=z(V, D), v=z(V, D), m_scale=z(V, 2), v_scale=z(V, 2))
    lz.sparse_apply_q8(**ok)
    for bad in (dict(table=z(V, D, d=torch.bfloat16)), dict(vals=z(3, D, d=torch.bfloat16)),
                dict(vals=z(3, D + 1, d=torch.float32)), dict(m=z(V, D, d=torch.float32)),
                dict(v=z(V, D - 1)), dict(m_scale=z(V, 1)), dict(v_scale=z(V, 4)[:, ::2]),
                dict(rows=z(6, d=torch.int32)[::2]), dict(rows=z(3, d=torch.int16)),
                dict(n_rows=z(1, d=torch.int32)), dict(m=z(V, D).cpu()), dict(step=0),
                dict(beta2=1.0), dict(dev_err=z(1, d=torch.int64)),
                dict(m=z(V, D + 8)[:, :D])):
        with pytest.raises(lz.LmError):
            lz.sparse_apply_q8(**{**ok, **bad})
