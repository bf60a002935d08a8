"""Host-side checks of the AdamW and relative-bias entry points (no GPU): the
buckets against whole numbers and a formula, the numpy form of the 8-bit moments
against its definition, and the refusals, which return before anything is
launched."""
import ctypes
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as M  # noqa: E402
import relbias_ref as R  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")
P, I64, I32, SZ, F, U64 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t,
                           ctypes.c_float, ctypes.c_uint64)
MODES = {"both": 0, "past": 1, "causal": 2}
INVAL, WORKSPACE, UNSUPPORTED = 1, 3, 5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_1810_10045_amd import build
        build.build()
    L = ctypes.CDLL(LIB)
    L.lm_rel_buckets.argtypes = [I32, I32, I32, P, P, P]
    L.lm_rel_bias.argtypes = [P, I64, I32, P, P, I32, I64, I64, I64, I64, I64, P, P, P, P, I32, P]
    L.lm_rel_bias_grad_workspace_bytes.argtypes = [I64, I64, I64, I64, I32, I32]
    L.lm_rel_bias_grad_workspace_bytes.restype = SZ
    L.lm_rel_bias_grad.argtypes = [P, I32, I64, I64, I64, I64, P, I64, P, P, I32, I32, P, I64, I32,
                                   P, SZ, P]
    L.lm_adamw_plan_bytes.argtypes = [P, I64]
    L.lm_adamw_plan_bytes.restype = SZ
    L.lm_adamw_plan.argtypes = [P, P, P, P, P, P, P, P, P, I64, I32, I32, P, SZ, P]
    L.lm_adamw.argtypes = [P, SZ, I64, I32, I32, I32, F, F, F, F, F, I64, P, U64, P, P]
    L.lm_sparse_apply_q8.argtypes = [P, I64, I64, I64, P, I32, P, I64, P, I64, F, F, F, F, F, I64,
                                     P, P, I64, P, P, I64, U64, P, P]
    return L


def segments(lib, nb, far, mode):
    starts, ids, n = (I32 * 257)(), (I32 * 257)(), I32()
    assert lib.lm_rel_buckets(nb, far, MODES[mode], starts, ids, ctypes.byref(n)) == 0
    return list(starts[:n.value]), list(ids[:n.value])


@pytest.mark.parametrize("mode", ["both", "past", "causal"])
@pytest.mark.parametrize("nb,far", [(4, 3), (4, 50), (8, 5), (16, 100), (32, 128), (32, 2), (32, 9),
                                    (64, 777), (64, 40), (256, 1000), (256, 200), (32, 100_000)])
def test_rel_buckets(lib, nb, far, mode):
    n = nb // 2 if mode == "both" else nb
    if far <= n // 2:
        starts, ids, k = (I32 * 257)(), (I32 * 257)(), I32()
        assert lib.lm_rel_buckets(nb, far, MODES[mode], starts, ids, ctypes.byref(k)) == INVAL
        return
    starts, ids = segments(lib, nb, far, mode)
    assert starts[0] == -2 ** 31 and all(a < b for a, b in zip(starts, starts[1:]))
    rels = sorted({s + d for s in starts[1:] for d in (-2, -1, 0, 1, 2)} |
                  set(range(-300, 300)) | {-2 ** 30, 2 ** 30, -far, far})
    for r in rels:
        s = max(i for i, a in enumerate(starts) if a <= r)
        assert ids[s] == R.bucket(r, nb, far, mode), (r, ids[s])


def test_rel_buckets_formula():
    """The whole-number borders are the logarithm's, away from ties."""
    for n, far in ((16, 128), (32, 128), (32, 777)):
        near = n // 2
        for d in range(near, 2000):
            x = math.log(d / near) / math.log(far / near) * (n - near)
            if abs(x - round(x)) > 1e-9:
                assert R.bucket(-d, n, far, "past") == min(near + math.floor(x), n - 1), (n, far, d)
    # ties, by hand: 16 buckets a side, 8 near ones, far 128 = 8 * 16: 8 steps of 16^(1/8)
    assert [R.bucket(-d, 16, 128, "past") for d in (7, 8, 15, 16, 31, 32, 63, 64, 127, 128, 10 ** 6)] \
        == [7, 8, 9, 10, 11, 12, 13, 14, 15, 15, 15]


def test_rel_buckets_refusals(lib):
    starts, ids, n = (I32 * 257)(), (I32 * 257)(), I32()
    call = lambda nb, far, mode, s=starts, i=ids, k=ctypes.byref(n): \
        lib.lm_rel_buckets(nb, far, mode, s, i, k)  # noqa: E731
    assert call(32, 128, 3) == UNSUPPORTED and call(257, 1000, 1) == UNSUPPORTED
    assert call(32, 1 << 24, 1) == UNSUPPORTED
    assert call(33, 128, 0) == INVAL and call(2, 128, 0) == INVAL and call(1, 128, 1) == INVAL
    assert call(0, 128, 1) == INVAL and call(-4, 128, 0) == INVAL
    assert call(32, 16, 1) == INVAL and call(32, 8, 0) == INVAL and call(32, -1, 1) == INVAL
    assert call(32, 128, 0, s=None) == INVAL and call(32, 128, 0, i=None) == INVAL
    assert call(32, 128, 0, k=None) == INVAL


def test_rel_bias_refusals(lib):
    starts, ids, n = (I32 * 257)(), (I32 * 257)(), I32()
    lib.lm_rel_buckets(32, 128, 0, starts, ids, ctypes.byref(n))
    n = n.value
    S = lambda *s: (I64 * 3)(*s)  # noqa: E731
    v = P(0x1000)

    def bias(table=v, ld=2, nb=32, st=starts, i=ids, k=n, B=1, H=2, Lq=4, Lk=8, q=0, add=None,
             sa=None, out=v, so=S(64, 32, 8), dtype=0):
        return lib.lm_rel_bias(table, ld, nb, st, i, k, B, H, Lq, Lk, q, add, sa, out, so, dtype,
                               None)

    def grad(dout=v, dtype=0, B=64, H=2, Lq=4, Lk=8, s=S(64, 32, 8), q=0, st=starts, i=ids, k=n,
             nb=32, d=v, ld=2, ws=v, nbytes=1 << 30):
        return lib.lm_rel_bias_grad(dout, dtype, B, H, Lq, Lk, s, q, st, i, k, nb, d, ld, 0, ws,
                                    nbytes, None)
    for f in (bias, grad):
        assert f(dtype=2) == UNSUPPORTED and f(B=-1) == INVAL and f(Lk=-1) == INVAL
        assert f(ld=1) == INVAL and f(q=(1 << 30) + 1) == UNSUPPORTED
        assert f(q=-(1 << 30) - 1) == UNSUPPORTED
        assert f(Lq=(1 << 24) + 1) == UNSUPPORTED
        assert f(B=1 << 24, H=1 << 24) == UNSUPPORTED and f(Lq=1 << 24, Lk=1 << 24) == UNSUPPORTED
        assert f(k=0) == INVAL and f(k=258) == UNSUPPORTED and f(nb=0) == INVAL
        assert f(nb=257) == UNSUPPORTED and f(nb=31) == INVAL  # ids reach 31
        assert f(st=None) == INVAL and f(i=None) == INVAL
        low = (I32 * 257)(*starts)
        low[0] = -5
        assert f(st=low) == INVAL
        low = (I32 * 257)(*starts)
        low[3] = low[2]
        assert f(st=low) == INVAL
        bad = (I32 * 257)(*ids)
        bad[1] = -2
        assert f(i=bad) == INVAL
    assert bias(table=None) == INVAL and bias(out=None) == INVAL and bias(so=None) == INVAL
    assert bias(out=P(0x1002)) == INVAL and bias(dtype=1, out=P(0x1001)) == INVAL
    # rows that meet: a row stride below Lk, a head inside a row, a repeated batch entry
    assert bias(so=S(64, 32, 7)) == INVAL and bias(so=S(64, 4, 8)) == INVAL
    assert bias(B=2, so=S(0, 32, 8)) == INVAL and bias(so=S(64, 32, -8)) == INVAL
    assert bias(add=v, sa=None) == INVAL and bias(add=v, sa=S(64, -1, 8)) == INVAL
    assert bias(add=P(0x1002), sa=S(64, 32, 8)) == INVAL
    assert grad(dout=None) == INVAL and grad(d=None) == INVAL and grad(ws=None) == INVAL
    assert grad(s=None) == INVAL and grad(s=S(64, 32, -8)) == INVAL and grad(dout=P(0x1002)) == INVAL
    assert grad(ws=P(0x1002)) == INVAL and grad(nbytes=3) == WORKSPACE
    # nothing to do: no launch
    assert bias(Lq=0) == 0 and bias(B=0) == 0 and bias(H=0) == 0 and grad(H=0) == 0
    q = lib.lm_rel_bias_grad_workspace_bytes
    assert q(64, 2, 4, 8, 0, n) >= 4 * 2 * n and q(1, 2, 4, 8, 0, n) == 0 and q(1, 2, 0, 8, 0, n) == 0
    assert q(1, 2, 4, 8, 7, n) == 0 and q(-1, 2, 4, 8, 0, n) == 0 and q(1, 2, 4, 8, 0, 0) == 0


def _plan(lib, sizes, states=32, gtype=0, tensors=None, shift=None, drop=None, short=0, copies=False,
          scales=None):
    """lm_adamw_plan on made-up addresses (the host reads none of them)."""
    k = len(sizes)
    sz = (I64 * k)(*sizes)
    at, lists = 1 << 20, {}
    for name, size in (("p", 4), ("g", 2 if gtype else 4), ("m", 4 if states == 32 else 1),
                       ("v", 4 if states == 32 else 1), ("ms", 1), ("vs", 1), ("c", 2)):
        a = (P * k)()
        for i, n in enumerate(sizes):
            a[i] = at
            at += max(n, 0) * size + 16
            at -= at % 16
        lists[name] = a
    if scales is None:
        scales = states == 8
    if not scales:
        lists["ms"] = lists["vs"] = None
    if not copies:
        lists["c"] = None
    if shift:
        lists[shift[0]][shift[1]] = shift[2](lists)
    if drop:
        lists[drop] = None
    need = lib.lm_adamw_plan_bytes(sz, k)
    buf = (ctypes.c_uint64 * (need // 8 + 2))()
    chunks = I64(-1)
    rc = lib.lm_adamw_plan(lists["p"], lists["g"], lists["m"], lists["v"], lists["ms"], lists["vs"],
                           lists["c"], sz, None, k if tensors is None else tensors, gtype, states,
                           buf, need - short, ctypes.byref(chunks))
    return rc, chunks.value


def test_adamw_plan(lib):
    assert _plan(lib, [1, 2048, 2049, 0, 5000]) == (0, 1 + 1 + 2 + 0 + 3)
    assert _plan(lib, [0, 0]) == (0, 0)
    assert _plan(lib, [100] * 500, states=8, gtype=1, copies=True) == (0, 500)
    for kw in (dict(states=16), dict(gtype=2)):
        assert _plan(lib, [100], **kw)[0] == UNSUPPORTED
    assert _plan(lib, [100], states=8, scales=False)[0] == INVAL
    assert _plan(lib, [100], states=32, scales=True)[0] == INVAL
    assert _plan(lib, [100], short=1)[0] == WORKSPACE
    assert _plan(lib, [100], tensors=-1)[0] == INVAL
    for name in "pgmv":
        assert _plan(lib, [100], drop=name)[0] == INVAL
        assert _plan(lib, [100, 50], shift=(name, 1, lambda a: None))[0] == INVAL
        assert _plan(lib, [100, 50], shift=(name, 1, lambda a: 0x900001))[0] == INVAL  # no element's


def test_adamw_plan_refuses_memory_that_meets(lib):
    for states, names in ((32, "pmv"), (8, ("p", "m", "v", "ms", "vs", "c"))):
        kw = dict(states=states, copies=states == 8)
        for x in names:
            for y in names:
                if x != y:  # tensor 1's x right at the last element of tensor 0's y
                    size = {"p": 4, "c": 2}.get(y, 4 if states == 32 else 1)
                    n = 4 if y in ("ms", "vs") else 100
                    end = lambda a, y=y, s=size, n=n: (a[y][0] + s * n - 1) // 4 * 4  # noqa: E731
                    assert _plan(lib, [100, 50], shift=(x, 1, end), **kw)[0] == INVAL, (x, y)
        # a gradient inside a parameter; one gradient for two tensors is read only
        assert _plan(lib, [100, 50], shift=("g", 1, lambda a: a["p"][0] + 40), **kw)[0] == INVAL
        assert _plan(lib, [100, 50], shift=("g", 1, lambda a: a["g"][0] + 40), **kw)[0] == 0
    # an empty tensor's addresses are not looked at
    assert _plan(lib, [100, 0], shift=("p", 1, lambda a: a["p"][0] + 1))[0] == 0


def test_adamw_plan_bytes(lib):
    q = lambda *s: lib.lm_adamw_plan_bytes((I64 * len(s))(*s), len(s))  # noqa: E731
    assert q() > 0 and q(0) > 0 and q(5) > 0 and q(5, 5) > q(5) and q(10_000) > q(5)
    assert q(-1) == 0 and q((1 << 42) + 1) == 0 and q(1 << 41, (1 << 41) + 1) == 0
    assert lib.lm_adamw_plan_bytes(None, 1) == 0 and lib.lm_adamw_plan_bytes(None, -1) == 0


def test_adamw_refusals(lib):
    v = P(0x1000)

    def step(plan=v, nbytes=1 << 20, chunks=1, gtype=0, states=32, b1=0.9, b2=0.999, t=1):
        return lib.lm_adamw(plan, nbytes, chunks, gtype, states, 0, 1e-3, b1, b2, 1e-8, 0.0, t,
                            None, 0, None, None)
    assert step(gtype=2) == UNSUPPORTED and step(states=4) == UNSUPPORTED
    assert step(nbytes=79) == WORKSPACE and step(chunks=-1) == INVAL and step(chunks=1 << 31) == INVAL
    assert step(plan=None) == INVAL and step(plan=P(0x1004)) == INVAL
    assert step(b1=1.0) == INVAL and step(b2=-1.0) == INVAL and step(b1=float("nan")) == INVAL
    assert step(t=0) == INVAL and step(chunks=0, plan=None) == 0

    def rows(table=v, V=10, D=40, ld=40, ids=v, idt=0, n=v, cap=3, vals=v, ldv=40, b1=0.9, t=1,
             m=v, mv=v, ldc=40, ms=v, vs=v, lds=2):
        return lib.lm_sparse_apply_q8(table, V, D, ld, ids, idt, n, cap, vals, ldv, 1e-3, b1, 0.999,
                                      1e-8, 0.0, t, m, mv, ldc, ms, vs, lds, 0, None, None)
    assert rows(idt=2) == UNSUPPORTED and rows(cap=1 << 31) == UNSUPPORTED
    assert rows(D=(1 << 24) + 1, ld=1 << 25, ldv=1 << 25,
                                               ldc=1 << 25, lds=1 << 25) == UNSUPPORTED
    for bad in (dict(V=-1), dict(D=-1), dict(cap=-1), dict(ld=39), dict(ldv=39), dict(ldc=39),
                dict(lds=1), dict(b1=1.0), dict(t=0), dict(table=None), dict(ids=None),
                dict(n=None), dict(vals=None), dict(m=None), dict(mv=None), dict(ms=None),
                dict(vs=None)):
        assert rows(**bad) == INVAL, bad
    assert rows(cap=0) == 0 and rows(D=0) == 0 and rows(V=0) == 0


def test_reference_moments():
    """The numpy form against its definition, by hand and by bounds."""
    x = np.array([448.0, 3.3, -0.01, 2.0 ** -9 * 0.4, 0.0], np.float32)
    codes, scale = M.encode(x, np.zeros(5), False)
    assert scale.tolist() == [127] and M.decode(codes, scale).tolist() == [448, 3.25, -0.009765625, 0, 0]
    codes, scale = M.encode(np.abs(x), np.full(5, 1 - 2.0 ** -20), True)
    assert M.decode(codes, scale).tolist() == [448, 3.5, 0.01171875, 2.0 ** -9, 0]
    assert M.encode(np.float32([448.0 * 1.0001]), np.zeros(1), False)[1].tolist() == [128]
    assert M.encode(np.float32([0.0]), np.zeros(1), True)[1].tolist() == [0]
    assert M.encode(np.float32([2.0 ** -140]), np.zeros(1), True)[1].tolist() == [0]
    rng = np.random.default_rng(1)
    y = (rng.normal(0, 1, 3200) * np.exp2(rng.integers(-60, 60, 100)).repeat(32)).astype(np.float32)
    got = M.decode(*M.encode(y, rng.random(3200), False))
    top = np.abs(y).reshape(-1, 32).max(1).repeat(32)
    assert (np.abs(got - y) <= np.maximum(np.abs(y) / 8, top * 2.0 ** -16)).all()
    w = M.words(np.arange(1 << 16), 5)
    for shift in (0, 12, 31):  # each bit half set, neighbours unrelated
        bit = (w >> np.uint32(shift)) & np.uint32(1)
        assert abs(bit.mean() - 0.5) < 6 * 0.5 / 256
        assert abs((bit[1:] ^ bit[:-1]).mean() - 0.5) < 6 * 0.5 / 256
    assert len(np.unique(M.words(np.arange(1 << 16), 5) ^ M.words(np.arange(1 << 16), 6))) > 1 << 15
