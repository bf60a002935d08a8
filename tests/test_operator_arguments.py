"""Host-side checks of what the AdamW and relative-bias entry points accept (no GPU):
calls that are refused return before anything is launched."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")
P, I64, I32, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
INVAL = 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_1810_10045_amd import build
        build.build()
    L = ctypes.CDLL(LIB)
    L.lm_rel_buckets.argtypes = [I32, I32, I32, P, P, P]
    L.lm_rel_bias.argtypes = [P, I64, I32, P, P, I32, I64, I64, I64, I64, I64, P, P, P, P, I32, P]
    L.lm_rel_bias_grad.argtypes = [P, I32, I64, I64, I64, I64, P, I64, P, P, I32, I32, P, I64, I32,
                                   P, SZ, P]
    return L


class Bias:
    """lm_rel_bias and lm_rel_bias_grad on made-up addresses (the host reads none of them)."""

    def __init__(self, lib):
        self.lib, self.starts, self.ids, n = lib, (I32 * 257)(), (I32 * 257)(), I32()
        assert lib.lm_rel_buckets(32, 128, 0, self.starts, self.ids, ctypes.byref(n)) == 0
        self.n = n.value

    def bias(self, shape, out, out_strides, add=None, add_strides=None, dtype=0):
        s = lambda x: None if x is None else (I64 * 3)(*x)  # noqa: E731
        return self.lib.lm_rel_bias(P(0x1000), shape[1], 32, self.starts, self.ids, self.n, *shape,
                                    0, add, s(add_strides), out, s(out_strides), dtype, None)

    def grad(self, shape, strides):
        return self.lib.lm_rel_bias_grad(P(0x100000), 0, *shape, (I64 * 3)(*strides), 0,
                                         self.starts, self.ids, self.n, 32, P(0x1000), shape[1], 0,
                                         P(0x2000), 1 << 40, None)


def test_rel_bias_strides_past_64_bits(lib):
    """A span of strides that does not fit in 63 bits: rows that meet are not let through by
    its wrapping around, and nothing that no memory holds is read."""
    f = Bias(lib)
    far, v = 1 << 40, P(0x100000)
    # (2^24 - 1) 2^40 wraps to a number below zero; b = 1, h = 0 and b = 0, h = 1 are one row
    assert f.bias((1 << 24, 2, 1, 1), v, (far, far, 1)) == INVAL
    assert f.bias((1 << 24, 2, 1, 1), v, (far, far - 1, 1)) == INVAL
    for shape, strides in (((1 << 24, 1, 1, 1), (far, 1, 1)), ((1, 1, 1 << 24, 4), (0, 0, far)),
                           ((2, 1 << 10, 1 << 21, 1), (1, far, far))):
        whole = (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])
        assert f.bias(shape, v, whole, P(1 << 44), strides) == INVAL
        assert f.grad(shape, strides) == INVAL


LAUNCHES = r"""
#include "launch_parts.hpp"
extern "C" int64_t parts(int64_t blocks, int threads, int fail_at, uint32_t* first, uint32_t* n,
                         int room) {
  int k = 0;
  const int rc = lmz::launch_parts(blocks, threads, [&](uint32_t f, uint32_t c) {
    if (k < room) first[k] = f, n[k] = c;
    return ++k == fail_at ? 4 : 0;
  });
  return rc * 1000 + k;
}
"""


def test_launches_stay_below_2_32_threads(tmp_path):
    """Every workgroup in one launch, and no launch of 2^32 threads."""
    (tmp_path / "parts.cpp").write_text(LAUNCHES)
    so = str(tmp_path / "parts.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_1810_10045_amd", "csrc"), "-o", so,
                    str(tmp_path / "parts.cpp")], check=True)
    f = ctypes.CDLL(so).parts
    f.argtypes, f.restype = [I64, I32, I32, P, P, I32], I64
    for threads in (256, 1024):
        most = (1 << 32) // threads - 1
        for blocks in (0, 1, 5, most - 1, most, most + 1, 2 * most, 2 * most + 1, (1 << 31) - 1):
            first, n = (ctypes.c_uint32 * 600)(), (ctypes.c_uint32 * 600)()
            k = f(blocks, threads, 0, first, n, 600)
            assert k == -(-blocks // most)
            at = 0
            for i in range(k):
                assert first[i] == at and 0 < n[i] * threads < 1 << 32
                at += n[i]
            assert at == blocks
    first, n = (ctypes.c_uint32 * 8)(), (ctypes.c_uint32 * 8)()
    assert f(1 << 26, 256, 2, first, n, 8) == 4002, "an error ends the launches"


MEET = r"""
#include "rows_meet.hpp"
extern "C" int meet(const int64_t* n, int64_t Lk, const int64_t* out, const int64_t* add,
                    int64_t at) {
  return static_cast<int>(lmz::rows_meet(n, Lk, out, add, at));
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("meet")
    (d / "meet.cpp").write_text(MEET)
    so = str(d / "meet.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_1810_10045_amd", "csrc"), "-o", so,
                    str(d / "meet.cpp")], check=True)
    f = ctypes.CDLL(so).meet
    f.argtypes = [P, I64, P, P, I64]
    return lambda n, Lk, out, add, at: f((I64 * 3)(*n), Lk, (I64 * 3)(*out), (I64 * 3)(*add), at)


def _places(n, Lk, s, at):
    i = [np.arange(k) * x for k, x in zip(n, s)]
    x = i[0][:, None, None, None] + i[1][:, None, None] + i[2][:, None] + np.arange(Lk)
    return set((x + at).ravel().tolist())


def _outs(rng, n, Lk):
    """Strides of rows that do not meet, in any order of the dimensions, with gaps."""
    s, inside = [0, 0, 0], Lk
    for d in rng.permutation(3):
        s[d] = inside + int(rng.integers(0, 4))
        if n[d] > 1:
            inside += (n[d] - 1) * s[d]
    return s


def test_rows_meet_as_counted(meet):
    """Against the elements themselves: equal strides (interleaved halves, shifts), strides in
    another order, repeated dimensions."""
    rng = np.random.default_rng(3)
    seen = {0: 0, 1: 0}
    for turn in range(6000):
        n, Lk = [int(x) for x in rng.integers(1, 5, 3)], int(rng.integers(1, 5))
        out = _outs(rng, n, Lk)
        add = list(out) if turn % 3 == 0 else _outs(rng, n, Lk) if turn % 3 == 1 else \
            [int(x) for x in rng.integers(0, 12, 3)]
        a = _places(n, Lk, out, 0)
        at = int(rng.integers(-max(a) - 3, max(a) + 4))
        if turn % 6 == 0:
            at = int(rng.integers(-2 * Lk, 2 * Lk + 1))
        want = bool(a & _places(n, Lk, add, at))
        assert meet(n, Lk, out, add, at) == want, (n, Lk, out, add, at)
        seen[want] += 1
    assert min(seen.values()) > 1000
    # two halves of a buffer's rows, of its heads; one element further; more rows than are tried
    assert meet([8, 16, 2048], 2048, [1 << 27, 1 << 23, 4096], [1 << 27, 1 << 23, 4096], 2048) == 0
    assert meet([8, 16, 2048], 2048, [1 << 27, 1 << 23, 4096], [1 << 27, 1 << 23, 4096], 2047) == 1
    assert meet([8, 16, 2048], 2048, [1 << 27, 1 << 22, 2048], [1 << 27, 1 << 22, 2048], 1 << 26) == 0
    assert meet([1 << 20, 16, 8], 4, [512, 32, 4], [512, 4, 64], 3) == 2
    assert meet([1 << 24, 1 << 8, 1 << 8], 1, [1 << 40, 1 << 8, 1], [1 << 40, 1 << 8, 1], 1 << 16) == 0


def test_rel_bias_refuses_scores_that_meet_the_output(lib):
    """The output over other rows of the scores; in place and side by side is taken (tried
    above: taken calls are launched)."""
    f = Bias(lib)
    v, shape, s = 1 << 20, (2, 3, 4, 8), (96, 32, 8)
    for dtype, size in ((0, 4), (1, 2)):
        for at in (size, -size, 32 * size, 7 * size, 191 * size, -191 * size):
            assert f.bias(shape, P(v), s, P(v + at), s, dtype) == INVAL
        # the same memory in another order, a repeated row of it
        assert f.bias(shape, P(v), s, P(v), (32, 64, 8), dtype) == INVAL
        assert f.bias(shape, P(v), s, P(v), (0, 0, 0), dtype) == INVAL
        assert f.bias((1 << 20, 16, 8, 4), P(v), (512, 32, 4), P(v), (512, 4, 64), dtype) == 5


def test_adamw_plan_names_an_entry_that_is_no_tensor():
    """A parameter without a gradient (None) is refused as other wrong entries are."""
    torch = pytest.importorskip("torch")
    from paper_1810_10045_amd import lmzipf as lz
    t = [torch.zeros(4), torch.zeros(4)]
    for name, i in (("grads", 0), ("grads", 1), ("m", 1), ("v", 0), ("copies", 1), ("m_scale", 0),
                    ("params", 1)):
        lists = dict(params=list(t), grads=list(t), m=list(t), v=list(t))
        lists.setdefault(name, list(t))[i] = None
        with pytest.raises(lz.LmError, match=f"{name}.{i}. must be a tensor"):
            lz.adamw_plan(**lists)
