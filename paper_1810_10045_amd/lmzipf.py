"""Thin ctypes binding of ``liblmzipf.so`` (C ABI in ``include/lmzipf.h``).

Argument marshalling only: every step runs in the HIP kernels of the library.
Tensors are torch CUDA tensors (PyTorch supplies device memory and the
current stream); nothing here computes on the host. If the library has not
been built, importing this module raises — there is no fallback path.

Entry points have the C names without the ``lm_`` prefix: ``unique``,
``segsum``, ``map_ids``, ``fill_values``, ``sparse_apply``, the binary16
payload forms ``fill_values_f16`` and ``sparse_apply_f16``, and
``sample_ids``; ``unique_workspace_bytes`` is the workspace query that
``unique`` makes itself, for callers that size a workspace up front.

Beside the embedding's path: ``adamw_plan`` and ``adamw`` (the AdamW step over
many tensors, moments in fp32 or 8 bits), ``sparse_apply_q8`` (the lazy step on
table rows with 8-bit moments), ``rel_buckets``, ``rel_bias`` and
``rel_bias_grad`` (a learned relative position bias and its gradient).
"""
from __future__ import annotations

import ctypes
import operator
import os
from typing import NamedTuple, Optional

import torch

# The current stream's handle (not a public name of torch: the public call where it is absent).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liblmzipf.so")

OK, E_INVAL, E_WORKSPACE, E_HIP, E_UNSUPPORTED = 0, 1, 3, 4, 5
DEVERR_ID_RANGE, DEVERR_NOT_FOUND, DEVERR_CAPACITY, DEVERR_SPIN = 1, 2, 4, 8
DEVERR_NONFINITE = 16
I32, I64 = 0, 1
F32, BF16 = 0, 1
FILL_EXPAND, FILL_SCATTER, FILL_SCATTER_ADD = 0, 1, 2
OPT_SGD, OPT_ADAM = 0, 1
REL_BOTH, REL_PAST, REL_CAUSAL = 0, 1, 2
MOMENT_BLOCK, REL_MAX_SEGMENTS = 32, 257
MAX_K = 1 << 30

EXPORTS = ("lm_status_string", "lm_abi_version", "lm_workspace_clear",
           "lm_unique_workspace_bytes", "lm_unique", "lm_segsum_workspace_bytes",
           "lm_segsum", "lm_map_ids", "lm_fill_values", "lm_sparse_apply",
           "lm_fill_values_f16", "lm_sparse_apply_f16", "lm_sample_ids",
           "lm_adamw_plan_bytes", "lm_adamw_plan", "lm_adamw", "lm_sparse_apply_q8",
           "lm_rel_buckets", "lm_rel_bias", "lm_rel_bias_grad_workspace_bytes",
           "lm_rel_bias_grad")


class LmError(RuntimeError):
    pass


class DeviceError(RuntimeError):
    """Raised by :func:`check` when a kernel reported a data error."""


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
            " (the HIP library is the only implementation of these entry points)")
    L = ctypes.CDLL(LIB_PATH)
    P, I64_, SZ, I32_, F = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t,
                           ctypes.c_int32, ctypes.c_float)
    L.lm_status_string.argtypes = [ctypes.c_int]
    L.lm_status_string.restype = ctypes.c_char_p
    L.lm_abi_version.argtypes = []
    L.lm_workspace_clear.argtypes = [P, SZ, P]
    L.lm_unique_workspace_bytes.argtypes = [I64_, I32_, I64_]
    L.lm_unique_workspace_bytes.restype = SZ
    L.lm_unique.argtypes = [P, I32_, I64_, I64_, P, P, P, P, P, P, P, P, SZ, P]
    L.lm_unique_noalloc.argtypes = [P, I32_, I64_, I64_, P, P, P, P, P, P, P, P]
    L.lm_segsum_workspace_bytes.argtypes = [I64_, I64_]
    L.lm_segsum_workspace_bytes.restype = SZ
    L.lm_segsum.argtypes = [P, I32_, I64_, I64_, I64_, P, P, P, P, I64_, P, I64_, P, P, SZ, P]
    L.lm_segsum_rows.argtypes = [P, I32_, I64_, I64_, I64_, P, P, P, P, P, I32_, I64_, P, I64_, I64_,
                                 P, P, SZ, P]
    L.lm_segsum_sgd.argtypes = [P, I32_, I64_, I64_, I64_, P, P, P, P, P, I32_, I64_, P, I64_, I64_,
                                F, P, P, SZ, P]
    L.lm_segsum_adam.argtypes = [P, I32_, I64_, I64_, I64_, P, P, P, P, P, I32_, I64_, P, I64_, I64_,
                                 F, F, F, F, F, I64_, P, P, P, P, SZ, P]
    L.lm_map_ids.argtypes = [P, P, I64_, P, P, I64_, I32_, P, P, P]
    L.lm_fill_values.argtypes = [P, I64_, P, P, I64_, P, P, I32_, I64_, P, I64_, I64_, I32_, P, P]
    L.lm_sparse_apply.argtypes = [P, I64_, I64_, I64_, P, I32_, P, I64_, P, I64_, I32_,
                                  F, F, F, F, F, I64_, P, P, P, P]
    L.lm_fill_values_f16.argtypes = [P, I64_, P, P, I64_, P, P, I32_, I64_, P, I64_, I64_, I32_,
                                     F, P, P]
    L.lm_sparse_apply_f16.argtypes = [P, I64_, I64_, I64_, P, I32_, P, I64_, P, I64_, F, I32_,
                                      F, F, F, F, F, I64_, P, P, P, P]
    L.lm_sample_ids.argtypes = [P, I64_, I64_, P, I32_, P]
    U64 = ctypes.c_uint64
    L.lm_adamw_plan_bytes.argtypes = [P, I64_]
    L.lm_adamw_plan_bytes.restype = SZ
    L.lm_adamw_plan.argtypes = [P, P, P, P, P, P, P, P, P, I64_, I32_, I32_, P, SZ, P]
    L.lm_adamw.argtypes = [P, SZ, I64_, I32_, I32_, I32_, F, F, F, F, F, I64_, P, U64, P, P]
    L.lm_sparse_apply_q8.argtypes = [P, I64_, I64_, I64_, P, I32_, P, I64_, P, I64_, F, F, F, F, F,
                                     I64_, P, P, I64_, P, P, I64_, U64, P, P]
    L.lm_rel_buckets.argtypes = [I32_, I32_, I32_, P, P, P]
    L.lm_rel_bias.argtypes = [P, I64_, I32_, P, P, I32_, I64_, I64_, I64_, I64_, I64_, P, P, P, P,
                              I32_, P]
    L.lm_rel_bias_grad_workspace_bytes.argtypes = [I64_, I64_, I64_, I64_, I32_, I32_]
    L.lm_rel_bias_grad_workspace_bytes.restype = SZ
    L.lm_rel_bias_grad.argtypes = [P, I32_, I64_, I64_, I64_, I64_, P, I64_, P, P, I32_, I32_, P,
                                   I64_, I32_, P, SZ, P]
    L.lm_segsum_set_two_launches.argtypes = [I32_]
    L.lm_test_force_wait_failure.argtypes = [I32_, ctypes.c_uint32]
    for f in ("lm_abi_version", "lm_workspace_clear", "lm_unique", "lm_unique_noalloc",
              "lm_segsum", "lm_segsum_rows", "lm_segsum_sgd", "lm_segsum_adam", "lm_map_ids",
              "lm_fill_values", "lm_sparse_apply", "lm_fill_values_f16", "lm_sparse_apply_f16",
              "lm_sample_ids", "lm_segsum_set_two_launches", "lm_test_force_wait_failure",
              "lm_adamw_plan", "lm_adamw", "lm_sparse_apply_q8", "lm_rel_buckets", "lm_rel_bias",
              "lm_rel_bias_grad"):
        getattr(L, f).restype = ctypes.c_int
    return L


_lib = _load()


def lib():
    return _lib


def status_string(rc: int) -> str:
    return _lib.lm_status_string(rc).decode()


def _call(rc: int, what: str):
    if rc != OK:
        raise LmError(f"{what}: {status_string(rc)}")


# The argument types above convert integers, so addresses and stream handles
# are passed as they are: a ctypes object for each of a call's 10 to 15
# pointers took 2 us of a call, and torch.cuda.current_stream(), which builds a
# Stream object to read the same handle from, 3.3 us (Unique and Seg-Sum of the
# smallest batches occupy the GPU for 17 us together).
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _idtype(t: torch.Tensor) -> int:
    if t.dtype == torch.int32:
        return I32
    if t.dtype == torch.int64:
        return I64
    raise LmError(f"word ids must be int32 or int64, got {t.dtype}")


def _gtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise LmError(f"gradients must be float32 or bfloat16, got {t.dtype}")


def _rows(t: torch.Tensor, what: str):
    if t.dim() != 2 or t.stride(1) != 1:
        raise LmError(f"{what} must be a 2-D tensor with unit column stride")
    return t.stride(0)


def _dev(t: torch.Tensor, what: str):
    if not t.is_cuda:
        raise LmError(f"{what} must be a CUDA (HIP) tensor")


class Workspace:
    """A device scratch buffer that grows on demand (no entry point needs
    particular initial contents). Torch's allocator returns 512-byte aligned
    blocks, above the 256 bytes the library asks for."""

    def __init__(self, device=None):
        self.device = torch.device(device or "cuda")
        self.buf = torch.empty(0, dtype=torch.uint8, device=self.device)

    def get(self, nbytes: int) -> torch.Tensor:
        nbytes = max(int(nbytes), 256)
        if self.buf.numel() < nbytes:
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self.buf


_default_ws = {}


def default_workspace(device) -> Workspace:
    key = torch.device(device)
    if key not in _default_ws:
        _default_ws[key] = Workspace(key)
    return _default_ws[key]


def check(dev_err: torch.Tensor):
    """Synchronise on dev_err and raise DeviceError if any kernel set a bit."""
    v = int(dev_err.item())
    if v:
        names = [n for b, n in ((DEVERR_ID_RANGE, "id out of range"),
                                (DEVERR_NOT_FOUND, "id not found"),
                                (DEVERR_CAPACITY, "capacity exceeded"),
                                (DEVERR_SPIN, "inter-workgroup wait gave up"),
                                (DEVERR_NONFINITE, "compressed value or second moment not finite")) if v & b]
        raise DeviceError(f"device error 0x{v:x}: {', '.join(names)}")


class UniqueResult(NamedTuple):
    uniq: torch.Tensor
    counts: torch.Tensor
    offsets: torch.Tensor
    inverse: torch.Tensor
    perm: torch.Tensor
    num_unique: torch.Tensor
    dev_err: torch.Tensor


def unique_buffers(K: int, V: int, id_dtype, device) -> UniqueResult:
    cap = max(1, min(K, V))
    z = dict(device=device)
    return UniqueResult(
        torch.empty(cap, dtype=id_dtype, **z), torch.empty(cap, dtype=torch.int32, **z),
        torch.empty(cap + 1, dtype=torch.int32, **z), torch.empty(max(K, 1), dtype=torch.int32, **z),
        torch.empty(max(K, 1), dtype=torch.int32, **z), torch.zeros(1, dtype=torch.int64, **z),
        torch.zeros(1, dtype=torch.int32, **z))


def _check_unique_out(out: UniqueResult, ids: torch.Tensor, V: int):
    """The output buffers must hold what the kernels write: min(K, V) types,
    one offset more, K inverse and perm entries, on the ids' device."""
    K = ids.numel()
    cap = min(K, V)
    dev, i32 = ids.device, torch.int32
    for t, n, dt in ((out.uniq, cap, ids.dtype), (out.counts, cap, i32), (out.offsets, cap + 1, i32),
                     (out.inverse, K, i32), (out.perm, K, i32), (out.num_unique, 1, torch.int64),
                     (out.dev_err, 1, i32)):
        if t.device != dev or t.dtype != dt or not t.is_contiguous() or t.numel() < n:
            raise LmError(f"unique output buffer: need {n} contiguous {dt} on {dev}")


def unique_workspace_bytes(K: int, V: int, id_dtype=torch.int32) -> int:
    """lm_unique_workspace_bytes: the workspace one lm_unique call of K ids
    of dtype id_dtype over [0, V) needs (0: the sizes are rejected)."""
    idt = I64 if id_dtype == torch.int64 else I32
    return int(_lib.lm_unique_workspace_bytes(K, idt, V))


def unique(ids: torch.Tensor, V: int, out: Optional[UniqueResult] = None,
           ws: Optional[Workspace] = None, stream=None) -> UniqueResult:
    """lm_unique: Sec. III-A steps 1/4. Returns device tensors; num_unique is
    a 1-element int64 tensor (no host sync)."""
    _dev(ids, "ids")
    K = ids.numel()
    idt = _idtype(ids)
    ids = ids.contiguous()
    if out is None:
        out = unique_buffers(K, V, ids.dtype, ids.device)
    _check_unique_out(out, ids, V)
    ws = ws or default_workspace(ids.device)
    need = _lib.lm_unique_workspace_bytes(K, idt, V)
    if need == 0 and K > 0:
        raise LmError("lm_unique_workspace_bytes rejected the sizes")
    buf = ws.get(need)
    _call(_lib.lm_unique(_ptr(ids), idt, K, V, _ptr(out.uniq), _ptr(out.counts), _ptr(out.offsets),
                         _ptr(out.inverse), _ptr(out.perm), _ptr(out.num_unique), _ptr(out.dev_err),
                         _ptr(buf), buf.numel(), _stream(stream)), "lm_unique")
    return out


UNIQUE_NOALLOC_MAX_K = 262144  # LM_UNIQUE_NOALLOC_MAX_K


def unique_noalloc(ids: torch.Tensor, V: int, out: UniqueResult, stream=None) -> UniqueResult:
    """lm_unique_noalloc: lm_unique with the library's own device workspace,
    for callers that cannot allocate. The outputs must be given (allocating
    them is the caller's business); at most UNIQUE_NOALLOC_MAX_K ids. Calls
    that overlap on one GPU share the workspace and race."""
    _dev(ids, "ids")
    if not ids.is_contiguous():
        raise LmError("ids must be contiguous (a copy would allocate)")
    K = ids.numel()
    _check_unique_out(out, ids, V)
    _call(_lib.lm_unique_noalloc(_ptr(ids), _idtype(ids), K, V, _ptr(out.uniq), _ptr(out.counts),
                                 _ptr(out.offsets), _ptr(out.inverse), _ptr(out.perm),
                                 _ptr(out.num_unique), _ptr(out.dev_err), _stream(stream)),
          "lm_unique_noalloc")
    return out


def segsum(grad: torch.Tensor, perm: torch.Tensor, inverse: torch.Tensor, offsets: torch.Tensor,
           num_unique: torch.Tensor, u_cap: Optional[int] = None,
           out: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None,
           ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """lm_segsum: Sec. III-A step 2. Returns the u_cap x D fp32 output (rows
    >= num_unique untouched)."""
    _dev(grad, "grad")
    K, D = grad.shape
    ld = _rows(grad, "grad")
    if u_cap is None:
        u_cap = offsets.numel() - 1
    if perm.numel() < K or inverse.numel() < K or offsets.numel() < 1:
        raise LmError("perm and inverse must hold K entries")
    if out is None:
        out = torch.empty((max(u_cap, 1), D), dtype=torch.float32, device=grad.device)
    if out.shape[0] < u_cap or out.shape[1] != D:
        raise LmError("out must be at least u_cap x D")
    ld_out = _rows(out, "out")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=grad.device)
    ws = ws or default_workspace(grad.device)
    buf = ws.get(_lib.lm_segsum_workspace_bytes(K, D))
    _call(_lib.lm_segsum(_ptr(grad), _gtype(grad), K, D, ld, _ptr(perm), _ptr(inverse), _ptr(offsets),
                         _ptr(num_unique), u_cap, _ptr(out), ld_out, _ptr(dev_err), _ptr(buf),
                         buf.numel(), _stream(stream)), "lm_segsum")
    return out


def segsum_rows(grad: torch.Tensor, perm: torch.Tensor, inverse: torch.Tensor,
                offsets: torch.Tensor, num_unique: torch.Tensor, row_ids: torch.Tensor,
                out: torch.Tensor, dev_err: Optional[torch.Tensor] = None,
                ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """lm_segsum_rows: Sec. III-A steps 2 and 5 in one pass: type u's sum goes
    to row row_ids[u] of `out` (e.g. the uniq ids into a dense V x D table);
    other rows of `out` are untouched. Returns `out`."""
    _dev(grad, "grad")
    _dev(row_ids, "row_ids")
    K, D = grad.shape
    ld = _rows(grad, "grad")
    if perm.numel() < K or inverse.numel() < K or offsets.numel() < 1:
        raise LmError("perm and inverse must hold K entries")
    if out.dim() != 2 or out.shape[1] != D or out.dtype != torch.float32:
        raise LmError("out must be an fp32 matrix with D columns")
    if not row_ids.is_contiguous():
        raise LmError("row_ids must be contiguous")
    ld_out = _rows(out, "out")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=grad.device)
    ws = ws or default_workspace(grad.device)
    buf = ws.get(_lib.lm_segsum_workspace_bytes(K, D))
    _call(_lib.lm_segsum_rows(_ptr(grad), _gtype(grad), K, D, ld, _ptr(perm), _ptr(inverse),
                              _ptr(offsets), _ptr(num_unique), _ptr(row_ids), _idtype(row_ids),
                              row_ids.numel(), _ptr(out), out.shape[0], ld_out, _ptr(dev_err),
                              _ptr(buf), buf.numel(), _stream(stream)), "lm_segsum_rows")
    return out


def segsum_sgd(grad: torch.Tensor, perm: torch.Tensor, inverse: torch.Tensor,
               offsets: torch.Tensor, num_unique: torch.Tensor, row_ids: torch.Tensor,
               table: torch.Tensor, lr: float, dev_err: Optional[torch.Tensor] = None,
               ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """lm_segsum_sgd: Sec. III-A steps 2 and 7 in one pass on one GPU:
    table[row_ids[u]] -= lr * (type u's sum), in place; other rows are
    untouched. Returns `table`."""
    _dev(grad, "grad")
    _dev(row_ids, "row_ids")
    K, D = grad.shape
    ld = _rows(grad, "grad")
    if perm.numel() < K or inverse.numel() < K or offsets.numel() < 1:
        raise LmError("perm and inverse must hold K entries")
    if table.dim() != 2 or table.shape[1] != D or table.dtype != torch.float32:
        raise LmError("table must be an fp32 matrix with D columns")
    if not row_ids.is_contiguous():
        raise LmError("row_ids must be contiguous")
    ld_t = _rows(table, "table")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=grad.device)
    ws = ws or default_workspace(grad.device)
    buf = ws.get(_lib.lm_segsum_workspace_bytes(K, D))
    _call(_lib.lm_segsum_sgd(_ptr(grad), _gtype(grad), K, D, ld, _ptr(perm), _ptr(inverse),
                             _ptr(offsets), _ptr(num_unique), _ptr(row_ids), _idtype(row_ids),
                             row_ids.numel(), _ptr(table), table.shape[0], ld_t, float(lr),
                             _ptr(dev_err), _ptr(buf), buf.numel(), _stream(stream)),
          "lm_segsum_sgd")
    return table


def segsum_adam(grad: torch.Tensor, perm: torch.Tensor, inverse: torch.Tensor,
                offsets: torch.Tensor, num_unique: torch.Tensor, row_ids: torch.Tensor,
                table: torch.Tensor, m: torch.Tensor, v: torch.Tensor, lr: float = 1e-3,
                beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                weight_decay: float = 0.0, step: int = 1, dev_err: Optional[torch.Tensor] = None,
                ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """lm_segsum_adam: Sec. III-A steps 2 and 7 in one pass on one GPU: the
    lazy-Adam step of table[row_ids[u]] (and of its m and v rows) with type
    u's sum as the gradient, in place; other rows are untouched. Returns
    `table`."""
    _dev(grad, "grad")
    _dev(row_ids, "row_ids")
    K, D = grad.shape
    ld = _rows(grad, "grad")
    if perm.numel() < K or inverse.numel() < K or offsets.numel() < 1:
        raise LmError("perm and inverse must hold K entries")
    if table.dim() != 2 or table.shape[1] != D or table.dtype != torch.float32:
        raise LmError("table must be an fp32 matrix with D columns")
    for t, n in ((m, "m"), (v, "v")):
        if t is None or t.shape != table.shape or t.stride() != table.stride() or t.dtype != table.dtype:
            raise LmError(f"{n} must have the table's shape, strides and dtype")
    if not row_ids.is_contiguous():
        raise LmError("row_ids must be contiguous")
    ld_t = _rows(table, "table")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=grad.device)
    ws = ws or default_workspace(grad.device)
    buf = ws.get(_lib.lm_segsum_workspace_bytes(K, D))
    _call(_lib.lm_segsum_adam(_ptr(grad), _gtype(grad), K, D, ld, _ptr(perm), _ptr(inverse),
                              _ptr(offsets), _ptr(num_unique), _ptr(row_ids), _idtype(row_ids),
                              row_ids.numel(), _ptr(table), table.shape[0], ld_t, float(lr),
                              float(beta1), float(beta2), float(eps), float(weight_decay),
                              int(step), _ptr(m), _ptr(v), _ptr(dev_err), _ptr(buf), buf.numel(),
                              _stream(stream)),
          "lm_segsum_adam")
    return table


def map_ids(sub_ids: torch.Tensor, n_sub: torch.Tensor, sup_ids: torch.Tensor,
            n_sup: torch.Tensor, out: Optional[torch.Tensor] = None,
            dev_err: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lm_map_ids: Sec. III-A step 4, the map J^ -> I^."""
    if sub_ids.dtype != sup_ids.dtype:
        raise LmError("sub_ids and sup_ids must share a dtype")
    cap = sub_ids.numel()
    if out is None:
        out = torch.empty(max(cap, 1), dtype=torch.int32, device=sub_ids.device)
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=sub_ids.device)
    if out.numel() < cap:
        raise LmError("map output shorter than sub_ids")
    _call(_lib.lm_map_ids(_ptr(sub_ids), _ptr(n_sub), cap, _ptr(sup_ids), _ptr(n_sup),
                          sup_ids.numel(), _idtype(sub_ids), _ptr(out), _ptr(dev_err),
                          _stream(stream)), "lm_map_ids")
    return out


_MODES = {"expand": FILL_EXPAND, "scatter": FILL_SCATTER, "scatter_add": FILL_SCATTER_ADD}


def fill_values(src: torch.Tensor, src_ids: torch.Tensor, n_src: torch.Tensor,
                dst: torch.Tensor, dst_ids: Optional[torch.Tensor] = None,
                n_dst: Optional[torch.Tensor] = None, mode: str = "expand",
                dev_err: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lm_fill_values: Sec. III-A step 5 (expand) or a row scatter."""
    D = src.shape[1]
    if dst.shape[1] != D:
        raise LmError("src and dst widths differ")
    if dst_ids is not None and dst_ids.dtype != src_ids.dtype:
        raise LmError("src_ids and dst_ids must share a dtype")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=src.device)
    # capacities: rows of src that have an id, rows of dst that have an id
    src_cap = min(src.shape[0], src_ids.numel())
    dst_rows = dst.shape[0] if dst_ids is None else min(dst.shape[0], dst_ids.numel())
    _call(_lib.lm_fill_values(_ptr(src), _rows(src, "src"), _ptr(src_ids), _ptr(n_src),
                              src_cap, _ptr(dst_ids), _ptr(n_dst), _idtype(src_ids), D,
                              _ptr(dst), dst_rows, _rows(dst, "dst"), _MODES[mode],
                              _ptr(dev_err), _stream(stream)), "lm_fill_values")
    return dst


def sparse_apply(table: torch.Tensor, rows: torch.Tensor, n_rows: torch.Tensor,
                 vals: torch.Tensor, opt: str = "sgd", lr: float = 0.1, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                 step: int = 1, m: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                 dev_err: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lm_sparse_apply: Sec. III-A step 7, in place on ``table`` (and m, v)."""
    V, D = table.shape
    if vals.shape[1] != D:
        raise LmError("vals and table widths differ")
    kind = {"sgd": OPT_SGD, "adam": OPT_ADAM}[opt]
    if kind == OPT_ADAM:
        for t, n in ((m, "m"), (v, "v")):
            if t is None or t.shape != table.shape or t.stride() != table.stride():
                raise LmError(f"Adam needs {n} shaped and strided like the table")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=table.device)
    rows_cap = min(rows.numel(), vals.shape[0])
    _call(_lib.lm_sparse_apply(_ptr(table), V, D, _rows(table, "table"), _ptr(rows),
                               _idtype(rows), _ptr(n_rows), rows_cap, _ptr(vals),
                               _rows(vals, "vals"), kind, lr, beta1, beta2, eps, weight_decay,
                               step, _ptr(m), _ptr(v), _ptr(dev_err), _stream(stream)),
          "lm_sparse_apply")
    return table


def _payload(t: torch.Tensor, what: str):
    if t.dtype not in (torch.float16, torch.int16, torch.uint16):
        raise LmError(f"{what} must hold binary16 (float16, or its bits as int16/uint16)")


def fill_values_f16(src: torch.Tensor, src_ids: torch.Tensor, n_src: torch.Tensor,
                    dst: torch.Tensor, dst_ids: Optional[torch.Tensor] = None,
                    n_dst: Optional[torch.Tensor] = None, mode: str = "expand",
                    scale: float = 1.0, dev_err: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """lm_fill_values_f16: Sec. III-C, EXPAND / SCATTER into a binary16 payload
    dst = binary16(src * scale)."""
    D = src.shape[1]
    _payload(dst, "dst")
    if dst.shape[1] != D:
        raise LmError("src and dst widths differ")
    if dst_ids is not None and dst_ids.dtype != src_ids.dtype:
        raise LmError("src_ids and dst_ids must share a dtype")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=src.device)
    src_cap = min(src.shape[0], src_ids.numel())
    dst_rows = dst.shape[0] if dst_ids is None else min(dst.shape[0], dst_ids.numel())
    _call(_lib.lm_fill_values_f16(_ptr(src), _rows(src, "src"), _ptr(src_ids), _ptr(n_src),
                                  src_cap, _ptr(dst_ids), _ptr(n_dst), _idtype(src_ids), D,
                                  _ptr(dst), dst_rows, _rows(dst, "dst"), _MODES[mode], scale,
                                  _ptr(dev_err), _stream(stream)), "lm_fill_values_f16")
    return dst


def sparse_apply_f16(table: torch.Tensor, rows: torch.Tensor, n_rows: torch.Tensor,
                     vals: torch.Tensor, inv_scale: float = 1.0, opt: str = "sgd",
                     lr: float = 0.1, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                     weight_decay: float = 0.0, step: int = 1, m: Optional[torch.Tensor] = None,
                     v: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """lm_sparse_apply_f16: step 7 from a binary16 payload, g = fp32(vals) * inv_scale."""
    V, D = table.shape
    _payload(vals, "vals")
    if vals.shape[1] != D:
        raise LmError("vals and table widths differ")
    kind = {"sgd": OPT_SGD, "adam": OPT_ADAM}[opt]
    if kind == OPT_ADAM:
        for t, n in ((m, "m"), (v, "v")):
            if t is None or t.shape != table.shape or t.stride() != table.stride():
                raise LmError(f"Adam needs {n} shaped and strided like the table")
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=table.device)
    rows_cap = min(rows.numel(), vals.shape[0])
    _call(_lib.lm_sparse_apply_f16(_ptr(table), V, D, _rows(table, "table"), _ptr(rows),
                                   _idtype(rows), _ptr(n_rows), rows_cap, _ptr(vals),
                                   _rows(vals, "vals"), inv_scale, kind, lr, beta1, beta2, eps,
                                   weight_decay, step, _ptr(m), _ptr(v), _ptr(dev_err),
                                   _stream(stream)), "lm_sparse_apply_f16")
    return table


def segsum_two_launches(enable: bool) -> bool:
    """lm_segsum_set_two_launches: every later lm_segsum call in the process
    takes the two-launch form (walk, then a separate fix-up kernel) while
    enabled. Returns the previous setting."""
    return bool(_lib.lm_segsum_set_two_launches(1 if enable else 0))


def force_wait_failure(enable: bool, spin_limit: int = 64):
    """lm_test_force_wait_failure: test hook for the failure path of the
    one-launch Seg-Sum's bounded waits (see include/lmzipf.h)."""
    _call(_lib.lm_test_force_wait_failure(1 if enable else 0, int(spin_limit)),
          "lm_test_force_wait_failure")


def sample_ids(r: torch.Tensor, V: int, out: Optional[torch.Tensor] = None,
               id_dtype=torch.int32, stream=None) -> torch.Tensor:
    """lm_sample_ids: Sec. III-B candidate sampler, ids = floor(r * V / 2^64)
    of caller-drawn 64-bit random words (``r`` int64 or uint64 bits)."""
    _dev(r, "r")
    if r.dtype not in (torch.int64, torch.uint64):
        raise LmError("random words must be 64-bit")
    if out is None:
        out = torch.empty(r.numel(), dtype=id_dtype, device=r.device)
    if out.numel() < r.numel():
        raise LmError("ids shorter than r")
    _call(_lib.lm_sample_ids(_ptr(r), r.numel(), V, _ptr(out), _idtype(out), _stream(stream)),
          "lm_sample_ids")
    return out


# ---------------------------------------------------------------------------
# AdamW over many tensors, and on table rows with 8-bit moments
# ---------------------------------------------------------------------------
def _on(device: torch.device, stream):
    """The handle of the call's stream, `device` being the current one."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(device.index)


def _elsewhere(device: torch.device, stream) -> bool:
    """Whether `device` is not the current one. A stream of another device than
    the tensors' is refused."""
    if stream is not None and stream.device != device:
        raise LmError(f"stream is on {stream.device}, the tensors are on {device}")
    return torch.cuda.current_device() != device.index


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise LmError(f"the call's tensors are on {device} and {t.device}")


# Autograd's note that the tensors were written in place: a backward pass that has saved
# one of them raises, as after torch's own operations.
_written = torch.autograd.graph.increment_version


def _one_of(t: Optional[torch.Tensor], dtype, what: str):
    if t is not None and (t.dtype != dtype or t.numel() < 1):
        raise LmError(f"{what} must be a {dtype} tensor of one element")


_CODES = (torch.float8_e4m3fn, torch.uint8)


def _codes(t: torch.Tensor, what: str):
    if t.dtype not in _CODES:
        raise LmError(f"{what} must hold e4m3 codes (float8_e4m3fn, or its bits as uint8)")


_SCALES = (torch.uint8, getattr(torch, "float8_e8m0fnu", torch.uint8))


def _scales(t: torch.Tensor, what: str):
    if t.dtype not in _SCALES:
        raise LmError(f"{what} must hold scale bytes (uint8 or float8_e8m0fnu)")


_grad_of = operator.attrgetter("grad")


def _owns(t: torch.Tensor, grad: torch.Tensor) -> bool:
    """Whether the memory of `grad` is that of `t.grad`."""
    own = t.grad if t.is_leaf else None
    return own is not None and own.layout == torch.strided and own.data_ptr() == grad.data_ptr()


class AdamwPlan(NamedTuple):
    """A list of tensors as ``adamw`` steps it: the table that names their
    memory on the device, and that memory itself, which it keeps alive also
    where a tensor has been given other memory since (`p.data = ...`), until
    every stream that stepped it is past its steps (so a stream of the caller's
    own making has to outlive these tensors, as for `Tensor.record_stream`).
    `streams`: the handles of those that the allocator knows of; `versions`: the
    tensors of which autograd is told that they were written; `owners`: the
    parameters and copies whose `.grad` the plan steps, `grads`: its addresses."""
    table: torch.Tensor
    tensors: tuple
    chunks: int
    gtype: int
    states: int
    copies: bool
    streams: set
    versions: tuple
    owners: tuple
    grads: list


def adamw_plan(params, grads, m, v, m_scale=None, v_scale=None, copies=None,
               decay=None) -> AdamwPlan:
    """lm_adamw_plan: lists of contiguous tensors of equal sizes on one device.
    params fp32, grads all fp32 or all bf16, m and v fp32; or 8-bit moments: m
    and v e4m3 codes (v of its square root), m_scale and v_scale one byte per
    MOMENT_BLOCK values. copies: bf16 copies of the parameters, written with
    every step. decay: one truth value per tensor, whether weight_decay
    applies. Copies the table to the device; make a new plan when a tensor
    (say, a gradient) gets other memory, and keep one as long as a captured
    graph steps it. A gradient that is the `.grad` of its parameter or copy has
    to stay that: ``adamw`` refuses the plan once it is not (after
    `zero_grad(set_to_none=True)`, say), as it would step an old gradient."""
    params, grads, m, v = (list(x) for x in (params, grads, m, v))
    lists = {"grads": grads, "m": m, "v": v}
    for name, x in (("m_scale", m_scale), ("v_scale", v_scale), ("copies", copies)):
        if x is not None:
            lists[name] = list(x)
    n = len(params)
    decay = None if decay is None else [int(bool(d)) for d in decay]
    for name, x in list(lists.items()) + ([] if decay is None else [("decay", decay)]):
        if len(x) != n:
            raise LmError(f"{name} has {len(x)} entries, params has {n}")
    for name, x in (("params", params), *lists.items()):
        for i, t in enumerate(x):
            if not isinstance(t, torch.Tensor):
                raise LmError(f"{name}[{i}] must be a tensor, got {type(t).__name__}")
    eight = "m_scale" in lists
    if eight != ("v_scale" in lists):
        raise LmError("8-bit moments need m_scale and v_scale")
    if not n:
        raise LmError("params is empty")
    device = params[0].device
    _dev(params[0], "params")
    gtype = _gtype(grads[0])
    for i, p in enumerate(params):
        k = p.numel()
        if p.dtype != torch.float32:
            raise LmError("params must be float32")
        blocks = -(-k // MOMENT_BLOCK)
        for name, t, want in ([("params", p, k)] + [(a, x[i], blocks if a.endswith("_scale") else k)
                                                    for a, x in lists.items()]):
            if t.device != device or not t.is_contiguous() or t.numel() != want:
                raise LmError(f"{name}[{i}] must be contiguous on {device} with {want} elements")
        if _gtype(grads[i]) != gtype:
            raise LmError("grads must share a dtype")
        for a in ("m", "v"):
            if eight:
                _codes(lists[a][i], a)
                _scales(lists[a + "_scale"][i], a + "_scale")
            elif lists[a][i].dtype != torch.float32:
                raise LmError(f"{a} must be float32 (8-bit moments come with scales)")
        if "copies" in lists and lists["copies"][i].dtype != torch.bfloat16:
            raise LmError("copies must be bfloat16")

    def pointers(x):
        return None if x is None else (ctypes.c_void_p * n)(*[t.data_ptr() for t in x])
    sizes = (ctypes.c_int64 * n)(*[p.numel() for p in params])
    need = _lib.lm_adamw_plan_bytes(sizes, n)
    if need == 0:
        raise LmError("lm_adamw_plan_bytes rejected the sizes")
    host = torch.empty(need, dtype=torch.uint8)
    chunks = ctypes.c_int64()
    _call(_lib.lm_adamw_plan(
        pointers(params), pointers(grads), pointers(m), pointers(v), pointers(lists.get("m_scale")),
        pointers(lists.get("v_scale")), pointers(lists.get("copies")), sizes,
        None if decay is None else (ctypes.c_int32 * n)(*decay), n, gtype, 8 if eight else 32,
        _ptr(host), need, ctypes.byref(chunks)), "lm_adamw_plan")
    keep = tuple(tuple(t.detach() for t in x) for x in [params] + list(lists.values()))
    # (views of one tensor share its version: one of them is enough)
    written = {id(t if t._base is None else t._base): t for t in params + lists.get("copies", [])}
    written = tuple(t.detach() for t in written.values())
    owned = [(o, g.data_ptr()) for owners in (params, lists.get("copies", []))
             for o, g in zip(owners, grads) if g.numel() and _owns(o, g)]
    with torch.cuda.device(device):
        return AdamwPlan(host.to(device), keep, chunks.value, gtype, 8 if eight else 32,
                         "copies" in lists, set(), written,
                         tuple(o for o, _ in owned), [a for _, a in owned])



def adamw(plan: AdamwPlan, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
          eps: float = 1e-8, weight_decay: float = 0.0, step: int = 1,
          grad_scale: Optional[torch.Tensor] = None, seed: int = 0,
          dev_err: Optional[torch.Tensor] = None, stream=None) -> None:
    """lm_adamw: one AdamW step of every tensor of the plan, in place, in one
    launch. grad_scale: a device fp32 number that multiplies every gradient.
    seed: of the 8-bit moments' rounding; give every step its own. dev_err tells
    of values that were kept as they were, since their second moment would not be
    finite; without it nothing does. A captured call repeats its step, seed and
    rates with every replay."""
    table = plan.table
    device = table.device
    if grad_scale is not None:
        _same_device(device, grad_scale)
        _one_of(grad_scale, torch.float32, "grad_scale")
    if dev_err is not None:
        _same_device(device, dev_err)
        _one_of(dev_err, torch.int32, "dev_err")
    if plan.owners and plan.grads != [g is not None and g.data_ptr()
                                      for g in map(_grad_of, plan.owners)]:
        raise LmError("a gradient is no longer the one that the plan names: keep its memory"
                      " (zero_grad(set_to_none=False)) or make a new plan")
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return adamw(plan, lr, beta1, beta2, eps, weight_decay, step, grad_scale, seed,
                         dev_err, stream)
    handle = _on(device, stream)
    if handle not in plan.streams:
        # The plan may hold the last reference to its memory, which is not to be reused before
        # this stream is past its steps (recording a tensor's own stream does nothing).
        at = stream or torch.cuda.current_stream()
        for t in (table, *(t for x in plan.tensors for t in x)):
            t.record_stream(at)
        plan.streams.add(handle)
    _call(_lib.lm_adamw(_ptr(table), table.numel(), plan.chunks, plan.gtype, plan.states,
                        plan.copies, lr, beta1, beta2, eps, weight_decay, step,
                        _ptr(grad_scale), seed, _ptr(dev_err), handle), "lm_adamw")
    _written(plan.versions)


def sparse_apply_q8(table: torch.Tensor, rows: torch.Tensor, n_rows: torch.Tensor,
                    vals: torch.Tensor, m: torch.Tensor, v: torch.Tensor, m_scale: torch.Tensor,
                    v_scale: torch.Tensor, lr: float = 1e-3, beta1: float = 0.9,
                    beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                    step: int = 1, seed: int = 0, dev_err: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """lm_sparse_apply_q8: the lazy AdamW step of ``sparse_apply(opt="adam")``
    with 8-bit moments, in place: m and v V x D codes (v of its square root),
    m_scale and v_scale V x ceil(D / MOMENT_BLOCK) bytes. seed, dev_err and
    captured calls as ``adamw``'s."""
    _dev(table, "table")
    V, D = table.shape
    if table.dtype != torch.float32 or vals.dtype != torch.float32:
        raise LmError("table and vals must be float32")
    cap, width = vals.shape
    if width != D:
        raise LmError("vals and table widths differ")
    if m.dtype not in _CODES or v.dtype not in _CODES:
        raise LmError("m and v must hold e4m3 codes (float8_e4m3fn, or its bits as uint8)")
    if m_scale.dtype not in _SCALES or v_scale.dtype not in _SCALES:
        raise LmError("m_scale and v_scale must hold scale bytes (uint8 or float8_e8m0fnu)")
    blocks = -(-D // MOMENT_BLOCK)
    if m.shape != (V, D) or v.shape != (V, D):
        raise LmError(f"m and v must be {V} x {D}")
    if m_scale.shape != (V, blocks) or v_scale.shape != (V, blocks):
        raise LmError(f"m_scale and v_scale must be {V} x {blocks}")
    if m.stride() != v.stride() or m_scale.stride() != v_scale.stride():
        raise LmError("m and v, and their scales, must share their strides")
    if not rows.is_contiguous():
        raise LmError("rows must be contiguous")
    _one_of(n_rows, torch.int64, "n_rows")
    _one_of(dev_err, torch.int32, "dev_err")
    _same_device(table.device, rows, n_rows, vals, m, v, m_scale, v_scale, dev_err)
    if _elsewhere(table.device, stream):
        with torch.cuda.device(table.device):
            return sparse_apply_q8(table, rows, n_rows, vals, m, v, m_scale, v_scale, lr, beta1,
                                   beta2, eps, weight_decay, step, seed, dev_err, stream)
    _call(_lib.lm_sparse_apply_q8(
        _ptr(table), V, D, _rows(table, "table"), _ptr(rows), _idtype(rows), _ptr(n_rows),
        min(rows.numel(), cap), _ptr(vals), _rows(vals, "vals"), lr, beta1, beta2,
        eps, weight_decay, step, _ptr(m), _ptr(v), _rows(m, "m"), _ptr(m_scale), _ptr(v_scale),
        _rows(m_scale, "m_scale"), seed, _ptr(dev_err), _on(table.device, stream)),
          "lm_sparse_apply_q8")
    _written(table)
    return table


# ---------------------------------------------------------------------------
# Relative position bias
# ---------------------------------------------------------------------------
class RelBuckets(NamedTuple):
    """Segments of the distance axis and their table rows (host memory)."""
    starts: ctypes.Array
    ids: ctypes.Array
    n_seg: int
    num_buckets: int


_REL_MODES = {"both": REL_BOTH, "past": REL_PAST, "causal": REL_CAUSAL}


def rel_buckets(num_buckets: int, max_distance: int, mode: str = "both") -> RelBuckets:
    """lm_rel_buckets: logarithmic buckets. mode "both": half for keys up to
    the query and half for those after it; "past": keys after the query are in
    bucket 0; "causal": they are masked. Computed once, for every later call."""
    starts = (ctypes.c_int32 * REL_MAX_SEGMENTS)()
    ids = (ctypes.c_int32 * REL_MAX_SEGMENTS)()
    n = ctypes.c_int32()
    if mode not in _REL_MODES:
        raise LmError(f"mode must be one of {sorted(_REL_MODES)}, got {mode!r}")
    _call(_lib.lm_rel_buckets(num_buckets, max_distance, _REL_MODES[mode], starts, ids,
                              ctypes.byref(n)), "lm_rel_buckets")
    return RelBuckets(starts, ids, n.value, num_buckets)


def _no_graph(what: str, *tensors):
    """A tensor that requires grad would come out of the call without its graph."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise LmError(f"{what} is not recorded by autograd: call it under torch.no_grad() or"
                          " in an autograd.Function (rel_bias_grad is the gradient of rel_bias)")


_Strides = ctypes.c_int64 * 3


def _scores(t: torch.Tensor, what: str):
    """Strides (b, h, i) of a B x H x Lq x Lk or H x Lq x Lk tensor with unit column stride."""
    strides = t.stride()
    if not 3 <= len(strides) <= 4 or (strides[-1] != 1 and t.shape[-1] > 1):
        raise LmError(f"{what} must be [B x] H x Lq x Lk with unit stride along the keys")
    return _Strides(*strides[:3]) if len(strides) == 4 else _Strides(0, *strides[:2])


def rel_bias(table: torch.Tensor, buckets: RelBuckets, Lq: int, Lk: int, q_start: int = 0,
             add: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             dtype=torch.float32, stream=None) -> torch.Tensor:
    """lm_rel_bias: table[bucket(j - (q_start + i)), h] for every head, query i
    and key j, as an H x Lq x Lk tensor of `dtype`; with `add` (B x H x Lq x Lk
    attention scores) the scores plus the bias, of their shape and dtype. `out`
    may be `add` itself. Not recorded by autograd: tensors that require grad are
    refused while grad mode is on."""
    _no_graph("rel_bias", table, add, out)
    _dev(table, "table")
    size = table.shape
    if len(size) != 2 or table.dtype != torch.float32 or size[0] != buckets.num_buckets:
        raise LmError(f"table must be float32 with {buckets.num_buckets} rows")
    H, device = size[1], table.device
    _same_device(device, add, out)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return rel_bias(table, buckets, Lq, Lk, q_start, add, out, dtype, stream)
    if add is not None:
        dtype, shape = add.dtype, add.shape
        if len(shape) != 4 or shape[1:] != (H, Lq, Lk):
            raise LmError(f"add must be B x {H} x {Lq} x {Lk}")
    else:
        shape = (H, Lq, Lk)
    given = out
    if out is None:
        out = _empty(shape, dtype, device, stream)
    elif out.shape != shape or out.dtype != dtype:
        raise LmError(f"out must be {' x '.join(map(str, shape))} of {dtype}")
    _call(_lib.lm_rel_bias(
        _ptr(table), _rows(table, "table"), buckets.num_buckets, buckets.starts, buckets.ids,
        buckets.n_seg, 1 if add is None else shape[0], H, Lq, Lk, q_start, _ptr(add),
        None if add is None else _scores(add, "add"), _ptr(out), _scores(out, "out"),
        _gtype(out), _on(device, stream)), "lm_rel_bias")
    if given is not None:
        _written(given)
    return out


def rel_bias_grad(dout: torch.Tensor, buckets: RelBuckets, q_start: int = 0,
                  out: Optional[torch.Tensor] = None, accumulate: bool = False,
                  ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """lm_rel_bias_grad: the table's gradient, num_buckets x H fp32, from that
    of the scores (B x H x Lq x Lk, or H x Lq x Lk). accumulate: add to `out`.
    Without `ws` the call takes its workspace from torch's allocator. Not
    recorded by autograd, as ``rel_bias``."""
    _no_graph("rel_bias_grad", dout, out)
    _dev(dout, "dout")
    strides, shape, device = _scores(dout, "dout"), dout.shape, dout.device
    B = shape[0] if len(shape) == 4 else 1
    H, Lq, Lk = shape[-3:]
    gtype = _gtype(dout)
    _same_device(device, out, None if ws is None else ws.buf)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return rel_bias_grad(dout, buckets, q_start, out, accumulate, ws, stream)
    given = out
    if out is None:
        if accumulate:
            raise LmError("accumulate needs out")
        out = _empty((buckets.num_buckets, H), torch.float32, device, stream)
    elif out.dtype != torch.float32 or out.shape != (buckets.num_buckets, H):
        raise LmError(f"out must be float32, {buckets.num_buckets} x {H}")
    need = _lib.lm_rel_bias_grad_workspace_bytes(B, H, Lq, Lk, gtype, buckets.n_seg)
    buf = None
    if need:
        buf = ws.get(need) if ws is not None else _empty((need,), torch.uint8, device, stream)
    _call(_lib.lm_rel_bias_grad(
        _ptr(dout), gtype, B, H, Lq, Lk, strides, q_start, buckets.starts, buckets.ids,
        buckets.n_seg, buckets.num_buckets, _ptr(out), _rows(out, "out"), bool(accumulate),
        _ptr(buf), need, _on(device, stream)), "lm_rel_bias_grad")
    if given is not None:
        _written(given)
    return out


def _empty(shape, dtype, device, stream):
    """A tensor that torch's allocator gives to the call's stream, and takes back
    in that stream's order."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)
