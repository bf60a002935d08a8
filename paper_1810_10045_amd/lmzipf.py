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
``rel_bias_grad`` (a learned relative position bias and its gradient),
``dropout``, ``layer_norm`` and ``layer_norm_grad``, ``token_logprobs`` and
``token_logprobs_grad`` (log probabilities of given tokens, entropy, top
alternatives).
"""
from __future__ import annotations

import ctypes
import operator
import os
import warnings
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

# The current stream's handle (not a public name of torch: the public call where it is absent).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# The current device's number, where the device is in use already: a third of the public call's time.
_this_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)

# The current stream's handle on a device.
_stream_of = _raw_stream or (lambda device: torch.cuda.current_stream(device).cuda_stream)

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
NORM_MAX_WIDTH, TOP_MAX = 16384, 64
MAX_K = 1 << 30

EXPORTS = ("lm_status_string", "lm_abi_version", "lm_workspace_clear",
           "lm_unique_workspace_bytes", "lm_unique", "lm_segsum_workspace_bytes",
           "lm_segsum", "lm_map_ids", "lm_fill_values", "lm_sparse_apply",
           "lm_fill_values_f16", "lm_sparse_apply_f16", "lm_sample_ids",
           "lm_adamw_plan_bytes", "lm_adamw_plan", "lm_adamw", "lm_sparse_apply_q8",
           "lm_rel_buckets", "lm_rel_bias", "lm_rel_bias_grad_workspace_bytes",
           "lm_rel_bias_grad", "lm_dropout", "lm_layer_norm", "lm_layer_norm_grad_workspace_bytes",
           "lm_layer_norm_grad", "lm_token_logprobs_workspace_bytes", "lm_token_logprobs",
           "lm_token_logprobs_grad")


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
    L.lm_dropout.argtypes = [P, I64_, P, I64_, P, I64_, I64_, I64_, I32_, F, U64, P, P]
    L.lm_layer_norm.argtypes = [P, I64_, P, I64_, I64_, I64_, I32_, P, P, F, F, U64, P, P, I64_, P,
                                I64_, P, P, P]
    L.lm_layer_norm_grad_workspace_bytes.argtypes = [I64_, I64_, I32_]
    L.lm_layer_norm_grad_workspace_bytes.restype = SZ
    L.lm_layer_norm_grad.argtypes = [P, I64_, P, I64_, P, I64_, I64_, I64_, I32_, P, P, P, F, U64, P,
                                     P, I64_, P, I64_, P, P, I32_, P, SZ, P]
    L.lm_token_logprobs_workspace_bytes.argtypes = [I64_, I64_, I32_, I32_]
    L.lm_token_logprobs_workspace_bytes.restype = SZ
    L.lm_token_logprobs.argtypes = [P, I64_, I64_, I64_, I32_, P, I32_, I64_, F, I32_, P, P, P, P, P,
                                    P, P, P, SZ, P]
    L.lm_token_logprobs_grad.argtypes = [P, I64_, I64_, I64_, I32_, P, I32_, I64_, F, P, P, P, P, P,
                                         P, I64_, P]
    L.lm_segsum_set_two_launches.argtypes = [I32_]
    L.lm_test_force_wait_failure.argtypes = [I32_, ctypes.c_uint32]
    for f in ("lm_abi_version", "lm_workspace_clear", "lm_unique", "lm_unique_noalloc",
              "lm_segsum", "lm_segsum_rows", "lm_segsum_sgd", "lm_segsum_adam", "lm_map_ids",
              "lm_fill_values", "lm_sparse_apply", "lm_fill_values_f16", "lm_sparse_apply_f16",
              "lm_sample_ids", "lm_segsum_set_two_launches", "lm_test_force_wait_failure",
              "lm_adamw_plan", "lm_adamw", "lm_sparse_apply_q8", "lm_rel_buckets", "lm_rel_bias",
              "lm_rel_bias_grad", "lm_dropout", "lm_layer_norm", "lm_layer_norm_grad",
              "lm_token_logprobs", "lm_token_logprobs_grad"):
        getattr(L, f).restype = ctypes.c_int
    return L


_lib = _load()


def lib():
    return _lib


def _load_calls():
    """The plain calls of dropout, layer norm and the token log probabilities without Python
    between the checks, the results' allocation and the library (``csrc/calls.cpp``): of a call
    of few rows that is more than half. It is built against one Python and one torch; where it is
    absent or cannot be loaded (None, and a warning) these calls take ctypes as all others do, to
    the same kernels."""
    try:
        from . import _lmzipf_calls as calls
    except ImportError as e:
        warnings.warn(f"short calls take longer without _lmzipf_calls ({e}): build it with"
                      " `python -c 'import __graft_entry__ as g; g.build()'`", RuntimeWarning)
        return None
    names = ("lm_dropout", "lm_layer_norm", "lm_layer_norm_grad_workspace_bytes",
             "lm_layer_norm_grad", "lm_token_logprobs_workspace_bytes", "lm_token_logprobs",
             "lm_token_logprobs_grad", "lm_status_string")
    calls.bind(LmError, *(ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in names))
    return calls


_calls = _load_calls()


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
    return _this_device() != device.index


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


def _no_graph(what: str, *tensors, gradient="rel_bias_grad is the gradient of rel_bias"):
    """A tensor that requires grad would come out of the call without its graph."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise LmError(f"{what} is not recorded by autograd: call it under torch.no_grad() or"
                          f" in an autograd.Function ({gradient})")
    _no_tangent(what, *tensors)


def _no_tangent(what: str, *tensors):
    """A tensor with a forward-mode tangent would come out of the call without it, under
    torch.no_grad() too, which is of reverse mode only."""
    # the level that is entered, -1 for none (not a public name: 0 where it is absent)
    if getattr(forward_ad, "_current_level", 0) < 0:
        return
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise LmError(f"{what} has no forward-mode derivative and would drop a tensor's tangent:"
                          " call it on forward_ad.unpack_dual(tensor).primal or in an"
                          " autograd.Function with a jvp")


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
    refused while grad mode is on, and tensors with a forward-mode tangent."""
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


# ---------------------------------------------------------------------------
# Dropout and layer norm
# ---------------------------------------------------------------------------
def _matrix(t: torch.Tensor, what: str):
    """(rows, D, ld) of a tensor whose last dimension is the columns; the others, one behind
    the other, are the rows."""
    shape = t.shape
    if not shape:
        raise LmError(f"{what} must have a dimension")
    D = shape[-1]
    if t.is_contiguous():
        return (t.numel() // D if D else 0), D, D
    strides = t.stride()
    rows, ld = 1, None
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n != 1 and rows and s != (s if ld is None else rows * ld):
            raise LmError(f"{what} must have its rows at equal distances")
        ld = s if n != 1 and ld is None else ld
        rows *= n
    if strides[-1] != 1 and D > 1:
        raise LmError(f"{what} must have unit column stride")
    return rows, D, D if ld is None else ld


def _like(t: Optional[torch.Tensor], x: torch.Tensor, what: str):
    """The row stride of an operand of x's shape and dtype (None: 0)."""
    if t is None:
        return 0
    shape = x.shape
    if t.shape != shape or t.dtype != x.dtype:
        raise LmError(f"{what} must be {' x '.join(map(str, shape))} of {x.dtype}")
    return shape[-1] if t.is_contiguous() else _matrix(t, what)[2]


def _new(x: torch.Tensor, stream):
    """A contiguous tensor of x's shape and dtype (torch.empty_like takes half the time of
    torch.empty, which a call of a few rows is made of)."""
    if stream is None and x.is_contiguous():
        return torch.empty_like(x)
    return _empty(x.shape, x.dtype, x.device, stream)


def _vector(t: Optional[torch.Tensor], n: int, what: str):
    if t is not None and (t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous()):
        raise LmError(f"{what} must be contiguous float32 with {n} elements")


def _seed(seed, device):
    """(number, address) of a seed that the host or the device holds."""
    if not isinstance(seed, torch.Tensor):
        return seed, None
    _one_of(seed, torch.int64, "seed")
    _same_device(device, seed)
    return 0, seed.data_ptr()


def dropout(x: torch.Tensor, p: float, seed, add: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lm_dropout: x with each element dropped with probability p (to multiples
    of 2^-16) and the others divided by 1 - p, plus `add`; x float32 or bfloat16,
    its last dimension the columns. The mask is a function of `seed`, the
    element's row and column and the number of columns: the gradient is
    `dropout(dout, p, seed)`. seed: a number, or an int64 tensor of one element
    on the device, which a captured call reads with every replay. Far values' masks
    correlate (lm_dropout says how much): a matrix of more than 2^33 elements goes
    into several calls, each with its own seed. `out` may be x or `add`. Not
    recorded by autograd, as ``rel_bias``."""
    if _calls and out is None and stream is None and x.is_cuda:
        here = _this_device()
        r = _calls.dropout(here, _stream_of(here), x, p, seed, add)
        if r is not None:
            return r[0]
    _no_graph("dropout", x, add, out, gradient="its gradient is dropout with the same seed")
    _dev(x, "x")
    device = x.device
    rows, D, ld = _matrix(x, "x")
    dtype = _gtype(x)
    _same_device(device, add, out)
    number, at = _seed(seed, device)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return dropout(x, p, seed, add, out, stream)
    ld_add, ld_out = _like(add, x, "add"), D
    given = out
    if out is None:
        out = _new(x, stream)
    else:
        ld_out = _like(out, x, "out")
    _call(_lib.lm_dropout(x.data_ptr(), ld, _ptr(add), ld_add, out.data_ptr(), ld_out, rows, D,
                          dtype, p, number, at, _on(device, stream)), "lm_dropout")
    if given is not None:
        _written(given)
    return out


class NormResult(NamedTuple):
    """y, what it is the norm of, and the statistics that the gradient takes."""
    y: torch.Tensor
    h: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor


_NORM_GRADIENT = "layer_norm_grad is the gradient of layer_norm"


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               add: Optional[torch.Tensor] = None, p: float = 0.0, seed=0,
               out: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None,
               stream=None) -> NormResult:
    """lm_layer_norm: y, the norm of h = add + dropout(x) over its last
    dimension (up to NORM_MAX_WIDTH), with float32 weight and bias. h is x itself
    where nothing is added or dropped, else `sum_out` (which may be `add`: the
    residual stream) or a new tensor; y goes to `out` (which may be x) or a new
    one. p and seed as ``dropout``'s. Not recorded by autograd, as ``rel_bias``."""
    if _calls and out is None and sum_out is None and stream is None and x.is_cuda:
        here = _this_device()
        r = _calls.layer_norm(here, _stream_of(here), x, weight, bias, eps, add, p, seed)
        if r is not None:
            return NormResult(*r)
    _no_graph("layer_norm", x, weight, bias, add, out, sum_out, gradient=_NORM_GRADIENT)
    _dev(x, "x")
    device = x.device
    rows, D, ld = _matrix(x, "x")
    dtype = _gtype(x)
    _vector(weight, D, "weight")
    _vector(bias, D, "bias")
    _same_device(device, weight, bias, add, out, sum_out)
    number, at = _seed(seed, device)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return layer_norm(x, weight, bias, eps, add, p, seed, out, sum_out, stream)
    ld_add, ld_y, ld_h, h = _like(add, x, "add"), D, D, sum_out
    if out is None:
        y = _new(x, stream)
    else:
        y, ld_y = out, _like(out, x, "out")
    if sum_out is not None:
        ld_h = _like(sum_out, x, "sum_out")
    elif add is not None or p > 0:
        h = _new(x, stream)
    mean, rstd = _empty((2, *x.shape[:-1]), torch.float32, device, stream).unbind()
    _call(_lib.lm_layer_norm(
        x.data_ptr(), ld, _ptr(add), ld_add, rows, D, dtype, _ptr(weight), _ptr(bias), eps, p,
        number, at, y.data_ptr(), ld_y, _ptr(h), ld_h, mean.data_ptr(), rstd.data_ptr(),
        _on(device, stream)), "lm_layer_norm")
    if out is not None:
        _written(out)
    if sum_out is not None:
        _written(sum_out)
    return NormResult(y, x if h is None else h, mean, rstd)


class NormGrad(NamedTuple):
    """Gradients: of h (and of the forward's `add`), of x (dh itself without
    dropout), of the weight and of the bias (None where there is none)."""
    dh: torch.Tensor
    dx: torch.Tensor
    dweight: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


def layer_norm_grad(dy: torch.Tensor, h: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                    weight: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None,
                    p: float = 0.0, seed=0, out: Optional[torch.Tensor] = None,
                    dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                    dbias: Optional[torch.Tensor] = None, bias: Optional[bool] = None,
                    accumulate: bool = False, ws: Optional[Workspace] = None,
                    stream=None) -> NormGrad:
    """lm_layer_norm_grad: from the gradient of y and what ``layer_norm``
    returned. add: the gradient that reaches h past the norm (the residual
    stream's). p and seed: the forward's. out (dh), dx: written, new where not
    given; they may be dy, h or add. dweight, dbias: float32, written, or with
    `accumulate` added to; new where not given, dweight where there is a weight,
    dbias as `bias` says (None: as the weight). Without `ws` the call takes its
    workspace from torch's allocator. Not recorded by autograd, as ``rel_bias``."""
    if (_calls and out is None and dx is None and dweight is None and dbias is None and
            not accumulate and ws is None and stream is None and dy.is_cuda):
        here = _this_device()
        r = _calls.layer_norm_grad(here, _stream_of(here), dy, h, mean, rstd, weight, add, p, seed,
                                   bias)
        if r is not None:
            return NormGrad(*r)
    _no_graph("layer_norm_grad", dy, h, weight, add, out, dx, dweight, dbias,
              gradient=_NORM_GRADIENT)
    _no_tangent("layer_norm_grad", mean, rstd)
    _dev(dy, "dy")
    device = dy.device
    rows, D, ld = _matrix(dy, "dy")
    dtype = _gtype(dy)
    for t, n, what in ((mean, rows, "mean"), (rstd, rows, "rstd"), (weight, D, "weight"),
                       (dweight, D, "dweight"), (dbias, D, "dbias")):
        _vector(t, n, what)
    _same_device(device, h, mean, rstd, weight, add, out, dx, dweight, dbias,
                 None if ws is None else ws.buf)
    number, at = _seed(seed, device)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return layer_norm_grad(dy, h, mean, rstd, weight, add, p, seed, out, dx, dweight, dbias,
                                   bias, accumulate, ws, stream)
    bias = weight is not None if bias is None else bias
    new = (dweight is None and weight is not None) + (dbias is None and bool(bias))
    if accumulate and (new or (dweight is None and dbias is None)):
        raise LmError("accumulate needs dweight, and dbias where there is a bias")
    ld_h, ld_add = _like(h, dy, "h"), _like(add, dy, "add")
    given = [t for t in (out, dx, dweight, dbias) if t is not None]
    if out is None:
        out = _new(dy, stream)
    if dx is None and p > 0:
        dx = _new(dy, stream)
    if new:
        fresh = list(_empty((new, D), torch.float32, device, stream).unbind())
        dweight = fresh.pop(0) if dweight is None and weight is not None else dweight
        dbias = fresh.pop(0) if dbias is None and bias else dbias
    buf, need = None, 0
    if dweight is not None or dbias is not None:
        need = _lib.lm_layer_norm_grad_workspace_bytes(rows, D, dtype)
        if need:
            buf = ws.get(need) if ws is not None else _empty((need,), torch.uint8, device, stream)
    _call(_lib.lm_layer_norm_grad(
        _ptr(dy), ld, _ptr(h), ld_h, _ptr(add), ld_add, rows, D, dtype, _ptr(mean), _ptr(rstd),
        _ptr(weight), p, number, at, _ptr(out), _like(out, dy, "out"), _ptr(dx),
        _like(dx, dy, "dx"), _ptr(dweight), _ptr(dbias), bool(accumulate), _ptr(buf), need,
        _on(device, stream)), "lm_layer_norm_grad")
    for t in given:
        _written(t)
    return NormGrad(out, out if dx is None else dx, dweight, dbias)


# ---------------------------------------------------------------------------
# Log probabilities of given tokens
# ---------------------------------------------------------------------------
class TokenLogprobs(NamedTuple):
    """Per row: the target's log probability (None without targets), the
    entropy, the largest logit and log sum exp(scale * (logit - peak)); the likeliest
    words' log probabilities and ids (None without `top`)."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    peak: torch.Tensor
    log_sum: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


_LOGP_GRADIENT = "token_logprobs_grad is the gradient of token_logprobs"


def _targets(targets: Optional[torch.Tensor], logits: torch.Tensor) -> int:
    if targets is None:
        return I32
    if targets.shape != logits.shape[:-1] or not targets.is_contiguous():
        raise LmError("targets must be contiguous, of the logits' shape without the last dimension")
    return _idtype(targets)


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None,
                   scale: float = 1.0, top: int = 0, ignore: int = -100,
                   dev_err: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None,
                   stream=None) -> TokenLogprobs:
    """lm_token_logprobs: log softmax(scale * logits) at each row's target (0
    where it is `ignore`), the entropy, and the `top` (up to TOP_MAX) likeliest
    words, of equal ones the lowest ids first. logits float32 or bfloat16, the
    words along the last dimension, -infinity where a word is masked. dev_err
    tells of targets outside the vocabulary (their logp is NaN). Without `ws` the
    call takes its workspace from torch's allocator. Not recorded by autograd, as
    ``rel_bias``."""
    if _calls and ws is None and stream is None and logits.is_cuda:
        here = _this_device()
        r = _calls.token_logprobs(here, _stream_of(here), logits, targets, scale, top, ignore,
                                  dev_err)
        if r is not None:
            return TokenLogprobs(*r)
    _no_graph("token_logprobs", logits, gradient=_LOGP_GRADIENT)
    _dev(logits, "logits")
    device = logits.device
    N, V, ld = _matrix(logits, "logits")
    dtype, idtype = _gtype(logits), _targets(targets, logits)
    _same_device(device, targets, dev_err, None if ws is None else ws.buf)
    _one_of(dev_err, torch.int32, "dev_err")
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return token_logprobs(logits, targets, scale, top, ignore, dev_err, ws, stream)
    shape = logits.shape[:-1]
    found = _empty((3 if targets is None else 4, *shape), torch.float32, device, stream).unbind()
    entropy, peak, log_sum = found[:3]
    logp = None if targets is None else found[3]
    top_logp = top_ids = None
    if top > 0:
        top_logp = _empty((*shape, top), torch.float32, device, stream)
        top_ids = _empty((*shape, top), torch.int32, device, stream)
    need = _lib.lm_token_logprobs_workspace_bytes(N, V, dtype, top)
    buf = None
    if need:
        buf = ws.get(need) if ws is not None else _empty((need,), torch.uint8, device, stream)
    _call(_lib.lm_token_logprobs(
        _ptr(logits), ld, N, V, dtype, _ptr(targets), idtype, ignore, scale, top, _ptr(logp),
        _ptr(entropy), _ptr(peak), _ptr(log_sum), _ptr(top_logp), _ptr(top_ids), _ptr(dev_err),
        _ptr(buf), need, _on(device, stream)), "lm_token_logprobs")
    return TokenLogprobs(logp, entropy, peak, log_sum, top_logp, top_ids)


def token_logprobs_grad(logits: torch.Tensor, targets: Optional[torch.Tensor],
                        peak: torch.Tensor, log_sum: torch.Tensor,
                        dlogp: Optional[torch.Tensor] = None,
                        entropy: Optional[torch.Tensor] = None,
                        dentropy: Optional[torch.Tensor] = None, scale: float = 1.0,
                        ignore: int = -100, out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """lm_token_logprobs_grad: the logits' gradient, in their dtype, from those
    of logp (dlogp) and of the entropy (dentropy, with the entropy itself), and
    what ``token_logprobs`` returned. `out` may be the logits. Not recorded by
    autograd, as ``rel_bias``."""
    if _calls and out is None and stream is None and logits.is_cuda:
        here = _this_device()
        r = _calls.token_logprobs_grad(here, _stream_of(here), logits, targets, peak, log_sum,
                                       dlogp, entropy, dentropy, scale, ignore)
        if r is not None:
            return r[0]
    _no_graph("token_logprobs_grad", logits, dlogp, dentropy, out, gradient=_LOGP_GRADIENT)
    _no_tangent("token_logprobs_grad", peak, log_sum, entropy)
    _dev(logits, "logits")
    device = logits.device
    N, V, ld = _matrix(logits, "logits")
    dtype, idtype = _gtype(logits), _targets(targets, logits)
    for t, what in ((peak, "peak"), (log_sum, "log_sum"), (dlogp, "dlogp"), (entropy, "entropy"),
                    (dentropy, "dentropy")):
        _vector(t, N, what)
    if dlogp is not None and targets is None:
        raise LmError("dlogp needs targets")
    if dentropy is not None and entropy is None:
        raise LmError("dentropy needs entropy")
    _same_device(device, targets, peak, log_sum, dlogp, entropy, dentropy, out)
    if _elsewhere(device, stream):
        with torch.cuda.device(device):
            return token_logprobs_grad(logits, targets, peak, log_sum, dlogp, entropy, dentropy,
                                       scale, ignore, out, stream)
    given = out
    if out is None:
        out = _new(logits, stream)
    _call(_lib.lm_token_logprobs_grad(
        _ptr(logits), ld, N, V, dtype, _ptr(targets), idtype, ignore, scale, _ptr(peak),
        _ptr(log_sum), _ptr(dlogp), _ptr(entropy), _ptr(dentropy), _ptr(out),
        _like(out, logits, "out"), _on(device, stream)), "lm_token_logprobs_grad")
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
