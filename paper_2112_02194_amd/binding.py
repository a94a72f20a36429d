"""ctypes binding of libals.so: same names as the C ABI (include/als.h), argument marshalling only.

Tables are torch tensors on the GPU (fp32 or bf16, row-major [rows, d]); sparse
matrices are ``Csr`` triples of device tensors.  Kernels are enqueued on torch's
current stream.  There is no CPU fallback: if the library is missing or no GPU
is visible, calls raise.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from dataclasses import dataclass
from operator import attrgetter
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libals.so")

ALS_OK, ALS_EINVAL, ALS_ESHAPE, ALS_EDTYPE, ALS_EALIAS, ALS_ENOTSPD, ALS_ENOMEM, ALS_EHIP = range(8)
ALS_F32, ALS_BF16 = 0, 1
PATH_AUTO, PATH_PRIMAL, PATH_DUAL = 0, 1, 2
SOLVER_DIRECT, SOLVER_CG, SOLVER_CG_FREE = 0, 1, 2

EXPORTS = ["als_create", "als_destroy", "als_gramian", "als_solve_rows", "als_epoch", "als_loss",
           "als_status_sync", "als_check_csr", "als_copy_probe", "als_set_timing", "als_get_timing",
           "als_strerror", "als_last_error", "als_gramian_static", "als_static_last_error", "als_topk",
           "als_quantize", "als_dequantize", "als_scores", "als_adjust", "als_select",
           "als_recur", "als_recur_step", "als_recur_backward", "als_sum_rows", "als_clip", "als_beam", "als_reorder"]


class c_als_csr(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("indptr", ctypes.c_void_p), ("indices", ctypes.c_void_p), ("values", ctypes.c_void_p)]


class c_als_table(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("d", ctypes.c_int32),
                ("ld", ctypes.c_int64), ("dtype", ctypes.c_int)]


class c_als_params(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("lambda_", ctypes.c_float), ("path", ctypes.c_int32),
                ("dual_max_k", ctypes.c_int32), ("split_nnz", ctypes.c_int32), ("solver", ctypes.c_int32),
                ("cg_max_iters", ctypes.c_int32), ("cg_tol", ctypes.c_float)]


class c_als_qtable(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("d", ctypes.c_int32),
                ("group", ctypes.c_int32)]


class c_als_matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("dtype", ctypes.c_int)]


class c_als_rules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("entries", ctypes.c_void_p), ("bias", ctypes.c_void_p),  # the lists: to c_als_csr
                ("allowed", ctypes.c_void_p), ("allowed_ld", ctypes.c_int64), ("penalties", ctypes.c_void_p),
                ("repetition", ctypes.c_float), ("presence", ctypes.c_float), ("frequency", ctypes.c_float)]


class c_als_beams(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int64), ("beams", ctypes.c_int32), ("k", ctypes.c_int32), ("ids", ctypes.c_void_p),
                ("scores", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("totals", ctypes.c_void_p), ("last", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("factors", ctypes.c_void_p), ("n_factors", ctypes.c_int32), ("end", ctypes.c_int32),
                ("temperature", ctypes.c_float)]


class AlsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libals status {status}: {message}")
        self.status = status


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libals.so (built by ``__graft_entry__.build()``); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not found: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(path)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    P = ctypes.POINTER
    lib.als_create.argtypes = [P(vp), i32]
    lib.als_destroy.argtypes = [vp]
    lib.als_gramian.argtypes = [vp, P(c_als_table), vp, vp]
    lib.als_solve_rows.argtypes = [vp, P(c_als_csr), P(c_als_table), vp, P(c_als_params), P(c_als_table), i64, i64, vp]
    lib.als_epoch.argtypes = [vp, P(c_als_csr), P(c_als_csr), P(c_als_table), P(c_als_table), P(c_als_params), vp]
    lib.als_loss.argtypes = [vp, P(c_als_csr), P(c_als_table), P(c_als_table), P(c_als_params), P(ctypes.c_double), vp]
    lib.als_status_sync.argtypes = [vp, vp]
    lib.als_check_csr.argtypes = [vp, P(c_als_csr), vp]
    lib.als_set_timing.argtypes = [vp, i32]
    lib.als_get_timing.argtypes = [vp, P(ctypes.c_double)]
    lib.als_copy_probe.argtypes = [vp, vp, vp, i64, vp]
    for name in EXPORTS[:11]:
        getattr(lib, name).restype = i32
    lib.als_strerror.argtypes = [i32]
    lib.als_strerror.restype = ctypes.c_char_p
    lib.als_last_error.argtypes = [vp]
    lib.als_last_error.restype = ctypes.c_char_p
    lib.als_gramian_static.argtypes = [i32, P(c_als_table), vp, vp]
    lib.als_gramian_static.restype = i32
    lib.als_topk.argtypes = [vp, P(c_als_table), P(c_als_table), P(c_als_csr), i32, vp, vp, vp]
    lib.als_topk.restype = i32
    lib.als_quantize.argtypes = [vp, P(c_als_table), P(c_als_qtable), vp]
    lib.als_dequantize.argtypes = [vp, P(c_als_qtable), P(c_als_table), vp]
    lib.als_scores.argtypes = [vp, P(c_als_table), P(c_als_qtable), P(c_als_matrix), vp]
    lib.als_adjust.argtypes = [vp, P(c_als_matrix), P(c_als_rules), P(c_als_matrix), vp]
    lib.als_select.argtypes = [vp, P(c_als_matrix), P(c_als_rules), ctypes.c_float, i32, vp, vp, vp, vp]
    lib.als_recur.argtypes = [vp, P(c_als_csr), P(c_als_table), P(c_als_table), P(c_als_table), P(c_als_table), P(c_als_table), vp]
    lib.als_recur_step.argtypes = [vp, vp, vp, P(c_als_table), P(c_als_table), P(c_als_table), P(c_als_table), vp]
    lib.als_recur_backward.argtypes = [vp, P(c_als_csr)] + [P(c_als_table)] * 9 + [vp]
    lib.als_sum_rows.argtypes = [vp, P(c_als_csr), P(c_als_table), P(c_als_table), vp]
    lib.als_clip.argtypes = [vp, vp, vp, i32, ctypes.c_double, vp, vp]
    lib.als_beam.argtypes = [vp, P(c_als_beams), vp, vp, vp, vp, vp]
    lib.als_reorder.argtypes = [vp, vp, i64, i32, vp, vp, i32, vp]
    for name in EXPORTS[16:]:
        getattr(lib, name).restype = i32
    lib.als_static_last_error.argtypes = []
    lib.als_static_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


@dataclass
class Csr:
    """CSR matrix on the GPU: int64 indptr [rows+1], int32 indices [nnz], optional fp32 values.  ``indices`` may be None for
    als_recur and als_recur_backward: an entry for each of the ``cols`` table rows, in their order."""
    rows: int
    cols: int
    indptr: torch.Tensor
    indices: Optional[torch.Tensor]
    values: Optional[torch.Tensor] = None

    @property
    def nnz(self) -> int:
        return self.cols if self.indices is None else int(self.indices.numel())

    def c(self) -> c_als_csr:
        indptr, indices, values = self.indptr, self.indices, self.values
        if indices is None:
            assert indptr.dtype is torch.int64 and indptr.is_contiguous() and indptr.numel() == self.rows + 1 and values is None
            return c_als_csr(self.rows, self.cols, self.cols, indptr.data_ptr(), None, None)
        nnz, vals = indices.numel(), None
        assert indptr.dtype is torch.int64 and indices.dtype is torch.int32
        assert indptr.is_contiguous() and indices.is_contiguous()
        assert indptr.numel() == self.rows + 1
        if values is not None:
            assert values.dtype is torch.float32 and values.is_contiguous()
            assert values.numel() == nnz
            vals = values.data_ptr()
        return c_als_csr(self.rows, self.cols, nnz, indptr.data_ptr(), indices.data_ptr() if nnz else None, vals)


def _table(t: torch.Tensor) -> c_als_table:
    if t.dim() != 2:
        raise ValueError("table must be 2-D with unit column stride")
    rows, d = t.shape
    ld, unit = t.stride() if rows else (d, 1)
    if unit != 1:
        raise ValueError("table must be 2-D with unit column stride")
    dtype = t.dtype
    if dtype is torch.float32:
        dt = ALS_F32
    elif dtype is torch.bfloat16:
        dt = ALS_BF16
    else:
        raise TypeError("table dtype must be float32 or bfloat16")
    return c_als_table(t.data_ptr() if rows and d else None, rows, d, ld if rows > 1 else max(ld, d), dt)


# torch's own short ways to the handle (about a microsecond less a call than a Stream object); where a version lacks them, the public one
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """Handle of torch's current stream on the current device."""
    if _raw_stream is None or _current_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


class Context:
    """Owns an ``als_ctx`` (workspace on one GPU)."""

    def __init__(self, device: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("libals needs a GPU: torch.cuda.is_available() is False")
        self.lib = load_library()
        self.handle = ctypes.c_void_p()
        st = self.lib.als_create(ctypes.byref(self.handle), device)
        if st != ALS_OK:
            raise AlsError(st, self.lib.als_strerror(st).decode())
        self.device = torch.device("cuda", device)

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.als_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != ALS_OK:
            raise AlsError(st, f"{self.lib.als_strerror(st).decode()}: {self.lib.als_last_error(self.handle).decode()}")


def make_params(alpha: float, lam: float, path: int = PATH_AUTO, dual_max_k: int = 0, split_nnz: int = 0,
                solver: int = 0, cg_max_iters: int = 0, cg_tol: float = 0.0) -> c_als_params:
    return c_als_params(alpha, lam, path, dual_max_k, split_nnz, solver, cg_max_iters, cg_tol)


def als_gramian(ctx: Context, V: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    d = V.shape[1]
    G = out if out is not None else torch.empty((d, d), dtype=torch.float32, device=V.device)
    tv = _table(V)
    ctx._check(ctx.lib.als_gramian(ctx.handle, ctypes.byref(tv), G.data_ptr(), _stream()))
    return G


def als_gramian_static(V: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """als_gramian without a context and without any allocation: ``out`` (fp32 [d, d]) is the caller's."""
    lib = load_library()
    assert out.dtype == torch.float32 and out.is_contiguous() and out.shape == (V.shape[1], V.shape[1])
    tv = _table(V)
    st = lib.als_gramian_static(V.device.index or 0, ctypes.byref(tv), out.data_ptr(), _stream())
    if st != ALS_OK:
        raise AlsError(st, f"{lib.als_strerror(st).decode()}: {lib.als_static_last_error().decode()}")
    return out


def als_solve_rows(ctx: Context, Y: Csr, V: torch.Tensor, G: torch.Tensor, params: c_als_params, X: torch.Tensor,
                   row_begin: int = 0, row_end: Optional[int] = None) -> torch.Tensor:
    cy, tv, tx = Y.c(), _table(V), _table(X)
    assert G.dtype == torch.float32 and G.is_contiguous()
    row_end = Y.rows if row_end is None else row_end
    ctx._check(ctx.lib.als_solve_rows(ctx.handle, ctypes.byref(cy), ctypes.byref(tv), G.data_ptr(),
                                      ctypes.byref(params), ctypes.byref(tx), row_begin, row_end, _stream()))
    return X


def als_epoch(ctx: Context, Y: Csr, Yt: Csr, W: torch.Tensor, H: torch.Tensor, params: c_als_params) -> None:
    cy, cyt, tw, th = Y.c(), Yt.c(), _table(W), _table(H)
    ctx._check(ctx.lib.als_epoch(ctx.handle, ctypes.byref(cy), ctypes.byref(cyt), ctypes.byref(tw),
                                 ctypes.byref(th), ctypes.byref(params), _stream()))


def als_loss(ctx: Context, Y: Csr, W: torch.Tensor, H: torch.Tensor, params: c_als_params) -> float:
    cy, tw, th = Y.c(), _table(W), _table(H)
    out = ctypes.c_double()
    ctx._check(ctx.lib.als_loss(ctx.handle, ctypes.byref(cy), ctypes.byref(tw), ctypes.byref(th),
                                ctypes.byref(params), ctypes.byref(out), _stream()))
    return out.value


def als_topk(ctx: Context, Q: torch.Tensor, H: torch.Tensor, k: int, exclude: Optional[Csr] = None):
    """Best k rows of H per row of Q by inner product -> (ids int32 [nq, k], scores fp32 [nq, k])."""
    tq, th = _table(Q), _table(H)
    ids = torch.empty((Q.shape[0], k), dtype=torch.int32, device=Q.device)
    scores = torch.empty((Q.shape[0], k), dtype=torch.float32, device=Q.device)
    ex = exclude.c() if exclude is not None else None
    ctx._check(ctx.lib.als_topk(ctx.handle, ctypes.byref(tq), ctypes.byref(th), ctypes.byref(ex) if ex is not None else None,
                                k, ids.data_ptr(), scores.data_ptr(), _stream()))
    return ids, scores


@dataclass
class QTable:
    """Table in 4 bits an entry: uint8 codes [rows, d/2] and bf16 scales [rows, d/group], both contiguous.  A range of
    rows of both is such a table too."""
    codes: torch.Tensor
    scales: torch.Tensor

    @property
    def shape(self):
        return self.codes.shape[0], 2 * self.codes.shape[1]

    @property
    def group(self) -> int:
        return 2 * self.codes.shape[1] // max(1, self.scales.shape[1])

    def c(self) -> c_als_qtable:
        codes, scales = self.codes, self.scales
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.bfloat16:
            raise TypeError("codes must be uint8 and scales bfloat16")
        if codes.dim() != 2 or scales.dim() != 2 or not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be 2-D and contiguous")
        rows, half = codes.shape
        scale_rows, groups = scales.shape
        if scale_rows != rows:
            raise ValueError("codes and scales differ in rows")
        if groups < 1 or 2 * half % groups:
            raise ValueError("a row must be a whole number of groups")
        return c_als_qtable(codes.data_ptr() or None, scales.data_ptr() or None, rows, 2 * half, 2 * half // groups)


@dataclass
class Rules:
    """What is done to scores [rows, cols], in this order; everything is optional.

    ``history``: Csr of the items a row has had, an item as often as it was had; such scores are divided by
    ``repetition`` (multiplied where negative), then lowered by ``frequency`` for every time and by ``presence`` once;
    ``penalties`` (fp32 [rows, 3]: repetition, presence, frequency) takes the place of the three numbers.
    ``bias`` (fp32 [cols]) and ``entries`` (Csr with values) are added.  ``allowed``: int32 words [rows or 1, >= cols/32],
    bit i % 32 of word i // 32 clear: the score of item i is -inf."""
    history: Optional[Csr] = None
    repetition: float = 1.0
    presence: float = 0.0
    frequency: float = 0.0
    penalties: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    entries: Optional[Csr] = None
    allowed: Optional[torch.Tensor] = None

    def tensors(self):
        out = [self.penalties, self.bias, self.allowed]
        for y in (self.history, self.entries):
            if y is not None:
                out += (y.indptr, y.indices, y.values)
        return out

    def c(self, rows: int, cols: int) -> c_als_rules:
        out = c_als_rules()
        out.repetition, out.presence, out.frequency = self.repetition, self.presence, self.frequency
        out.lists = lists = []  # keeps what the structure points to
        if self.history is not None:
            lists.append(self.history.c())
            out.history = ctypes.addressof(lists[-1])
        if self.entries is not None:
            lists.append(self.entries.c())
            out.entries = ctypes.addressof(lists[-1])
        bias, penalties, allowed = self.bias, self.penalties, self.allowed
        if bias is not None:
            if bias.dtype is not torch.float32 or bias.dim() != 1 or bias.numel() != cols or not bias.is_contiguous():
                raise ValueError("bias must be contiguous float32 [cols]")
            out.bias = bias.data_ptr()
        if penalties is not None:
            if penalties.dtype is not torch.float32 or penalties.shape != (rows, 3) or not penalties.is_contiguous():
                raise ValueError("penalties must be contiguous float32 [rows, 3]")
            out.penalties = penalties.data_ptr()
        if allowed is not None:
            if allowed.dtype is not torch.int32 or allowed.dim() != 2:
                raise ValueError("allowed must be int32 [rows or 1, at least (cols + 31) // 32]")
            sets, words = allowed.shape
            if (sets != rows and sets != 1) or words < (cols + 31) // 32:
                raise ValueError("allowed must be int32 [rows or 1, at least (cols + 31) // 32]")
            step, unit = allowed.stride()
            if words > 1 and unit != 1:
                raise ValueError("allowed must have unit column stride")
            out.allowed = allowed.data_ptr() or None
            # one set for all rows: no step from row to row (an expanded tensor has none by itself)
            out.allowed_ld = 0 if sets == 1 else step
        return out


def _matrix(t: torch.Tensor) -> c_als_matrix:
    if t.dim() != 2:
        raise ValueError("scores must be 2-D with unit column stride")
    rows, cols = t.shape
    ld, unit = t.stride()
    if cols > 1 and unit != 1:
        raise ValueError("scores must be 2-D with unit column stride")
    dtype = t.dtype
    if dtype is torch.float32:
        dt = ALS_F32
    elif dtype is torch.bfloat16:
        dt = ALS_BF16
    else:
        raise TypeError("scores must be float32 or bfloat16")
    return c_als_matrix(t.data_ptr() or None, rows, cols, ld if rows > 1 else max(ld, cols), dt)


def _here(ctx: Context, *tensors) -> None:
    device = ctx.device.index
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("every tensor must be on the context's GPU")


def als_quantize(ctx: Context, X: torch.Tensor, group: int = 32, out: Optional[QTable] = None) -> QTable:
    """X in 4 bits an entry, one bf16 scale per ``group`` entries of a row (at most d, so 16 for d = 16)."""
    tx = _table(X)
    if out is None:
        rows, d = X.shape
        if group not in (16, 32, 64, 128) or group > d:
            raise ValueError("group must be 16, 32, 64 or 128 and at most d")
        out = QTable(torch.empty((rows, d // 2), dtype=torch.uint8, device=X.device),
                     torch.empty((rows, d // group), dtype=torch.bfloat16, device=X.device))
    ct = out.c()
    _here(ctx, X, out.codes, out.scales)
    ctx._check(ctx.lib.als_quantize(ctx.handle, ctypes.byref(tx), ctypes.byref(ct), _stream()))
    return out


def als_dequantize(ctx: Context, T: QTable, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of T as an ordinary table."""
    X = out if out is not None else torch.empty(T.shape, dtype=dtype, device=T.codes.device)
    ct, tx = T.c(), _table(X)
    _here(ctx, X, T.codes, T.scales)
    ctx._check(ctx.lib.als_dequantize(ctx.handle, ctypes.byref(ct), ctypes.byref(tx), _stream()))
    return X


def als_scores(ctx: Context, Q: torch.Tensor, T: QTable, out: Optional[torch.Tensor] = None,
               dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """Inner products of every row of Q with every row of T -> [Q rows, T rows], fp32 or bf16."""
    S = out if out is not None else torch.empty((Q.shape[0], T.codes.shape[0]), dtype=dtype, device=Q.device)
    tq, ct, cs = _table(Q), T.c(), _matrix(S)
    _here(ctx, Q, T.codes, T.scales, S)
    ctx._check(ctx.lib.als_scores(ctx.handle, ctypes.byref(tq), ctypes.byref(ct), ctypes.byref(cs), _stream()))
    return S


def als_adjust(ctx: Context, S: torch.Tensor, rules: Rules, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """S changed by the rules, in place unless ``out`` (of S's shape, fp32 or bf16) is given."""
    Y = out if out is not None else S
    cs, cy, cr = _matrix(S), _matrix(Y), rules.c(*S.shape)
    _here(ctx, S, Y, *rules.tensors())
    ctx._check(ctx.lib.als_adjust(ctx.handle, ctypes.byref(cs), ctypes.byref(cr), ctypes.byref(cy), _stream()))
    return Y


def als_select(ctx: Context, S: torch.Tensor, k: int, rules: Optional[Rules] = None, temperature: float = 1.0):
    """Best k of every row of S changed by the rules -> (ids int32 [rows, k], scores fp32 [rows, k], lse fp32 [rows]).

    ``scores / temperature - lse[:, None]`` are the log-probabilities of the returned items among all of the row."""
    cs = _matrix(S)
    cr = None
    if rules is not None:
        cr = ctypes.byref(rules.c(*S.shape))
        _here(ctx, *rules.tensors())
    _here(ctx, S)
    ids = torch.empty((S.shape[0], max(k, 0)), dtype=torch.int32, device=S.device)
    scores = torch.empty((S.shape[0], max(k, 0)), dtype=torch.float32, device=S.device)
    lse = torch.empty((S.shape[0],), dtype=torch.float32, device=S.device)
    ctx._check(ctx.lib.als_select(ctx.handle, ctypes.byref(cs), cr, temperature, k, ids.data_ptr(), scores.data_ptr(),
                                  lse.data_ptr(), _stream()))
    return ids, scores, lse


def _opt(t: Optional[torch.Tensor]):
    """A table that may be left out, as an argument."""
    return None if t is None else ctypes.byref(_table(t))


def _ids(t: Optional[torch.Tensor], rows: int, name: str):
    """Address of int32 [rows], one after the other."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.dim() != 1 or t.shape[0] != rows or not t.is_contiguous():
        raise ValueError(name + " must be contiguous int32, one per row")
    return t.data_ptr() or None


def als_recur(ctx: Context, Y: Csr, V: torch.Tensor, F: torch.Tensor, H0: Optional[torch.Tensor] = None, all_states: bool = False,
              dtype: torch.dtype = torch.float32, last: Optional[torch.Tensor] = None, states: Optional[torch.Tensor] = None):
    """h = s h + (1 - s) V[item], s = sigmoid(F[item]), over every row's entries in their order -> (last, states or None).

    ``last`` [Y.rows, d]: each row's last state; ``states`` [Y.nnz, d]: the state after each entry, where ``all_states`` or a
    tensor for them is given.  Tensors that are given are written, others are made in ``dtype``.  Y.indices None: entry p takes row p."""
    d = V.shape[1]
    if last is None:
        last = torch.empty((Y.rows, d), dtype=dtype, device=V.device)
    if states is None and all_states:
        states = torch.empty((Y.nnz, d), dtype=dtype, device=V.device)
    cy, tv, tf, tl = Y.c(), _table(V), _table(F), _table(last)
    _here(ctx, V, F, H0, last, states, Y.indptr, Y.indices)
    ctx._check(ctx.lib.als_recur(ctx.handle, ctypes.byref(cy), ctypes.byref(tv), ctypes.byref(tf), _opt(H0), _opt(states),
                                 ctypes.byref(tl), _stream()))
    return last, states


def als_recur_step(ctx: Context, items: torch.Tensor, V: torch.Tensor, F: torch.Tensor, H: torch.Tensor,
                   parents: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One more entry for each row: s H[parent] + (1 - s) V[item].  ``out`` may be H where there are no parents."""
    rows = items.shape[0]
    X = out if out is not None else torch.empty((rows, H.shape[1]), dtype=H.dtype, device=H.device)
    if X.shape[0] != rows:
        raise ValueError("out must have one row per item")
    tv, tf, th, tx = _table(V), _table(F), _table(H), _table(X)
    _here(ctx, items, V, F, H, parents, X)
    ctx._check(ctx.lib.als_recur_step(ctx.handle, _ids(items, rows, "items"), _ids(parents, rows, "parents"), ctypes.byref(tv),
                                      ctypes.byref(tf), ctypes.byref(th), ctypes.byref(tx), _stream()))
    return X


def als_recur_backward(ctx: Context, Y: Csr, V: torch.Tensor, F: torch.Tensor, states: torch.Tensor,
                       d_states: Optional[torch.Tensor] = None, d_last: Optional[torch.Tensor] = None, H0: Optional[torch.Tensor] = None,
                       dtype: Optional[torch.dtype] = None, out=None):
    """Gradients of als_recur -> (dV [nnz, d], dF [nnz, d], dH0 [rows, d] or None without H0), the first two a row per entry,
    of the states' type: als_sum_rows over the entries with the same item gives the tables'.  ``out``: the three to write."""
    dtype = states.dtype if dtype is None else dtype
    if out is not None:
        dV, dF, dH0 = out
    else:
        dV, dF = (torch.empty(states.shape, dtype=dtype, device=V.device) for _ in range(2))
        dH0 = None if H0 is None else torch.empty((Y.rows, V.shape[1]), dtype=dtype, device=V.device)
    cy, tv, tf, ts, tdv, tdf = Y.c(), _table(V), _table(F), _table(states), _table(dV), _table(dF)
    _here(ctx, V, F, states, d_states, d_last, H0, dV, dF, dH0, Y.indptr, Y.indices)
    ctx._check(ctx.lib.als_recur_backward(ctx.handle, ctypes.byref(cy), ctypes.byref(tv), ctypes.byref(tf), _opt(H0), ctypes.byref(ts),
                                          _opt(d_states), _opt(d_last), ctypes.byref(tdv), ctypes.byref(tdf), _opt(dH0), _stream()))
    return dV, dF, dH0


def als_sum_rows(ctx: Context, Y: Csr, E: torch.Tensor, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """Sum of the rows of E that each row of Y stores, times Y's values -> [Y.rows, d]."""
    X = out if out is not None else torch.empty((Y.rows, E.shape[1]), dtype=dtype, device=E.device)
    cy, te, tx = Y.c(), _table(E), _table(X)
    _here(ctx, E, X, Y.indptr, Y.indices, Y.values)
    ctx._check(ctx.lib.als_sum_rows(ctx.handle, ctypes.byref(cy), ctypes.byref(te), ctypes.byref(tx), _stream()))
    return X


_CODES = {torch.float32: ALS_F32, torch.bfloat16: ALS_BF16}


_dtype_of = attrgetter("dtype")


def _flat_values(device: int, tensors):
    """Tensors whose elements lie one after the other, a row each, as an array of c_als_matrix (five 64-bit words)."""
    count, Tensor = len(tensors), torch.Tensor
    words, sizes = array("q", bytes(40 * count)), array("q", map(Tensor.numel, tensors))
    words[0::5], words[1::5], words[2::5], words[3::5] = array("q", map(Tensor.data_ptr, tensors)), array("q", (1,)) * count, sizes, sizes
    try:
        words[4::5] = array("q", map(_CODES.__getitem__, map(_dtype_of, tensors)))
    except KeyError:
        raise TypeError("tensors must be float32 or bfloat16") from None
    if set(map(Tensor.get_device, tensors)) - {device}:
        raise ValueError("every tensor must be on the context's GPU")
    return words


def _row_values(device: int, tensors):
    """The same of 2-D tensors with unit column stride."""
    words = array("q")
    for t in tensors:
        m = _matrix(t)
        if t.get_device() != device:
            raise ValueError("every tensor must be on the context's GPU")
        words.extend((m.data or 0, m.rows, m.cols, m.ld, m.dtype))
    return words


def als_clip(ctx: Context, tensors, bound: float, out=None) -> torch.Tensor:
    """The norm over all elements of all tensors (float64, on the GPU); the tensors are scaled by bound / norm where that is
    below 1, in place or into ``out`` (a tensor for each).  Tensors of any shape whose elements lie one after the other, or 2-D
    ones with unit column stride."""
    n, device = len(tensors), ctx.device.index
    if out is not None and len(out) != n:
        raise ValueError("out must have a tensor for each")
    contiguous = torch.Tensor.is_contiguous
    if all(map(contiguous, tensors)) and (out is None or all(map(contiguous, out))):
        values = _flat_values
    else:  # those whose elements lie one after the other as one row
        if out is not None and any([x.shape != y.shape for x, y in zip(tensors, out)]):
            raise ValueError("out must have a tensor of the same shape for each")
        lone = [contiguous(x) and (out is None or contiguous(out[j])) for j, x in enumerate(tensors)]
        tensors = [x.view(1, -1) if f else x for x, f in zip(tensors, lone)]
        out = out and [y.view(1, -1) if f else y for y, f in zip(out, lone)]
        values = _row_values
    X, Y = values(device, tensors), None if out is None else values(device, out)
    if Y is not None and X[2::5] != Y[2::5]:
        raise ValueError("out must have a tensor of the same size for each")
    norm = torch.empty((), dtype=torch.float64, device=ctx.device)
    ctx._check(ctx.lib.als_clip(ctx.handle, X.buffer_info()[0], None if Y is None else Y.buffer_info()[0], n, bound, norm.data_ptr(), _stream()))
    return norm


def _per_row(t: Optional[torch.Tensor], rows: int, dtype: torch.dtype, name: str):
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != rows or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype}, one per beam")
    return t.data_ptr() or None


def als_beam(ctx: Context, ids: torch.Tensor, scores: torch.Tensor, lse: Optional[torch.Tensor], totals: Optional[torch.Tensor], beams: int,
             temperature: float = 1.0, last: Optional[torch.Tensor] = None, end: int = -1, lengths: Optional[torch.Tensor] = None,
             factors: Optional[torch.Tensor] = None):
    """The best ``beams`` continuations of each group of ``beams`` rows, from the rows' best items as als_select returns them ->
    (parents int32, items int32, totals fp32, lengths int32), one per beam, a group's best first.

    totals + scores / temperature - lse orders them (times ``factors``[length] where given; None for ``totals``: the first step, a
    group's first row alone counts).  ``last``: each beam's last item; a beam whose last is ``end`` stays as it is."""
    rows, k = ids.shape
    if beams < 1 or rows % beams:
        raise ValueError("rows must be a whole number of groups of beams")
    if ids.dtype is not torch.int32 or scores.dtype is not torch.float32 or scores.shape != ids.shape:
        raise ValueError("ids must be int32 [rows, k] and scores float32 of the same shape")
    if not ids.is_contiguous() or not scores.is_contiguous():
        raise ValueError("ids and scores must be contiguous")
    if factors is not None and (factors.dtype is not torch.float32 or factors.dim() != 1 or not factors.is_contiguous() or not factors.numel()):
        raise ValueError("factors must be contiguous float32, one at least")
    c = c_als_beams(rows // beams, beams, k, ids.data_ptr() or None, scores.data_ptr() or None, _per_row(lse, rows, torch.float32, "lse"),
                    _per_row(totals, rows, torch.float32, "totals"), _per_row(last, rows, torch.int32, "last"),
                    _per_row(lengths, rows, torch.int32, "lengths"), None if factors is None else factors.data_ptr(),
                    0 if factors is None else factors.numel(), end, temperature)
    _here(ctx, ids, scores, lse, totals, last, lengths, factors)
    parents, items, new_lengths = torch.empty((3, rows), dtype=torch.int32, device=ids.device).unbind()
    new_totals = torch.empty(rows, dtype=torch.float32, device=ids.device)
    ctx._check(ctx.lib.als_beam(ctx.handle, ctypes.byref(c), parents.data_ptr(), items.data_ptr(), new_totals.data_ptr(),
                                new_lengths.data_ptr(), _stream()))
    return parents, items, new_totals, new_lengths


def _states(device: int, tensors, rows: int):
    """What goes with the beams, a row each whose elements lie one after the other, as an array of c_als_matrix (five 64-bit words)."""
    words = array("q")
    for t in tensors:
        if t.dim() < 1 or t.shape[0] != rows:
            raise ValueError("a state must have one row per beam")
        es = t.element_size()
        if es not in (2, 4, 8):
            raise TypeError("elements of a state must have 2, 4 or 8 bytes")
        if t.is_contiguous():
            cols = ld = t.numel() // rows if rows else 0
        else:
            cols = 1
            for size, step in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
                if size != 1 and step != cols:
                    raise ValueError("the elements of a state's row must lie one after the other")
                cols *= size
            ld = t.stride(0) if rows > 1 else cols
        if es == 8:
            cols, ld = 2 * cols, 2 * ld
        if t.get_device() != device:
            raise ValueError("every tensor must be on the context's GPU")
        words.extend((t.data_ptr(), rows, cols, ld, ALS_BF16 if es == 2 else ALS_F32))
    return words


def als_reorder(ctx: Context, parents: torch.Tensor, beams: int, states, out=None):
    """Row parents[r] of every state to row r, in place or into ``out`` (a tensor for each); elements of 2, 4 or 8 bytes of any kind.
    Rows of parents outside r's own group of ``beams`` rows (-1, say) become zeros."""
    rows, n, device = parents.shape[0], len(states), ctx.device.index
    if beams < 1 or rows % beams:
        raise ValueError("rows must be a whole number of groups of beams")
    if out is not None and (len(out) != n or any([x.dtype is not y.dtype or x.shape != y.shape for x, y in zip(states, out)])):
        raise ValueError("out must have a tensor of the same shape and type for each")
    X, Y = _states(device, states, rows), None if out is None else _states(device, out, rows)
    p = _ids(parents, rows, "parents")
    _here(ctx, parents)
    ctx._check(ctx.lib.als_reorder(ctx.handle, p, rows // beams, beams, X.buffer_info()[0], None if Y is None else Y.buffer_info()[0], n, _stream()))
    return states if out is None else out


def als_status_sync(ctx: Context) -> None:
    ctx._check(ctx.lib.als_status_sync(ctx.handle, _stream()))


def als_check_csr(ctx: Context, Y: Csr) -> None:
    cy = Y.c()
    ctx._check(ctx.lib.als_check_csr(ctx.handle, ctypes.byref(cy), _stream()))


def als_copy_probe(ctx: Context, src: torch.Tensor, dst: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes and src.is_contiguous() and dst.is_contiguous()
    ctx._check(ctx.lib.als_copy_probe(ctx.handle, src.data_ptr(), dst.data_ptr(), nbytes, _stream()))


def als_set_timing(ctx: Context, enabled: bool) -> None:
    ctx._check(ctx.lib.als_set_timing(ctx.handle, int(enabled)))


TIMING_SLOTS = (["gramian", "classify", "transform_z", "transform_x", "primal", "segment", "reduce", "dual_k4", "dual_k8"]
                + [f"dual_k{16 * (c + 1)}" for c in range(8)])


def als_get_timing(ctx: Context) -> dict:
    """ms per kernel slot, and under "launches" the number of timed launches of each slot."""
    n = len(TIMING_SLOTS)
    buf = (ctypes.c_double * (2 * n))()
    ctx._check(ctx.lib.als_get_timing(ctx.handle, buf))
    out = dict(zip(TIMING_SLOTS, list(buf)[:n]))
    out["launches"] = dict(zip(TIMING_SLOTS, list(buf)[n:]))
    return out
