"""ctypes binding of libals.so: same names as the C ABI (include/als.h), argument marshalling only.

Tables are torch tensors on the GPU (fp32 or bf16, row-major [rows, d]); sparse
matrices are ``Csr`` triples of device tensors.  Kernels are enqueued on torch's
current stream.  There is no CPU fallback: if the library is missing or no GPU
is visible, calls raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
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
           "als_quantize", "als_dequantize", "als_scores", "als_adjust", "als_select"]


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
    for name in ("als_quantize", "als_dequantize", "als_scores", "als_adjust", "als_select"):
        getattr(lib, name).restype = i32
    lib.als_static_last_error.argtypes = []
    lib.als_static_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


@dataclass
class Csr:
    """CSR matrix on the GPU: int64 indptr [rows+1], int32 indices [nnz], optional fp32 values."""
    rows: int
    cols: int
    indptr: torch.Tensor
    indices: torch.Tensor
    values: Optional[torch.Tensor] = None

    @property
    def nnz(self) -> int:
        return int(self.indices.numel())

    def c(self) -> c_als_csr:
        indptr, indices, values = self.indptr, self.indices, self.values
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
    ld, unit = t.stride()
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
