"""Thin Python binding of ``libef21.so`` (see ``include/ef21.h``): argument marshalling only.

PyTorch supplies device memory (``tensor.data_ptr()``) and the stream; every step of the EF21
hot path runs inside the library's HIP kernels.  There is no fallback: a missing library or a
failing call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libef21.so")

EF21_OK, EF21_EINVAL, EF21_ENOMEM, EF21_EHIP, EF21_ESTATE = 0, -1, -2, -3, -4
ORDER_GRAD_FIRST, ORDER_STEP_FIRST, PLUS, CLASSIC_EF, ONE_LAUNCH = 0, 1, 2, 4, 8
LOSS_LOGISTIC, LOSS_LEAST_SQUARES = 0, 1

# every symbol include/ef21.h declares
SYMBOLS = (
    "ef21_last_error", "ef21_create", "ef21_destroy", "ef21_set_stream", "ef21_topk",
    "ef21_set_problem_dense", "ef21_set_problem_csr", "ef21_set_state", "ef21_get_state",
    "ef21_get_messages", "ef21_local_grad", "ef21_step", "ef21_set_timing", "ef21_get_timing", "ef21_kernel_name",
    "ef21_hbm_read", "ef21_hbm_copy", "ef21_get_choices", "ef21_set_loss", "ef21_set_minibatch", "ef21_theory_stepsize",
    "ef21_topk_static", "ef21_embed", "ef21_embed_grad_workspace", "ef21_embed_grad", "ef21_token_logps", "ef21_token_logps_grad",
    "ef21_preference_loss_workspace", "ef21_preference_loss", "ef21_policy_loss_workspace", "ef21_policy_loss",
)
K_COUNT = 11
VALUE_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # EF21_F32, EF21_BF16, EF21_F16
TOKEN_TYPES = {torch.int32: 0, torch.int64: 1}                          # EF21_I32, EF21_I64


class EF21Error(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libef21 error {code}: {text}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Open libef21.so (built in-tree by paper_2106_05203_amd/build.py) and declare prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2106_05203_amd.build` "
            "(there is no non-HIP fallback)")
    lib = C.CDLL(LIB_PATH)
    p, i32, i64, f32, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint32
    lib.ef21_last_error.argtypes = []
    lib.ef21_last_error.restype = C.c_char_p
    lib.ef21_create.argtypes = [i32, i64, i64, f32]
    lib.ef21_create.restype = p
    lib.ef21_destroy.argtypes = [p]
    lib.ef21_set_stream.argtypes = [p, p]
    lib.ef21_topk.argtypes = [p, i32, i64, i64, p, p, p]
    lib.ef21_topk_static.argtypes = [p, i32, i64, i64, p, p, p]
    lib.ef21_set_problem_dense.argtypes = [p, p, p, i64, f32]
    lib.ef21_set_problem_csr.argtypes = [p, p, p, p, p, i64, f32]
    lib.ef21_set_state.argtypes = [p, p, p, p]
    lib.ef21_get_state.argtypes = [p, p, p, p]
    lib.ef21_get_messages.argtypes = [p, p, p]
    lib.ef21_local_grad.argtypes = [p, p, p]
    lib.ef21_step.argtypes = [p, p, u32]
    lib.ef21_set_timing.argtypes = [p, C.c_int]
    lib.ef21_get_timing.argtypes = [p, p, p, C.c_int]
    lib.ef21_kernel_name.argtypes = [C.c_int]
    lib.ef21_get_choices.argtypes = [p, p, p]
    lib.ef21_set_loss.argtypes = [p, C.c_int]
    lib.ef21_set_minibatch.argtypes = [p, p, C.c_int64]
    lib.ef21_theory_stepsize.argtypes = [p, C.c_int32, p, p, p]
    lib.ef21_hbm_read.argtypes = [p, C.c_int64, p, p]
    lib.ef21_hbm_copy.argtypes = [p, p, C.c_int64, p]
    lib.ef21_embed.argtypes = [p, C.c_int, i64, i64, i64, p, C.c_int, i64, f32, p, C.c_int, i64, p]
    lib.ef21_embed_grad_workspace.argtypes = [i32, i64, i64, i64, p]
    lib.ef21_embed_grad.argtypes = [p, C.c_int, i64, p, C.c_int, i32, i64, i64, i64, f32, p, i64, C.c_int, p, i64, p]
    logits = [p, C.c_int, i64, i64, i64, p, C.c_int]
    lib.ef21_token_logps.argtypes = [*logits, p, p, p]
    lib.ef21_token_logps_grad.argtypes = [*logits, p, p, p, i64, p]
    lib.ef21_preference_loss_workspace.argtypes = [i64, i32, p]
    lib.ef21_preference_loss.argtypes = [*logits, p, i32, p, f32, f32, C.c_int, C.c_int, p, p, p, p, i64, p, i64, p]
    lib.ef21_policy_loss_workspace.argtypes = [i64, p]
    lib.ef21_policy_loss.argtypes = [*logits, p, p, p, p, f32, f32, f32, p, p, p, p, i64, p, i64, p]
    for name in SYMBOLS[2:]:
        getattr(lib, name).restype = C.c_int
    lib.ef21_kernel_name.restype = C.c_char_p
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != EF21_OK:
        raise EF21Error(rc, load_library().ef21_last_error().decode())


def _dev(t: torch.Tensor, dtype: torch.dtype, shape=None) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a tensor in GPU memory")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"expected a contiguous {dtype} tensor, got {t.dtype} (contiguous={t.is_contiguous()})")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _opt(t, dtype, shape=None):
    return None if t is None else _dev(t, dtype, shape)


# torch.cuda.current_stream() builds a Stream object (2.8 us); the handle alone takes 0.3.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _current_stream_ptr() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def ef21_topk(rows: torch.Tensor, k: int, out_idx: torch.Tensor | None = None,
              out_val: torch.Tensor | None = None, static: bool = False):
    """Batched Top-k (ef21_topk, or ef21_topk_static if `static`) of rows [n][d] on torch's current stream.
    Returns (idx [n][k] int32 ascending, val [n][k] float32)."""
    lib = load_library()
    if rows.dim() != 2:
        raise ValueError("rows must be [n][d]")
    n, d = rows.shape
    if out_idx is None:
        out_idx = torch.empty(n, max(k, 0), dtype=torch.int32, device=rows.device)
    if out_val is None:
        out_val = torch.empty(n, max(k, 0), dtype=torch.float32, device=rows.device)
    call = lib.ef21_topk_static if static else lib.ef21_topk
    _check(call(_dev(rows, torch.float32), n, d, k, _dev(out_idx, torch.int32), _dev(out_val, torch.float32),
                _current_stream_ptr()))
    return out_idx, out_val


def ef21_hbm_read(src: torch.Tensor, sink: torch.Tensor) -> None:
    """One plain read of `src` (ef21_hbm_read) on torch's current stream; measurement only."""
    lib = load_library()
    _check(lib.ef21_hbm_read(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(), _current_stream_ptr()))


def ef21_hbm_copy(dst: torch.Tensor, src: torch.Tensor) -> None:
    """dst <- src by a plain copy kernel (ef21_hbm_copy) on torch's current stream; measurement only."""
    lib = load_library()
    if dst.numel() * dst.element_size() != src.numel() * src.element_size():
        raise ValueError("dst and src must have the same size in bytes")
    _check(lib.ef21_hbm_copy(dst.data_ptr(), src.data_ptr(), src.numel() * src.element_size(), _current_stream_ptr()))


# -- the two ends of a language model (stateless, on torch's current stream; see include/ef21.h)
# A call on a few tokens takes as long as its checks here, so they touch every tensor few times.
_F32 = torch.float32
_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _gpu(t, what: str) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a tensor in GPU memory")


def _matrix(t: torch.Tensor, what: str):
    """(address, type, rows, width, stride) of a matrix whose rows are contiguous."""
    _gpu(t, what)
    kind = VALUE_TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{what}: unsupported type {t.dtype}")
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{what}: expected two dimensions, got {tuple(shape)}")
    rows, width = shape
    step, unit = t.stride()
    if unit != 1 and width > 1 and rows > 0:
        raise TypeError(f"{what}: rows must be contiguous")
    return t.data_ptr(), kind, rows, width, step if rows > 1 else width


def _token_list(t: torch.Tensor, what: str):
    """(address, type) of contiguous tokens or labels."""
    _gpu(t, what)
    kind = TOKEN_TYPES.get(t.dtype)
    if kind is None or not t.is_contiguous():
        raise TypeError(f"{what}: expected contiguous int32 or int64, got {t.dtype} (contiguous={t.is_contiguous()})")
    return t.data_ptr(), kind


def _vector(t, length: int, what: str, dtype=_F32) -> int:
    """Address of a contiguous vector."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == (length,) and t.is_contiguous():
        return t.data_ptr()
    _gpu(t, what)
    if t.dtype is not dtype or not t.is_contiguous():
        raise TypeError(f"{what}: expected contiguous {dtype}, got {t.dtype} (contiguous={t.is_contiguous()})")
    raise ValueError(f"{what}: expected shape ({length},), got {tuple(t.shape)}")


def _optional(t, length: int, what: str):
    return None if t is None else _vector(t, length, what)


def _stream_of(*tensors) -> int:
    """The current stream of the device that all tensors are on, which must be the current one."""
    device = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on one device")
    if _raw_device() != device:
        raise ValueError(f"the tensors are on device {device}, which is not the current one")
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _size(call, *sizes) -> int:
    size = C.c_int64()
    _check(call(*sizes, C.byref(size)))
    return size.value


def ef21_embed(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: torch.Tensor | None = None,
               dtype: torch.dtype | None = None) -> torch.Tensor:
    """scale * table[tokens] (ef21_embed): table [vocab][width], tokens of any shape (contiguous); out [..., width] of the
    table's type, of `dtype`, or as given."""
    lib = load_library()
    at, kind, vocab, width, stride = _matrix(table, "table")
    ids, id_type = _token_list(tokens, "tokens")
    if out is None:
        out = torch.empty(*tokens.shape, width, dtype=dtype or table.dtype, device=table.device)
    to, out_type, rows, cols, out_stride = _matrix(out if out.dim() == 2 else out.view(-1, width), "out")
    if cols != width or rows != tokens.numel():
        raise ValueError(f"out must have {tokens.numel()} rows of {width} entries")
    _check(lib.ef21_embed(at, kind, vocab, width, stride, ids, id_type, rows, scale, to, out_type, out_stride, _stream_of(table, tokens, out)))
    return out


@functools.lru_cache(maxsize=256)
def ef21_embed_grad_workspace(n: int, count: int, vocab: int, width: int) -> int:
    """Bytes of workspace that ef21_embed_grad needs."""
    return _size(load_library().ef21_embed_grad_workspace, n, count, vocab, width)


def ef21_embed_grad(grad_out: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0, out: torch.Tensor | None = None,
                    accumulate: bool = False, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Gradients of the table (ef21_embed_grad): grad_out [n][count][width], tokens [n][count]; returns fp32 [n][vocab][width]
    (`out`, whose workers may lie further apart, for example a block of columns of the rows that EF21.step takes)."""
    lib = load_library()
    _gpu(grad_out, "grad_out")
    shape = grad_out.shape
    if len(shape) != 3 or tokens.shape != shape[:2]:
        raise ValueError("grad_out must be [n][count][width] and tokens [n][count]")
    n, count, width = shape
    kind = VALUE_TYPES.get(grad_out.dtype)
    if kind is None:
        raise TypeError(f"grad_out: unsupported type {grad_out.dtype}")
    ids, id_type = _token_list(tokens, "tokens")
    # the workers' rows as one matrix
    across, down, unit = grad_out.stride()
    stride = down if count > 1 else across if n > 1 else width
    if n * count == 0:
        stride = width
    elif (unit != 1 and width > 1) or (n > 1 and across != count * stride):
        raise TypeError("grad_out: entries of a row must be contiguous and the workers' rows follow one another at one stride")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the gradient to add to")
        out = torch.empty(n, vocab, width, dtype=_F32, device=grad_out.device)
    if out.dtype is not _F32 or not out.is_cuda or out.shape != (n, vocab, width):
        raise TypeError(f"out must be float32 [{n}][{vocab}][{width}] in GPU memory")
    apart, row, one = out.stride()
    if (row != width and vocab > 1) or (one != 1 and width > 1):
        raise TypeError("out: each worker's table must be contiguous")
    if workspace is None:
        workspace = torch.empty(ef21_embed_grad_workspace(n, count, vocab, width), dtype=torch.uint8, device=grad_out.device)
    _check(lib.ef21_embed_grad(grad_out.data_ptr(), kind, stride, ids, id_type, n, count, vocab, width, scale, out.data_ptr(), apart, int(accumulate),
                               workspace.data_ptr(), workspace.nbytes, _stream_of(grad_out, tokens, out, workspace)))
    return out


def _logit_rows(logits, labels):
    at, kind, rows, vocab, stride = _matrix(logits, "logits")
    ids, id_type = _token_list(labels, "labels")
    if labels.shape != (rows,):
        raise ValueError(f"labels must be [{rows}]")
    return (at, kind, rows, vocab, stride, ids, id_type), rows


def _logit_grad(grad, logits):
    """(tensor or None, address, stride) of the gradient: `grad` is a tensor to write, True for a new one, False or None for none."""
    if grad is None or grad is False:
        return None, None, 0
    if grad is True:
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    at, _, _, _, stride = _matrix(grad, "grad")
    if grad.dtype is not logits.dtype or grad.shape != logits.shape:
        raise ValueError("grad must have the logits' type and shape")
    return grad, at, stride


def _new(t, length: int, like):
    return torch.empty(length, dtype=_F32, device=like.device) if t is None else t


def ef21_token_logps(logits: torch.Tensor, labels: torch.Tensor, logp: torch.Tensor | None = None, lse: torch.Tensor | None = None):
    """(logp [rows], lse [rows]) of the labels under the softmax of each row of logits [rows][vocab] (ef21_token_logps)."""
    lib = load_library()
    args, rows = _logit_rows(logits, labels)
    logp, lse = _new(logp, rows, logits), _new(lse, rows, logits)
    _check(lib.ef21_token_logps(*args, _vector(logp, rows, "logp"), _vector(lse, rows, "lse"), _stream_of(logits, labels, logp, lse)))
    return logp, lse


def ef21_token_logps_grad(logits: torch.Tensor, labels: torch.Tensor, lse: torch.Tensor, grad_logp: torch.Tensor,
                          out: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient of the logits from that of the log-probabilities (ef21_token_logps_grad); `out` may be the logits."""
    lib = load_library()
    args, rows = _logit_rows(logits, labels)
    out, to, stride = _logit_grad(True if out is None else out, logits)
    _check(lib.ef21_token_logps_grad(*args, _vector(lse, rows, "lse"), _vector(grad_logp, rows, "grad_logp"), to, stride,
                                     _stream_of(logits, labels, lse, grad_logp, out)))
    return out


@functools.lru_cache(maxsize=256)
def ef21_preference_loss_workspace(rows: int, pairs: int) -> int:
    """Bytes of workspace that ef21_preference_loss needs."""
    return _size(load_library().ef21_preference_loss_workspace, rows, pairs)


def ef21_preference_loss(logits: torch.Tensor, labels: torch.Tensor, seq_start: torch.Tensor, ref_logp: torch.Tensor, beta: float,
                         smoothing: float = 0.0, loss: int = LOSS_LOGISTIC, mean: bool = False, pair_weight: torch.Tensor | None = None,
                         out_loss: torch.Tensor | None = None, logp: torch.Tensor | None = None, grad: "torch.Tensor | bool | None" = True,
                         workspace: torch.Tensor | None = None):
    """(loss [pairs], logp [rows], grad [rows][vocab] or None) of ef21_preference_loss; seq_start int64 [2 pairs + 1] on the
    device.  grad: a tensor to write (the logits themselves if they are not needed again), True for a new one, False for none."""
    lib = load_library()
    args, rows = _logit_rows(logits, labels)
    pairs = (seq_start.numel() - 1) // 2
    if pairs < 1:
        raise ValueError("seq_start must be [2 pairs + 1]")
    starts = _vector(seq_start, 2 * pairs + 1, "seq_start", torch.int64)
    out_loss, logp = _new(out_loss, pairs, logits), _new(logp, rows, logits)
    grad, to, stride = _logit_grad(grad, logits)
    if workspace is None:
        workspace = torch.empty(ef21_preference_loss_workspace(rows, pairs), dtype=torch.uint8, device=logits.device)
    _check(lib.ef21_preference_loss(*args, starts, pairs, _vector(ref_logp, rows, "ref_logp"), beta, smoothing, int(loss), int(mean),
                                    _optional(pair_weight, pairs, "pair_weight"), _vector(out_loss, pairs, "out_loss"), _vector(logp, rows, "logp"), to,
                                    stride, workspace.data_ptr(), workspace.nbytes,
                                    _stream_of(logits, labels, seq_start, ref_logp, pair_weight, out_loss, logp, grad, workspace)))
    return out_loss, logp, grad


@functools.lru_cache(maxsize=256)
def ef21_policy_loss_workspace(rows: int) -> int:
    """Bytes of workspace that ef21_policy_loss needs."""
    return _size(load_library().ef21_policy_loss_workspace, rows)


def ef21_policy_loss(logits: torch.Tensor, labels: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, clip_low: float,
                     clip_high: float, ref_logp: torch.Tensor | None = None, kl: float = 0.0, weight: torch.Tensor | None = None,
                     out_loss: torch.Tensor | None = None, token_loss: torch.Tensor | None = None, logp: torch.Tensor | None = None,
                     grad: "torch.Tensor | bool | None" = True, workspace: torch.Tensor | None = None):
    """(loss [1], token_loss [rows], logp [rows], grad [rows][vocab] or None) of ef21_policy_loss; grad as in
    ef21_preference_loss."""
    lib = load_library()
    args, rows = _logit_rows(logits, labels)
    out_loss, token_loss, logp = _new(out_loss, 1, logits), _new(token_loss, rows, logits), _new(logp, rows, logits)
    grad, to, stride = _logit_grad(grad, logits)
    if workspace is None:
        workspace = torch.empty(ef21_policy_loss_workspace(rows), dtype=torch.uint8, device=logits.device)
    _check(lib.ef21_policy_loss(*args, _vector(old_logp, rows, "old_logp"), _vector(advantages, rows, "advantages"),
                                _optional(ref_logp, rows, "ref_logp"), _optional(weight, rows, "weight"), clip_low, clip_high, kl,
                                _vector(out_loss, 1, "out_loss"), _vector(token_loss, rows, "token_loss"), _vector(logp, rows, "logp"), to, stride,
                                workspace.data_ptr(), workspace.nbytes,
                                _stream_of(logits, labels, old_logp, advantages, ref_logp, weight, out_loss, token_loss, logp, grad, workspace)))
    return out_loss, token_loss, logp, grad


class EF21:
    """Handle of the C library: state of Algorithm 2 for n workers batched on one GPU."""

    def __init__(self, n: int, d: int, k: int, gamma: float, device="cuda:0"):
        self._lib = load_library()
        self.n, self.d, self.k, self.gamma = int(n), int(d), int(k), float(gamma)
        self.device = torch.device(device)
        self._keep = []     # borrowed problem tensors stay alive with the handle
        self._batch = None  # and the rows of the minibatch
        with torch.cuda.device(self.device):
            self._h = self._lib.ef21_create(self.n, self.d, self.k, self.gamma)
        if not self._h:
            raise EF21Error(EF21_EINVAL, self._lib.ef21_last_error().decode())
        self.use_current_stream()

    # -- plumbing
    def _call(self, function, *args) -> None:
        """function(handle, *args) with the handle's device current; switching there and back costs as much as a small
        call's own host work, so it is left out where that device is the current one already."""
        if self.device.index is None or torch.cuda.current_device() == self.device.index:
            _check(function(self._h, *args))
            return
        with torch.cuda.device(self.device):
            _check(function(self._h, *args))

    def use_current_stream(self) -> None:
        with torch.cuda.device(self.device):
            _check(self._lib.ef21_set_stream(self._h, _current_stream_ptr()))

    def close(self) -> None:
        if getattr(self, "_h", None):
            with torch.cuda.device(self.device):
                _check(self._lib.ef21_destroy(self._h))
            self._h = None
            self._keep = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- problem
    def set_problem_dense(self, A: torch.Tensor, y: torch.Tensor, lam: float) -> None:
        n, m, d = A.shape
        if (n, d) != (self.n, self.d):
            raise ValueError("A must be [n][m][d]")
        self._call(self._lib.ef21_set_problem_dense, _dev(A, torch.float32), _dev(y, torch.float32, (n, m)), m,
                   float(lam))
        self._keep = [A, y]
        self._batch = None

    def set_problem_csr(self, rowptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor, y: torch.Tensor, m: int,
                        lam: float) -> None:
        if rowptr.numel() != self.n * m + 1 or col.numel() != val.numel():
            raise ValueError("rowptr must have n*m+1 entries and col, val equal lengths")
        self._call(self._lib.ef21_set_problem_csr, _dev(rowptr, torch.int64), _dev(col, torch.int32),
                   _dev(val, torch.float32), _dev(y, torch.float32, (self.n, m)), m,
                   float(lam))
        self._keep = [rowptr, col, val, y]
        self._batch = None

    # -- state
    def set_state(self, x=None, g_i=None, g=None) -> None:
        self._call(self._lib.ef21_set_state, _opt(x, torch.float32, (self.d,)),
                   _opt(g_i, torch.float32, (self.n, self.d)),
                   _opt(g, torch.float32, (self.d,)))

    def get_state(self):
        x = torch.empty(self.d, dtype=torch.float32, device=self.device)
        g_i = torch.empty((self.n, self.d), dtype=torch.float32, device=self.device)
        g = torch.empty(self.d, dtype=torch.float32, device=self.device)
        self._call(self._lib.ef21_get_state, x.data_ptr(), g_i.data_ptr(), g.data_ptr())
        return x, g_i, g

    def get_x(self) -> torch.Tensor:
        x = torch.empty(self.d, dtype=torch.float32, device=self.device)
        self._call(self._lib.ef21_get_state, x.data_ptr(), None, None)
        return x

    def get_messages(self):
        idx = torch.empty((self.n, self.k), dtype=torch.int32, device=self.device)
        val = torch.empty((self.n, self.k), dtype=torch.float32, device=self.device)
        self._call(self._lib.ef21_get_messages, idx.data_ptr(), val.data_ptr())
        return idx, val

    def set_loss(self, loss: int) -> None:
        self._call(self._lib.ef21_set_loss, int(loss))

    def set_minibatch(self, rows: "torch.Tensor | None") -> None:
        """rows: int32 [n][tau] on the device (kept alive by the handle and read at every gradient), or None
        for full gradients."""
        with torch.cuda.device(self.device):
            if rows is None:
                _check(self._lib.ef21_set_minibatch(self._h, None, 0))
                self._batch = None
                return
            assert rows.dtype == torch.int32 and rows.is_cuda and rows.is_contiguous() and rows.dim() == 2
            assert rows.shape[0] == self.n
            _check(self._lib.ef21_set_minibatch(self._h, rows.data_ptr(), int(rows.shape[1])))
            self._batch = rows

    def theory_stepsize(self, iterations: int = 200):
        """(gamma, L, L_i [n]) of Theorem 1 for the attached problem, eigenvalues by power iteration on the GPU."""
        gamma, L = C.c_double(), C.c_double()
        L_i = (C.c_double * self.n)()
        self._call(self._lib.ef21_theory_stepsize, int(iterations), C.byref(gamma), C.byref(L), L_i)
        return gamma.value, L.value, list(L_i)

    def get_choices(self):
        """(branch [n] int32: 1 = plain compressor chosen, distortions [n][2] float64: B_i, M_i) of the last
        step taken with PLUS."""
        branch = torch.empty(self.n, dtype=torch.int32, device=self.device)
        bm = torch.empty((self.n, 2), dtype=torch.float64, device=self.device)
        self._call(self._lib.ef21_get_choices, branch.data_ptr(), bm.data_ptr())
        return branch, bm

    # -- measurement
    def set_timing(self, enabled: bool) -> None:
        self._call(self._lib.ef21_set_timing, int(bool(enabled)))

    def get_timing(self, reset: bool = True) -> dict:
        """{kernel class: (milliseconds, launches)} accumulated while timing was enabled."""
        ms = (C.c_double * K_COUNT)()
        cnt = (C.c_int64 * K_COUNT)()
        self._call(self._lib.ef21_get_timing, C.addressof(ms), C.addressof(cnt), int(reset))
        return {self._lib.ef21_kernel_name(i).decode(): (ms[i], cnt[i]) for i in range(K_COUNT) if cnt[i]}

    # -- the hot path
    def local_grad(self, x: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        if out is None:
            out = torch.empty((self.n, self.d), dtype=torch.float32, device=self.device)
        self._call(self._lib.ef21_local_grad, _opt(x, torch.float32, (self.d,)),
                   _dev(out, torch.float32, (self.n, self.d)))
        return out

    def step(self, grads: torch.Tensor | None = None, order: int = ORDER_GRAD_FIRST) -> None:
        self._call(self._lib.ef21_step, _opt(grads, torch.float32, (self.n, self.d)), int(order))
