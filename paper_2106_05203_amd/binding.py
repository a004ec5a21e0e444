"""Thin Python binding of ``libef21.so`` (see ``include/ef21.h``): argument marshalling only.

PyTorch supplies device memory (``tensor.data_ptr()``) and the stream; every step of the EF21
hot path runs inside the library's HIP kernels.  There is no fallback: a missing library or a
failing call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import operator
import os
import struct
import threading
from typing import NamedTuple

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
    "ef21_token_stats_workspace", "ef21_token_stats", "ef21_token_stats_grad", "ef21_grad_norm_workspace", "ef21_grad_norm", "ef21_adamw",
    "ef21_adamw_counted",
)
K_COUNT = 11
VALUE_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # EF21_F32, EF21_BF16, EF21_F16
TOKEN_TYPES = {torch.int32: 0, torch.int64: 1}                          # EF21_I32, EF21_I64


STATE_BLOCK = 256                                                       # entries that share the scales of 8-bit states


class EF21Error(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libef21 error {code}: {text}")
        self.code = code


class AdamwTensor(C.Structure):
    """ef21_adamw_tensor"""
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("copy", C.c_void_p), ("count", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32),
                ("weight_decay", C.c_float)]


class AdamwOptions(C.Structure):
    """ef21_adamw_options"""
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64), ("lr_device", C.c_void_p),
                ("step_device", C.c_void_p), ("grad_scale", C.c_void_p), ("seed", C.c_uint64), ("stochastic", C.c_int32)]


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
    lib.ef21_token_stats_workspace.argtypes = [C.c_int, i64, i64, i32, p]
    lib.ef21_token_stats.argtypes = [*logits, i32, p, p, p, p, p, p, p, i64, p]
    lib.ef21_token_stats_grad.argtypes = [*logits, p, p, p, p, p, i64, C.c_int, p]
    lib.ef21_grad_norm_workspace.argtypes = [i32, p]
    lib.ef21_grad_norm.argtypes = [p, p, p, i32, f32, f32, p, p, p, i64, p]
    lib.ef21_adamw.argtypes = [p, i32, p, p]
    lib.ef21_adamw_counted.argtypes = [p, i32, p, p, p]
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


class TokenStats(NamedTuple):
    """What ef21_token_stats returns; None where it was not asked for."""
    logp: "torch.Tensor | None"          # [rows]
    lse: torch.Tensor                    # [rows]
    entropy: torch.Tensor                # [rows]
    top_tokens: "torch.Tensor | None"    # [rows][k] int32
    top_logp: "torch.Tensor | None"      # [rows][k]
    sums: "torch.Tensor | None"          # [rows][2], for ef21_token_stats_grad


@functools.lru_cache(maxsize=256)
def ef21_token_stats_workspace(kind: int, rows: int, vocab: int, k: int) -> int:
    """Bytes of workspace that ef21_token_stats needs for logits of type `kind` (VALUE_TYPES)."""
    return _size(load_library().ef21_token_stats_workspace, kind, rows, vocab, k)


def _maybe_labelled(logits, labels):
    if labels is not None:
        return _logit_rows(logits, labels)
    at, kind, rows, vocab, stride = _matrix(logits, "logits")
    return (at, kind, rows, vocab, stride, None, 0), rows


def _shaped(t, shape, dtype, like, what: str):
    """t, or a new tensor; contiguous and of that shape and type."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    _gpu(t, what)
    if t.dtype is not dtype or not t.is_contiguous():
        raise TypeError(f"{what}: expected contiguous {dtype}, got {t.dtype} (contiguous={t.is_contiguous()})")
    if t.shape != shape:
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def ef21_token_stats(logits: torch.Tensor, labels: torch.Tensor | None = None, k: int = 0, logp: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None, entropy: torch.Tensor | None = None, top_tokens: torch.Tensor | None = None,
                     top_logp: torch.Tensor | None = None, sums: "torch.Tensor | bool | None" = None,
                     workspace: torch.Tensor | None = None) -> TokenStats:
    """Log-probabilities of the labels (if any), lse, entropy and the k most likely tokens of each row of logits [rows][vocab]
    (ef21_token_stats).  sums: what ef21_token_stats_grad needs: a tensor to write, True for a new one, False or None for none."""
    lib = load_library()
    args, rows = _maybe_labelled(logits, labels)
    if labels is not None:
        logp = _new(logp, rows, logits)
    elif logp is not None:
        raise ValueError("logp needs labels")
    lse, entropy = _new(lse, rows, logits), _new(entropy, rows, logits)
    if k > 0:
        top_tokens, top_logp = _shaped(top_tokens, (rows, k), torch.int32, logits, "top_tokens"), _shaped(top_logp, (rows, k), _F32, logits, "top_logp")
    elif top_tokens is not None or top_logp is not None:
        raise ValueError("top_tokens and top_logp need k > 0")
    sums = None if sums is None or sums is False else _shaped(None if sums is True else sums, (rows, 2), _F32, logits, "sums")
    need = ef21_token_stats_workspace(args[1], rows, args[3], k)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=logits.device)
    _check(lib.ef21_token_stats(*args, k, _optional(logp, rows, "logp"), _vector(lse, rows, "lse"), _vector(entropy, rows, "entropy"),
                                top_tokens.data_ptr() if k > 0 else None, top_logp.data_ptr() if k > 0 else None,
                                None if sums is None else sums.data_ptr(), None if workspace is None else workspace.data_ptr(),
                                0 if workspace is None else workspace.nbytes,
                                _stream_of(logits, labels, logp, lse, entropy, top_tokens, top_logp, sums, workspace)))
    return TokenStats(logp, lse, entropy, top_tokens, top_logp, sums)


def ef21_token_stats_grad(logits: torch.Tensor, labels: torch.Tensor | None, sums: torch.Tensor, entropy: torch.Tensor,
                          grad_logp: torch.Tensor | None = None, grad_entropy: torch.Tensor | None = None, out: torch.Tensor | None = None,
                          accumulate: bool = False) -> torch.Tensor:
    """The gradient of the logits from those of the log-probabilities and entropies (ef21_token_stats_grad).  `out` may be the logits;
    with accumulate it is a gradient of them that is added to."""
    lib = load_library()
    args, rows = _maybe_labelled(logits, labels)
    if accumulate and (out is None or out is True):
        raise ValueError("accumulate needs the gradient to add to")
    out, to, stride = _logit_grad(True if out is None else out, logits)
    _shaped(sums, (rows, 2), _F32, logits, "sums")
    _check(lib.ef21_token_stats_grad(*args, sums.data_ptr(), _vector(entropy, rows, "entropy"), _optional(grad_logp, rows, "grad_logp"),
                                     _optional(grad_entropy, rows, "grad_entropy"), to, stride, int(accumulate),
                                     _stream_of(logits, labels, sums, entropy, grad_logp, grad_entropy, out)))
    return out


# -- the step of a model's parameters
class TensorList:
    """Tensors that are looked at once and used in many calls: contiguous, fp32, bf16 or fp16, on one device.  What is used is the memory that they
    have then, also if their .data is another's later on."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.device = _one_device(self.tensors, "tensors")
        _all_dense(self.tensors, VALUE_TYPES, "tensors")
        n = len(self.tensors)
        self._held = [t.untyped_storage() for t in self.tensors]
        self._spaces, self._lock = {}, threading.Lock()                  # by stream: calls on two of them may overlap; and one thread's at a time
        self.addresses = (C.c_void_p * n)(*[t.data_ptr() for t in self.tensors])
        self.types = (C.c_int32 * n)(*[VALUE_TYPES[t.dtype] for t in self.tensors])
        self.counts = (C.c_int64 * n)(*[t.numel() for t in self.tensors])

    def __len__(self):
        return len(self.tensors)

    def workspace(self, stream: int, bytes_of: int) -> torch.Tensor:
        """A workspace for ef21_grad_norm on a stream.  A captured call has one of its own."""
        space = self._spaces.get(stream)
        if space is None or torch.cuda.is_current_stream_capturing():
            space = torch.empty(bytes_of, dtype=torch.uint8, device=self.tensors[0].device)
            if not torch.cuda.is_current_stream_capturing():
                self._spaces[stream] = space
        return space


def _dense(t, types, what: str, i: int) -> None:
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in types and t.is_contiguous():
        return
    what = f"{what}[{i}]"
    _gpu(t, what)
    if t.dtype not in types or not t.is_contiguous():
        raise TypeError(f"{what}: expected contiguous {' or '.join(str(d) for d in types)}, got {t.dtype} (contiguous={t.is_contiguous()})")


def _spans(starts: list, stops: list):
    """Without those of no length."""
    if all(map(operator.lt, starts, stops)):
        return starts, stops
    some = [(start, stop) for start, stop in zip(starts, stops) if start < stop]
    return [start for start, _ in some], [stop for _, stop in some]


def _are_tensors(things) -> bool:
    return all([issubclass(kind, torch.Tensor) for kind in set(map(type, things))])


def _all_dense(tensors, types, what: str) -> None:
    """_dense of all of a list, in a few passes over it: a tenth of the time of a call for each."""
    if not (_are_tensors(tensors) and {t.dtype for t in tensors}.issubset(types) and {t.is_cuda for t in tensors} == {True}
            and all([t.is_contiguous() for t in tensors])):
        for i, t in enumerate(tensors):
            _dense(t, types, what, i)


def _one_device(tensors, what: str) -> int:
    if not tensors:
        raise ValueError(f"{what}: none given")
    devices = {t.get_device() for t in tensors} if _are_tensors(tensors) else {-1}
    if min(devices) < 0:
        raise TypeError(f"{what}: expected tensors in GPU memory")
    device = devices.pop()
    if devices:
        raise ValueError(f"{what}: all tensors must be on one device")
    return device


@functools.lru_cache(maxsize=256)
def ef21_grad_norm_workspace(tensor_count: int) -> int:
    """Bytes of workspace that ef21_grad_norm needs."""
    return _size(load_library().ef21_grad_norm_workspace, tensor_count)


def ef21_grad_norm(grads, max_norm: float = math.inf, scale: float = 1.0, norm: torch.Tensor | None = None, factor: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None):
    """(norm [1], factor [1]) of all gradients together (ef21_grad_norm); grads: a TensorList, or tensors.  `factor` is what AdamW.step
    takes as grad_scale.  Calls that share a workspace follow each other."""
    lib = load_library()
    grads = grads if isinstance(grads, TensorList) else TensorList(grads)
    like = grads.tensors[0]
    norm, factor = _new(norm, 1, like), _new(factor, 1, like)
    stream = _stream_of(like, norm, factor, workspace)
    args = grads.addresses, grads.types, grads.counts, len(grads), scale, max_norm, _vector(norm, 1, "norm"), _vector(factor, 1, "factor")
    with grads._lock:
        if workspace is None:
            workspace = grads.workspace(stream, ef21_grad_norm_workspace(len(grads)))
        _check(lib.ef21_grad_norm(*args, workspace.data_ptr(), workspace.nbytes, stream))
    return norm, factor


class AdamW:
    """AdamW (ef21_adamw) over many tensors, with the states of each.

    params, grads: contiguous tensors (grads may also be given to every step); a gradient of another type than its parameter is fine.
    bits: 32 or 8 for the states, or a list of one or the other per tensor.  m, v, m_scale, v_scale: states to go on with (fp32, or
    float8_e4m3fn with one fp32 scale per 256 entries), each a list per tensor; new ones otherwise, also for None in a list.
    copies: a list of bf16 or fp16 tensors (or None) that receive the new fp32 parameters.  weight_decay: a number, or one per tensor.
    stochastic, seed: see include/ef21.h.  steps: the number of the last step that was taken, which may be set.  The tensors stay the caller's; the object keeps them alive and works on the memory
    that they have when they are given, also if their .data is another's later on.  Steps of one object follow each other: in one thread,
    and on one stream or on streams that wait for each other.
    """

    def __init__(self, params, grads=None, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, bits=32, m=None, v=None, m_scale=None,
                 v_scale=None, copies=None, stochastic: bool = False, seed: int = 0):
        self._lib = load_library()
        self.params = list(params)
        n = len(self.params)
        self.device = _one_device(self.params, "params")
        per = self._per_tensor
        bits, decay = per(bits, n, "bits"), per(weight_decay, n, "weight_decay")
        self.copies = per(copies, n, "copies")
        self.m, self.v, self.m_scale, self.v_scale = per(m, n, "m"), per(v, n, "v"), per(m_scale, n, "m_scale"), per(v_scale, n, "v_scale")
        _all_dense(self.params, VALUE_TYPES, "params")
        if not all([b == 32 or b == 8 for b in bits]):
            raise ValueError("bits must be 8 or 32")
        self._shapes, counts = [p.shape for p in self.params], [p.numel() for p in self.params]
        eight = [i for i, b in enumerate(bits) if b == 8]
        kinds = [torch.float8_e4m3fn if b == 8 else _F32 for b in bits]
        sizes = [count if b == 8 else 4 * count for count, b in zip(counts, bits)]
        blocks = [-(-counts[i] // STATE_BLOCK) for i in eight]
        at_params = [p.data_ptr() for p in self.params]
        starts, ends = list(at_params), [at + count * p.itemsize for at, count, p in zip(at_params, counts, self.params)]
        columns = [at_params, [0] * n]
        for states in (self.m, self.v):
            states[:] = self._states(states, kinds, self._shapes, "states", range(n))
            columns.append([t.data_ptr() for t in states])
            starts += columns[-1]
            ends += [at + size for at, size in zip(columns[-1], sizes)]
        for scales in (self.m_scale, self.v_scale):
            column = [0] * n
            if len(eight) < n:
                for i, (b, t) in enumerate(zip(bits, scales)):
                    if b == 32 and t is not None:
                        raise ValueError(f"scales[{i}]: 32-bit states have none")
            if eight:
                given = self._states([scales[i] for i in eight], [_F32] * len(eight), [torch.Size((b,)) for b in blocks], "scales", eight)
                for i, t, at, block in zip(eight, given, [t.data_ptr() for t in given], blocks):
                    scales[i], column[i] = t, at
                    starts.append(at)
                    ends.append(at + 4 * block)
            columns.append(column)
        column, types = [0] * n, [0] * n
        for i, copy in enumerate(self.copies):
            if copy is None:
                continue
            _dense(copy, (torch.bfloat16, torch.float16), "copies", i)
            if self.params[i].dtype is not _F32:
                raise TypeError(f"copies[{i}]: copies are of fp32 parameters")
            if copy.shape != self._shapes[i]:
                raise ValueError(f"copies[{i}]: expected shape {tuple(self._shapes[i])}, got {tuple(copy.shape)}")
            column[i], types[i] = copy.data_ptr(), VALUE_TYPES[copy.dtype]
            starts.append(column[i])
            ends.append(column[i] + 2 * counts[i])
        self._columns = [*columns, column, counts, [VALUE_TYPES[p.dtype] for p in self.params], [0] * n, types, [float(x) for x in decay]]
        written = [t for group in (self.params, self.m, self.v, self.m_scale, self.v_scale, self.copies) for t in group if t is not None]
        _one_device(written, "params, states and copies")
        self._held = [t.untyped_storage() for t in written]
        self._written = _spans(starts, ends)
        self.grads = None
        if grads is not None:
            self.grads = self._take(grads)
        else:
            self._check_apart(([], []))
        self._options = AdamwOptions(0.0, float(betas[0]), float(betas[1]), float(eps), 1, None, None, None, int(seed) & (2 ** 64 - 1), int(bool(stochastic)))
        # The number of the last step: the host's, or counted on the device once a step might be skipped there (`_counted`: what the counter is
        # known to hold); None if a tensor of the caller's has it.
        self._steps, self._counting, self._counted = 0, False, 0
        self._counter = torch.zeros(2, dtype=torch.int64, device=self.params[0].device)

    @property
    def steps(self) -> "int | None":
        """The number of the last step that was taken (waits for the device where it is counted there); None where the caller's tensor has it."""
        return int(self._counter[0]) if self._counting else self._steps

    @steps.setter
    def steps(self, number: int) -> None:
        if number < 0:
            raise ValueError("steps must not be negative")
        self._counter[:1].fill_(number)
        self._steps = self._counted = number

    def _count(self) -> None:
        """From here on the device counts."""
        if self._counting or self._counted == self._steps:
            return
        if torch.cuda.is_current_stream_capturing():
            raise ValueError("a captured step=None goes on from a number on the device: set `steps` before the capture, or give a tensor")
        self._counter[:1].fill_(self._steps)
        self._counted = self._steps

    _ROW = struct.Struct("7Qq3if")                                       # AdamwTensor
    _GRAD, _GRAD_TYPE = 1, 9                                             # its columns of gradients

    @staticmethod
    def _per_tensor(x, n: int, what: str) -> list:
        if not isinstance(x, (list, tuple)):
            return [x] * n
        if len(x) != n:
            raise ValueError(f"{what}: expected {n}, got {len(x)}")
        return list(x)

    def _states(self, given: list, kinds: list, shapes: list, what: str, numbers) -> list:
        """The states or scales of the tensors `numbers`: those given, and new ones in the place of None."""
        if not (_are_tensors(given) and [t.dtype for t in given] == kinds and [t.shape for t in given] == shapes
                and {t.is_cuda for t in given} == {True} and all([t.is_contiguous() for t in given])):
            given = [self._state(t, kind, shape, self.params[i], what, i) for t, kind, shape, i in zip(given, kinds, shapes, numbers)]
        return given

    @staticmethod
    def _state(t, kind, shape, like, what: str, i: int):
        if t is None:
            return torch.zeros(shape, dtype=torch.uint8 if kind.itemsize == 1 else kind, device=like.device).view(kind)
        _dense(t, (kind,), what, i)
        if t.shape != shape:
            raise ValueError(f"{what}[{i}]: expected shape {tuple(shape)}, got {tuple(t.shape)}")
        return t

    def _check_apart(self, grads) -> None:
        """What is written overlaps nothing; grads: their starts and stops, which may overlap one another."""
        # spans are apart where, in order, each ends before the next begins
        starts, stops = sorted(self._written[0] + grads[0]), sorted(self._written[1] + grads[1])
        if all(map(operator.le, stops, starts[1:])):
            return
        end = end_written = 0                                            # of all before, and of the written ones
        for start, stop, written in sorted([(*span, True) for span in zip(*self._written)] + [(*span, False) for span in zip(*grads)]):
            if start < (end if written else end_written):
                raise ValueError("parameters, states, copies and gradients must not overlap")
            end = max(end, stop)
            if written:
                end_written = max(end_written, stop)

    def _take(self, grads) -> list:
        """Takes the addresses of gradients."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError(f"grads: expected {len(self.params)}, got {len(grads)}")
        _all_dense(grads, VALUE_TYPES, "grads")
        shapes = [g.shape for g in grads]
        if shapes != self._shapes:
            i = [a == b for a, b in zip(shapes, self._shapes)].index(False)
            raise ValueError(f"grads[{i}]: expected shape {tuple(self._shapes[i])}, got {tuple(shapes[i])}")
        if _one_device(grads, "grads") != self.device:
            raise ValueError("grads: not on the parameters' device")
        at = [g.data_ptr() for g in grads]
        self._check_apart(_spans(at, [start + g.nbytes for start, g in zip(at, grads)]))
        self._columns[self._GRAD], self._columns[self._GRAD_TYPE] = at, [VALUE_TYPES[g.dtype] for g in grads]
        self._table = (AdamwTensor * len(grads)).from_buffer_copy(b"".join([self._ROW.pack(*row) for row in zip(*self._columns)]))
        self._held_grads = [g.untyped_storage() for g in grads]
        return grads

    def step(self, lr, step: "int | torch.Tensor | None" = None, grad_scale: torch.Tensor | None = None, grads=None) -> None:
        """One step.  lr: a number, or an fp32 tensor [1] on the device; grad_scale: fp32 [1] on the device, such as ef21_grad_norm's factor (where it
        is not finite the step is skipped: nothing is changed); grads: gradients for this step and the following ones.
        step: its number from 1 on, an int64 tensor [1] on the device, or None for the one after the last that was taken: with grad_scale, or captured,
        the device counts (at each replay), and a skipped step does not count.  A number that is given does, and after a tensor's one has to be given."""
        if grads is not None:
            self.grads = self._take(grads)
        if self.grads is None:
            raise ValueError("no gradients given")
        o, on_device = self._options, isinstance(lr, torch.Tensor)
        o.lr, o.lr_device = (0.0, _vector(lr, 1, "lr")) if on_device else (lr, None)
        o.grad_scale = _optional(grad_scale, 1, "grad_scale")
        stepped = isinstance(step, torch.Tensor)
        if stepped:
            o.step, o.step_device = 1, _vector(step, 1, "step", torch.int64)
        elif step is None and self._steps is None:
            raise ValueError("the last step's number was on the device: give this one's")
        else:
            o.step, o.step_device = (1 if self._counting else self._steps + 1) if step is None else step, None
        stream = _stream_of(self.params[0], lr if on_device else None, step if stepped else None, grad_scale)
        if step is None and (self._counting or grad_scale is not None or torch.cuda.is_current_stream_capturing()):
            self._count()
            _check(self._lib.ef21_adamw_counted(self._table, len(self.params), C.byref(o), self._counter.data_ptr(), stream))
            self._counting = True
            return
        _check(self._lib.ef21_adamw(self._table, len(self.params), C.byref(o), stream))
        if stepped:
            self._steps, self._counting, self._counted = None, False, None
        elif self._counting:
            self._counter[:1].fill_(o.step)
        else:
            self._steps = o.step


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

    def get_g(self, out: torch.Tensor | None = None) -> torch.Tensor:
        """The estimate g of the gradient [d]."""
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=self.device)
        self._call(self._lib.ef21_get_state, None, None, _dev(out, torch.float32, (self.d,)))
        return out

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
