"""ctypes binding of hr_scores.h: products in 8 bits, log probabilities and distillation over matrices of scores.

As in ``binding``: functions with the names of the C entry points take tensors (or raw addresses) and sizes; the others
check their tensors, allocate results and workspace on the current stream of the tensors' device, and call those.
Matrices may be slices of columns of wider ones (rows contiguous); others are copied first.

Nothing here is recorded by autograd: results require no gradient, whatever their operands do.  A training step hands the gradient
that ``distill_step`` or a ``..._backward`` call returns to ``scores.backward(gradient)``.  ``out=`` counts as a change in place of that
tensor: where a recorded operation still needs its values, its backward pass says so.
"""
import ctypes
import functools
import inspect
from typing import NamedTuple, Optional

import torch

from .binding import _DTYPE, _addr, _check, _stream, HR_K_MAX, HrError, hr_last_error, lib

HR_I8_K_MAX, HR_LIST_MAX, HR_ROW_MAX = 131071, 512, 1 << 30
HR_WORKSPACE_ALIGN = 256

_c, _p = ctypes, ctypes.c_void_p
_i32, _i64, _f32, _size = _c.c_int32, _c.c_int64, _c.c_float, _c.c_size_t
_rows_args = [_p, _i64, _i32, _i64, _i64, _f32]
lib.hr_i8_quantize.argtypes = [_p, _i64, _i32, _i64, _i64, _p, _i64, _p, _p]
lib.hr_i8_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.hr_i8_workspace_bytes.restype = _size
lib.hr_i8_product.argtypes = [_p, _i64, _p, _p, _i64, _p, _p, _i64, _i64, _i64, _p, _i64, _i32, _p, _size, _p]
lib.hr_i8_linear.argtypes = [_p, _i64, _i32, _p, _i64, _p, _p, _i64, _i64, _i64, _p, _i64, _i32, _p, _size, _p]
lib.hr_logprobs_workspace_bytes.argtypes = [_i64, _i64, _i32]
lib.hr_logprobs_workspace_bytes.restype = _size
lib.hr_logprobs.argtypes = _rows_args + [_p, _i32, _i32, _p, _p, _p, _p, _p, _p, _size, _p]
lib.hr_logprobs_backward.argtypes = _rows_args + [_p, _i32, _p, _p, _p, _p, _p, _i64, _p]
lib.hr_distill_workspace_bytes.argtypes = [_i64, _i64, _i32]
lib.hr_distill_workspace_bytes.restype = _size
lib.hr_distill_forward.argtypes = _rows_args + [_p, _p, _i32, _p, _p, _p, _p, _size, _p]
lib.hr_distill_backward.argtypes = _rows_args + [_p, _p, _i32, _p, _p, _p, _i64, _p]
lib.hr_distill_step.argtypes = _rows_args + [_p, _p, _i32, _p, _p, _p, _p, _p, _i64, _p, _size, _p]


# ---- the C entry points by name

def hr_i8_quantize(x, ldx, dtype, m, k, q, ldq, scale, stream=None):
    _check(lib.hr_i8_quantize(_addr(x), ldx, dtype, m, k, _addr(q), ldq, _addr(scale), _stream(stream)))


def hr_i8_workspace_bytes(m, n, k):
    return int(lib.hr_i8_workspace_bytes(m, n, k))


def hr_i8_product(a, lda, a_scale, b, ldb, b_scale, bias, m, n, k, out, ldo, out_dtype, workspace, workspace_bytes, stream=None):
    _check(lib.hr_i8_product(_addr(a), lda, _addr(a_scale), _addr(b), ldb, _addr(b_scale), _addr(bias), m, n, k, _addr(out), ldo,
                             out_dtype, _addr(workspace), workspace_bytes, _stream(stream)))


def hr_i8_linear(x, ldx, x_dtype, b, ldb, b_scale, bias, m, n, k, out, ldo, out_dtype, workspace, workspace_bytes, stream=None):
    _check(lib.hr_i8_linear(_addr(x), ldx, x_dtype, _addr(b), ldb, _addr(b_scale), _addr(bias), m, n, k, _addr(out), ldo, out_dtype,
                            _addr(workspace), workspace_bytes, _stream(stream)))


def hr_logprobs_workspace_bytes(rows, n, k):
    return int(lib.hr_logprobs_workspace_bytes(rows, n, k))


def hr_logprobs(logits, ld, dtype, rows, n, scale, given, ngiven, k, out_logprobs, out_entropy, out_norm, out_top_ids, out_top_logprobs,
                workspace, workspace_bytes, stream=None):
    _check(lib.hr_logprobs(_addr(logits), ld, dtype, rows, n, scale, _addr(given), ngiven, k, _addr(out_logprobs), _addr(out_entropy),
                           _addr(out_norm), _addr(out_top_ids), _addr(out_top_logprobs), _addr(workspace), workspace_bytes,
                           _stream(stream)))


def hr_logprobs_backward(logits, ld, dtype, rows, n, scale, given, ngiven, entropy, norm, grad_logprobs, grad_entropy, grad_logits,
                         ldg, stream=None):
    _check(lib.hr_logprobs_backward(_addr(logits), ld, dtype, rows, n, scale, _addr(given), ngiven, _addr(entropy), _addr(norm),
                                    _addr(grad_logprobs), _addr(grad_entropy), _addr(grad_logits), ldg, _stream(stream)))


def hr_distill_workspace_bytes(rows, n, k):
    return int(lib.hr_distill_workspace_bytes(rows, n, k))


def hr_distill_forward(logits, ld, dtype, rows, n, scale, ids, teacher, k, out_loss, out_norm, out_q, workspace, workspace_bytes,
                       stream=None):
    _check(lib.hr_distill_forward(_addr(logits), ld, dtype, rows, n, scale, _addr(ids), _addr(teacher), k, _addr(out_loss),
                                  _addr(out_norm), _addr(out_q), _addr(workspace), workspace_bytes, _stream(stream)))


def hr_distill_backward(logits, ld, dtype, rows, n, scale, ids, q, k, norm, weights, grad_logits, ldg, stream=None):
    _check(lib.hr_distill_backward(_addr(logits), ld, dtype, rows, n, scale, _addr(ids), _addr(q), k, _addr(norm), _addr(weights),
                                   _addr(grad_logits), ldg, _stream(stream)))


def hr_distill_step(logits, ld, dtype, rows, n, scale, ids, teacher, k, weights, out_loss, out_norm, out_q, grad_logits, ldg, workspace,
                    workspace_bytes, stream=None):
    _check(lib.hr_distill_step(_addr(logits), ld, dtype, rows, n, scale, _addr(ids), _addr(teacher), k, _addr(weights), _addr(out_loss),
                               _addr(out_norm), _addr(out_q), _addr(grad_logits), ldg, _addr(workspace), workspace_bytes,
                               _stream(stream)))


# ---- tensors in, tensors out
# A call of these for one row takes less time on the GPU than Python takes around it: addresses and streams go to the library as
# plain numbers, sizes of workspaces are kept by shape, and the library is called without another function in between.

_raw_stream = torch._C._cuda_getCurrentRawStream          # (current_stream() makes an object first: 3 us)


def _kept(f):
    """Sizes that f gives, kept by shape; 0, a refusal, is raised and not kept: its message is that of the call that made it."""
    @functools.lru_cache(1024)
    def need(*shape):
        size = f(*shape)
        if size == 0:
            raise HrError(-1, hr_last_error())
        return size
    return need


_i8_bytes = _kept(lib.hr_i8_workspace_bytes)
_logprobs_bytes = _kept(lib.hr_logprobs_workspace_bytes)
_distill_bytes = _kept(lib.hr_distill_workspace_bytes)
_I8 = {torch.int8: None}


def _on_device(f):
    """The device of f's first argument is the current one while f runs."""
    name = next(iter(inspect.signature(f).parameters))

    @functools.wraps(f)
    def call(*args, **kw):
        t = args[0] if args else kw.get(name)
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device.index == torch._C._cuda_getDevice():
            return f(*args, **kw)
        with torch.cuda.device(t.device):
            return f(*args, **kw)
    return call


def _matrix(t, name, dtypes, columns=None):
    """A device matrix of one of the types whose rows are contiguous, and the distance between its rows."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise HrError(-1, f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise HrError(-1, f"{name} has dtype {t.dtype}, want one of {[str(d) for d in dtypes]}")
    if t.dim() != 2 or (columns is not None and t.shape[1] != columns):
        raise HrError(-1, f"{name} has shape {tuple(t.shape)}, want {('*', '*' if columns is None else columns)}")
    rows, cols = t.shape
    ld, step = t.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        t = t.contiguous()
        ld = cols
    return t, (ld if rows > 1 else max(cols, 1))


def _like(t, name, dtype, shape, device):
    """A contiguous tensor of this type and shape on the device."""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise HrError(-1, f"{name} must be a tensor on {device}")
    if t.dtype != dtype or t.shape != shape:
        raise HrError(-1, f"{name} is {t.dtype} {tuple(t.shape)}, want {dtype} {tuple(shape)}")
    return t.contiguous()


def _result(out, name, dtype, shape, device):
    """Where a result matrix goes, and the distance between its rows: a new one, or the caller's."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device), max(shape[1], 1)
    if not isinstance(out, torch.Tensor) or out.device != device or out.dtype != dtype or out.shape != shape:
        raise HrError(-1, f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device}")
    ld = out.stride(0)
    if (shape[1] > 1 and out.stride(1) != 1) or (shape[0] > 1 and ld < shape[1]):
        raise HrError(-1, f"{name} must have contiguous rows that do not overlap")
    return out, (ld if shape[0] > 1 else max(shape[1], 1))


def _written(out, result):
    """The result; where it lies in a tensor of the caller's (out), autograd learns that this has changed."""
    if out is not None:
        torch.autograd.graph.increment_version(out)
    return result


_unused = {}


def _workspace(need, device):
    """Of this many bytes; where a call wants none but has to be given one, always the same, which nothing reads or writes."""
    if need > HR_WORKSPACE_ALIGN:
        return torch.empty(need, dtype=torch.uint8, device=device)
    ws = _unused.get(device)
    if ws is None:
        ws = _unused[device] = torch.empty(HR_WORKSPACE_ALIGN, dtype=torch.uint8, device=device)
    return ws


def _at(t):
    return None if t is None else t.data_ptr()


def _padded(n):
    return (n + 63) // 64 * 64


@_on_device
def quantize_rows(x):
    """Rows of x [m, k] in 8 bits: (int8 [m, k], float32 scale [m]).  The rows lie a multiple of 64 bytes apart."""
    x, ld = _matrix(x, "x", _DTYPE)
    m, k = x.shape
    dev = x.device
    q = torch.empty(m, _padded(k), dtype=torch.int8, device=dev)
    scale = torch.empty(m, dtype=torch.float32, device=dev)
    _check(lib.hr_i8_quantize(x.data_ptr(), ld, _DTYPE[x.dtype], m, k, q.data_ptr(), q.shape[1], scale.data_ptr(), _raw_stream(dev.index)))
    return q[:, :k], scale


def _i8_matrix(t, name, columns=None):
    """An int8 matrix, copied where the library would read behind its memory (rows on 16-byte boundaries of a length that is not)."""
    t, ld = _matrix(t, name, _I8, columns)
    rows, k = t.shape
    if k % 16 and rows and ld % 16 == 0 and t.data_ptr() % 16 == 0 and \
            t.storage_offset() + (rows - 1) * ld + (k + 15) // 16 * 16 > t.untyped_storage().nbytes():
        copy = torch.zeros(rows, _padded(k), dtype=torch.int8, device=t.device)
        copy[:, :k] = t
        return copy[:, :k], copy.shape[1]
    return t, ld


def _product_operands(m, k, dev, b, b_scale, bias, dtype, out):
    b, ldb = _i8_matrix(b, "b", k)
    n = b.shape[0]
    if b.device != dev:
        raise HrError(-1, f"b is on {b.device}, want {dev}")
    if dtype not in _DTYPE:
        raise HrError(-1, f"dtype {dtype}: want float32, float16 or bfloat16")
    b_scale = _like(b_scale, "b_scale", torch.float32, (n,), dev)
    bias = None if bias is None else _like(bias, "bias", torch.float32, (n,), dev)
    result, ldo = _result(out, "out", dtype, (m, n), dev)
    return b, ldb, n, b_scale, bias, result, ldo, _workspace(_i8_bytes(m, n, k), dev)


@_on_device
def i8_product(a, a_scale, b, b_scale, bias=None, dtype=torch.float32, out=None):
    """a [m, k] times b [n, k] transposed, both int8, in the scales [m] and [n] of their rows, plus bias [n]: [m, n] in dtype.
    Not recorded by autograd."""
    a, lda = _i8_matrix(a, "a")
    m, k = a.shape
    dev = a.device
    a_scale = _like(a_scale, "a_scale", torch.float32, (m,), dev)
    b, ldb, n, b_scale, bias, result, ldo, ws = _product_operands(m, k, dev, b, b_scale, bias, dtype, out)
    _check(lib.hr_i8_product(a.data_ptr(), lda, a_scale.data_ptr(), b.data_ptr(), ldb, b_scale.data_ptr(), _at(bias), m, n, k, result.data_ptr(),
                             ldo, _DTYPE[dtype], ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return _written(out, result)


@_on_device
def i8_linear(x, b, b_scale, bias=None, dtype=torch.float32, out=None):
    """Rows of floats x [m, k], quantised row by row, times b [n, k] int8 transposed: [m, n] in dtype.
    Not recorded by autograd."""
    x, ldx = _matrix(x, "x", _DTYPE)
    m, k = x.shape
    dev = x.device
    b, ldb, n, b_scale, bias, result, ldo, ws = _product_operands(m, k, dev, b, b_scale, bias, dtype, out)
    _check(lib.hr_i8_linear(x.data_ptr(), ldx, _DTYPE[x.dtype], b.data_ptr(), ldb, b_scale.data_ptr(), _at(bias), m, n, k, result.data_ptr(), ldo,
                            _DTYPE[dtype], ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return _written(out, result)


class Logprobs(NamedTuple):
    """What ``logprobs`` finds: ln p of the given entries, entropy and norm of every row, its best alternatives."""
    logprobs: Optional[torch.Tensor]
    entropy: torch.Tensor
    norm: torch.Tensor
    top_ids: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


def _list(ids, name, rows, device):
    if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int64, torch.int32):
        raise HrError(-1, f"{name} must be an integer tensor")
    if ids.device != device or ids.dim() != 2 or ids.shape[0] != rows or ids.shape[1] > HR_LIST_MAX:
        raise HrError(-1, f"{name} must be a [{rows}, 0..{HR_LIST_MAX}] tensor on {device}")
    return (ids if ids.dtype == torch.int64 else ids.to(torch.int64)).contiguous()


@_on_device
def logprobs(logits, given=None, k=0, scale=1.0):
    """softmax(scale * logits) of every row [rows, n]: log probabilities of the given entries [rows, g], entropy, the k best.
    Not recorded by autograd: the gradient is ``logprobs_backward``."""
    z, ld = _matrix(logits, "logits", _DTYPE)
    rows, n = z.shape
    dev = z.device
    g, lp, ids, top = 0, None, None, None
    if given is not None:
        given = _list(given, "given", rows, dev)
        g = given.shape[1]
        lp = torch.empty(rows, g, dtype=torch.float32, device=dev)
    ws = _workspace(_logprobs_bytes(rows, n, k), dev)
    entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    norm = torch.empty(rows, 2, dtype=torch.float32, device=dev)
    if k > 0:
        ids = torch.empty(rows, k, dtype=torch.int64, device=dev)
        top = torch.empty(rows, k, dtype=torch.float32, device=dev)
    _check(lib.hr_logprobs(z.data_ptr(), ld, _DTYPE[z.dtype], rows, n, scale, _at(given), g, k, _at(lp), entropy.data_ptr(), norm.data_ptr(),
                           _at(ids), _at(top), ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return Logprobs(lp, entropy, norm, ids, top)


@_on_device
def logprobs_backward(logits, given, result, grad_logprobs=None, grad_entropy=None, scale=1.0, out=None):
    """Gradient with respect to the logits, given those with respect to the result's logprobs [rows, g] and entropy [rows]
    (None: 0).  ``out`` may be the logits themselves."""
    z, ld = _matrix(logits, "logits", _DTYPE)
    rows, n = z.shape
    dev = z.device
    given = None if given is None else _list(given, "given", rows, dev)
    g = 0 if given is None else given.shape[1]
    entropy = _like(result.entropy, "result.entropy", torch.float32, (rows,), dev)
    norm = _like(result.norm, "result.norm", torch.float32, (rows, 2), dev)
    if grad_logprobs is not None:
        if given is None:
            raise HrError(-1, "grad_logprobs without given entries")
        grad_logprobs = _like(grad_logprobs, "grad_logprobs", torch.float32, (rows, g), dev)
    if grad_entropy is not None:
        grad_entropy = _like(grad_entropy, "grad_entropy", torch.float32, (rows,), dev)
    grad, ldg = _result(out, "out", z.dtype, (rows, n), dev)
    _check(lib.hr_logprobs_backward(z.data_ptr(), ld, _DTYPE[z.dtype], rows, n, scale, _at(given), g, entropy.data_ptr(), norm.data_ptr(),
                                    _at(grad_logprobs), _at(grad_entropy), grad.data_ptr(), ldg, _raw_stream(dev.index)))
    return _written(out, grad)


def _taught(logits, ids, name, values):
    z, ld = _matrix(logits, "logits", _DTYPE)
    ids = _list(ids, "ids", z.shape[0], z.device)
    if ids.shape[1] < 1:
        raise HrError(-1, "ids has no columns")
    return z, ld, ids, _like(values, name, torch.float32, ids.shape, z.device)


@_on_device
def distill_forward(logits, ids, teacher, scale=1.0):
    """Loss [rows] of the logits [rows, n] against a teacher's scores [rows, k] of the entries ids [rows, k] (-1: empty), and what
    ``distill_backward`` needs: (loss, norm, q).  Not recorded by autograd."""
    z, ld, ids, teacher = _taught(logits, ids, "teacher", teacher)
    rows, n = z.shape
    k, dev = ids.shape[1], z.device
    loss = torch.empty(rows, dtype=torch.float32, device=dev)
    norm = torch.empty(rows, 2, dtype=torch.float32, device=dev)
    q = torch.empty(rows, k, dtype=torch.float32, device=dev)
    ws = _workspace(_distill_bytes(rows, n, k), dev)
    _check(lib.hr_distill_forward(z.data_ptr(), ld, _DTYPE[z.dtype], rows, n, scale, ids.data_ptr(), teacher.data_ptr(), k, loss.data_ptr(),
                                  norm.data_ptr(), q.data_ptr(), ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return loss, norm, q


@_on_device
def distill_backward(logits, ids, q, norm, weights=None, scale=1.0, out=None):
    """Gradient with respect to the logits; weights [rows]: that of the caller's loss with respect to every row's (None: 1).
    ``out`` may be the logits themselves."""
    z, ld, ids, q = _taught(logits, ids, "q", q)
    rows, n = z.shape
    dev = z.device
    norm = _like(norm, "norm", torch.float32, (rows, 2), dev)
    weights = None if weights is None else _like(weights, "weights", torch.float32, (rows,), dev)
    grad, ldg = _result(out, "out", z.dtype, (rows, n), dev)
    _check(lib.hr_distill_backward(z.data_ptr(), ld, _DTYPE[z.dtype], rows, n, scale, ids.data_ptr(), q.data_ptr(), ids.shape[1],
                                   norm.data_ptr(), _at(weights), grad.data_ptr(), ldg, _raw_stream(dev.index)))
    return _written(out, grad)


@_on_device
def distill_step(logits, ids, teacher, weights=None, scale=1.0, out=None):
    """``distill_forward`` and ``distill_backward`` in one, for weights known beforehand: (loss [rows], gradient [rows, n]).
    Not recorded by autograd: the gradient goes to ``logits.backward``.  ``out`` may be the logits themselves."""
    z, ld, ids, teacher = _taught(logits, ids, "teacher", teacher)
    rows, n = z.shape
    k, dev = ids.shape[1], z.device
    weights = None if weights is None else _like(weights, "weights", torch.float32, (rows,), dev)
    loss = torch.empty(rows, dtype=torch.float32, device=dev)
    grad, ldg = _result(out, "out", z.dtype, (rows, n), dev)
    ws = _workspace(_distill_bytes(rows, n, k), dev)
    _check(lib.hr_distill_step(z.data_ptr(), ld, _DTYPE[z.dtype], rows, n, scale, ids.data_ptr(), teacher.data_ptr(), k, _at(weights),
                               loss.data_ptr(), None, None, grad.data_ptr(), ldg, ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return loss, _written(out, grad)
