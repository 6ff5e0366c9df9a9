"""ctypes binding of hr_layers.h: layer norm, gated feed-forward blocks, AdamW.

As in ``scores``: functions with the names of the C entry points take tensors (or raw addresses) and sizes; the others check their
tensors, allocate results and workspace on the current stream of the tensors' device, and call those.  Matrices may be slices of columns
of wider ones (rows contiguous); others are copied first.

Nothing here is recorded by autograd: a training step calls the ``..._backward`` functions itself, last layer first.  ``out=``, and what
``adamw`` updates, counts as a change in place of that tensor.
"""
import ctypes
import functools
import struct
from itertools import chain
from typing import NamedTuple, Optional

import torch

from .binding import _DTYPE, _addr, _check, _stream, HR_F32, HrError, lib
from .scores import _at, _current_device, _kept, _like, _matrix, _on_device, _raw_stream, _result, _workspace, _written

HR_SILU, HR_GELU, HR_GELU_TANH = 0, 1, 2
HR_GATED_MAX, HR_ADAMW_BLOCK = 1 << 19, 256
_ACT = {"silu": HR_SILU, "gelu": HR_GELU, "gelu_tanh": HR_GELU_TANH}

_c, _p = ctypes, ctypes.c_void_p
_i32, _i64, _f32, _f64, _size = _c.c_int32, _c.c_int64, _c.c_float, _c.c_double, _c.c_size_t
lib.hr_layer_norm.argtypes = [_p, _i64, _i32, _i64, _i64, _p, _p, _i32, _f32, _p, _i64, _p, _p]
lib.hr_layer_norm_workspace_bytes.argtypes = [_i64, _i64]
lib.hr_layer_norm_workspace_bytes.restype = _size
lib.hr_layer_norm_backward.argtypes = [_p, _i64, _i32, _i64, _i64, _p, _i32, _p, _p, _i64, _p, _i64, _p, _p, _p, _size, _p]
lib.hr_gated_workspace_bytes.argtypes = [_i64, _i64, _i64, _i32]
lib.hr_gated_workspace_bytes.restype = _size
lib.hr_gated.argtypes = [_p, _i64, _p, _i64, _p, _i64, _i32, _i64, _i64, _i64, _i32, _p, _i64, _p, _p, _size, _p]
lib.hr_gated_backward_workspace_bytes.argtypes = [_i64, _i64, _i64, _i32]
lib.hr_gated_backward_workspace_bytes.restype = _size
lib.hr_gated_backward.argtypes = [_p, _i64, _p, _i64, _p, _i64, _i32, _i64, _i64, _i64, _i32, _p, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _size, _p]
lib.hr_adamw.argtypes = [_p, _i32, _f64, _f64, _f64, _f64, _i64, _p, _p, _p]
lib.hr_adamw_moments.argtypes = [_p, _p, _p, _i64, _p, _p, _p]


class hr_adamw_tensor(ctypes.Structure):
    """One tensor of hr_adamw."""
    _fields_ = [("param", _p), ("grad", _p), ("master", _p), ("m", _p), ("v", _p), ("exponents", _p), ("n", _i64), ("weight_decay", _f32),
                ("param_dtype", _i32), ("grad_dtype", _i32)]


@functools.lru_cache(64)
def _tables(n):
    """n of these, as struct packs them."""
    return struct.Struct("@" + "6Pqfii4x" * n)


# ---- the C entry points by name

def hr_layer_norm(x, ldx, dtype, rows, n, weight, bias, weight_dtype, eps, out, ldo, out_stats, stream=None):
    _check(lib.hr_layer_norm(_addr(x), ldx, dtype, rows, n, _addr(weight), _addr(bias), weight_dtype, eps, _addr(out), ldo, _addr(out_stats),
                             _stream(stream)))


def hr_layer_norm_workspace_bytes(rows, n):
    return int(lib.hr_layer_norm_workspace_bytes(rows, n))


def hr_layer_norm_backward(x, ldx, dtype, rows, n, weight, weight_dtype, stats, grad_out, ldg, grad_x, ldgx, grad_weight, grad_bias, workspace,
                           workspace_bytes, stream=None):
    _check(lib.hr_layer_norm_backward(_addr(x), ldx, dtype, rows, n, _addr(weight), weight_dtype, _addr(stats), _addr(grad_out), ldg,
                                      _addr(grad_x), ldgx, _addr(grad_weight), _addr(grad_bias), _addr(workspace), workspace_bytes,
                                      _stream(stream)))


def hr_gated_workspace_bytes(m, k, f, dtype):
    return int(lib.hr_gated_workspace_bytes(m, k, f, dtype))


def hr_gated(x, ldx, w_gate, ldwg, w_up, ldwu, dtype, m, k, f, activation, out, ldo, out_pre, workspace, workspace_bytes, stream=None):
    _check(lib.hr_gated(_addr(x), ldx, _addr(w_gate), ldwg, _addr(w_up), ldwu, dtype, m, k, f, activation, _addr(out), ldo, _addr(out_pre),
                        _addr(workspace), workspace_bytes, _stream(stream)))


def hr_gated_backward_workspace_bytes(m, k, f, dtype):
    return int(lib.hr_gated_backward_workspace_bytes(m, k, f, dtype))


def hr_gated_backward(x, ldx, w_gate, ldwg, w_up, ldwu, dtype, m, k, f, activation, pre, grad_out, ldgo, grad_x, ldgx, grad_w_gate, ldgg,
                      grad_w_up, ldgu, workspace, workspace_bytes, stream=None):
    _check(lib.hr_gated_backward(_addr(x), ldx, _addr(w_gate), ldwg, _addr(w_up), ldwu, dtype, m, k, f, activation, _addr(pre), _addr(grad_out),
                                 ldgo, _addr(grad_x), ldgx, _addr(grad_w_gate), ldgg, _addr(grad_w_up), ldgu, _addr(workspace),
                                 workspace_bytes, _stream(stream)))


def hr_adamw(tensors, count, lr, beta1, beta2, eps, step, device_step=None, grad_scale=None, stream=None):
    """tensors: an array of ``hr_adamw_tensor`` in host memory."""
    _check(lib.hr_adamw(ctypes.cast(tensors, _p), count, lr, beta1, beta2, eps, step, _addr(device_step), _addr(grad_scale), _stream(stream)))


def hr_adamw_moments(m, v, exponents, n, out_m, out_v, stream=None):
    _check(lib.hr_adamw_moments(_addr(m), _addr(v), _addr(exponents), n, _addr(out_m), _addr(out_v), _stream(stream)))


# ---- tensors in, tensors out

_norm_bytes = _kept(lib.hr_layer_norm_workspace_bytes)
_gated_bytes = _kept(lib.hr_gated_workspace_bytes)
_gated_backward_bytes = _kept(lib.hr_gated_backward_workspace_bytes)


class LayerNorm(NamedTuple):
    """What ``layer_norm`` gives: the rows, and mean and 1 / spread of each, [rows, 2]."""
    out: torch.Tensor
    stats: torch.Tensor


class LayerNormGrads(NamedTuple):
    """Gradients of rows, weight and bias."""
    x: torch.Tensor
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]


def _vector(t, name, n, dtype, device):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise HrError(-1, f"{name} must be a tensor on {device}")
    if (t.dtype is not torch.float32 and t.dtype is not dtype) or t.shape != (n,):
        raise HrError(-1, f"{name} is {t.dtype} {tuple(t.shape)}, want {torch.float32} or {dtype} {(n,)}")
    return t if t.is_contiguous() else t.contiguous()


@_on_device
def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None):
    """Rows of x [rows, n] with mean and spread taken out, times weight [n], plus bias [n] (both float32 or both of x's type).
    ``out`` may be x itself.  Not recorded by autograd: the gradients are ``layer_norm_backward``'s."""
    x, ldx = _matrix(x, "x", _DTYPE)
    rows, n = x.shape
    dev, dtype = x.device, x.dtype
    weight, bias = _vector(weight, "weight", n, dtype, dev), _vector(bias, "bias", n, dtype, dev)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise HrError(-1, f"weight is {weight.dtype}, bias {bias.dtype}")
    given = weight if weight is not None else bias
    y, ldo = _result(out, "out", dtype, (rows, n), dev)
    stats = torch.empty(rows, 2, dtype=torch.float32, device=dev)
    _check(lib.hr_layer_norm(x.data_ptr(), ldx, _DTYPE[dtype], rows, n, _at(weight), _at(bias), HR_F32 if given is None else _DTYPE[given.dtype], eps,
                             y.data_ptr(), ldo, stats.data_ptr(), _raw_stream(dev.index)))
    return LayerNorm(_written(out, y), stats)


@_on_device
def layer_norm_backward(x, weight, stats, grad_out, parameters=True, out=None):
    """Gradients of a ``layer_norm`` call from that of its rows, grad_out [rows, n]; stats as it returned them.  Those of weight and bias have
    weight's type (float32 where it is None), and are None where ``parameters`` is false.  ``out``, for that of x, may be grad_out itself."""
    x, ldx = _matrix(x, "x", _DTYPE)
    rows, n = x.shape
    dev, dtype = x.device, x.dtype
    weight = _vector(weight, "weight", n, dtype, dev)
    stats = _like(stats, "stats", torch.float32, (rows, 2), dev)
    dy, ldg = _matrix(grad_out, "grad_out", {dtype: None}, n)
    if dy.device != dev or dy.shape != x.shape:
        raise HrError(-1, f"grad_out must be a {(rows, n)} tensor on {dev}")
    kind = torch.float32 if weight is None else weight.dtype
    dx, ldgx = _result(out, "out", dtype, (rows, n), dev)
    dw = db = None
    if parameters:
        dw = torch.empty(n, dtype=kind, device=dev)
        db = torch.empty_like(dw)
    ws = _workspace(_norm_bytes(rows, n), dev)
    _check(lib.hr_layer_norm_backward(x.data_ptr(), ldx, _DTYPE[dtype], rows, n, _at(weight), _DTYPE[kind], stats.data_ptr(), dy.data_ptr(), ldg,
                                      dx.data_ptr(), ldgx, _at(dw), _at(db), ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return LayerNormGrads(_written(out, dx), dw, db)


class Gated(NamedTuple):
    """What ``gated`` gives: act(gate) * up, and gate and up of every row, [m, 2, f] float32, where they were to be kept."""
    out: torch.Tensor
    pre: Optional[torch.Tensor]


class GatedGrads(NamedTuple):
    """Gradients of the rows and of both matrices."""
    x: Optional[torch.Tensor]
    w_gate: Optional[torch.Tensor]
    w_up: Optional[torch.Tensor]


def _gated_operands(x, w_gate, w_up, activation):
    x, ldx = _matrix(x, "x", _DTYPE)
    m, k = x.shape
    if activation not in _ACT:
        raise HrError(-1, f"activation {activation!r}: want one of {sorted(_ACT)}")
    w_gate, ldwg = _matrix(w_gate, "w_gate", {x.dtype: None}, k)
    f = w_gate.shape[0]
    w_up, ldwu = _matrix(w_up, "w_up", {x.dtype: None}, k)
    if w_up.shape[0] != f:
        raise HrError(-1, f"w_gate has {f} rows, w_up {w_up.shape[0]}")
    if w_gate.device != x.device or w_up.device != x.device:
        raise HrError(-1, f"w_gate and w_up must be on {x.device}")
    return x, ldx, w_gate, ldwg, w_up, ldwu, m, k, f


@_on_device
def gated(x, w_gate, w_up, activation="silu", keep=False, out=None):
    """act(x w_gate') * (x w_up') of x [m, k] and w_gate, w_up [f, k], all of one type: [m, f].  activation: "silu", "gelu" or "gelu_tanh".
    keep: gate and up come back too, for ``gated_backward``.  Not recorded by autograd."""
    x, ldx, w_gate, ldwg, w_up, ldwu, m, k, f = _gated_operands(x, w_gate, w_up, activation)
    dev, kind = x.device, _DTYPE[x.dtype]
    ws = _workspace(_gated_bytes(m, k, f, kind), dev)
    h, ldo = _result(out, "out", x.dtype, (m, f), dev)
    pre = torch.empty(m, 2, f, dtype=torch.float32, device=dev) if keep else None
    _check(lib.hr_gated(x.data_ptr(), ldx, w_gate.data_ptr(), ldwg, w_up.data_ptr(), ldwu, kind, m, k, f, _ACT[activation], h.data_ptr(), ldo, _at(pre),
                        ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return Gated(_written(out, h), pre)


@_on_device
def gated_backward(x, w_gate, w_up, pre, grad_out, activation="silu", rows=True, matrices=True):
    """Gradients of a ``gated`` call from that of its result, grad_out [m, f]; pre as it kept it.  rows, matrices: whether that of x and those of
    w_gate and w_up are wanted (None otherwise)."""
    x, ldx, w_gate, ldwg, w_up, ldwu, m, k, f = _gated_operands(x, w_gate, w_up, activation)
    dev, kind = x.device, _DTYPE[x.dtype]
    pre = _like(pre, "pre", torch.float32, (m, 2, f), dev)
    dh, ldgo = _matrix(grad_out, "grad_out", {x.dtype: None}, f)
    if dh.device != dev or dh.shape[0] != m:
        raise HrError(-1, f"grad_out must be a {(m, f)} tensor on {dev}")
    ws = _workspace(_gated_backward_bytes(m, k, f, kind), dev)
    dx = torch.empty(m, k, dtype=x.dtype, device=dev) if rows else None
    dg = du = None
    if matrices:
        dg = torch.empty(f, k, dtype=x.dtype, device=dev)
        du = torch.empty_like(dg)
    _check(lib.hr_gated_backward(x.data_ptr(), ldx, w_gate.data_ptr(), ldwg, w_up.data_ptr(), ldwu, kind, m, k, f, _ACT[activation], pre.data_ptr(),
                                 dh.data_ptr(), ldgo, _at(dx), k, _at(dg), k, _at(du), k, ws.data_ptr(), ws.numel(), _raw_stream(dev.index)))
    return GatedGrads(dx, dg, du)


def adamw_state(param, bits=32):
    """Moments of a tensor that has taken no step, for ``adamw``: (m, v, exponents); exponents are None where bits is 32."""
    if bits not in (32, 8):
        raise HrError(-1, f"bits={bits}: want 32 or 8")
    kind = torch.float32 if bits == 32 else torch.uint8
    m, v = (torch.zeros(param.shape, dtype=kind, device=param.device) for _ in range(2))
    blocks = (param.numel() + HR_ADAMW_BLOCK - 1) // HR_ADAMW_BLOCK
    return m, v, None if bits == 32 else torch.zeros(blocks, 2, dtype=torch.uint8, device=param.device)


def _refuse(i, p, g, w, m, v, e, device):
    """Says what is wrong with the i-th tensor of a step, if anything is."""
    for name, t in (("params", p), ("grads", g), ("m", m), ("v", v), ("masters", w), ("exponents", e)):
        if t is None and name in ("masters", "exponents"):
            continue
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != device:
            raise HrError(-1, f"{name}[{i}] must be a tensor on {device}")
        if name != "grads" and not t.is_contiguous():
            raise HrError(-1, f"{name}[{i}] is not contiguous")
        if name != "exponents" and t.numel() != p.numel():
            raise HrError(-1, f"{name}[{i}] has {t.numel()} numbers, params[{i}] {p.numel()}")
    for name, t in (("params", p), ("grads", g)):
        if t.dtype not in _DTYPE:
            raise HrError(-1, f"{name}[{i}] has dtype {t.dtype}, want one of {[str(d) for d in _DTYPE]}")
    if g.shape != p.shape:
        raise HrError(-1, f"grads[{i}] has shape {tuple(g.shape)}, params[{i}] {tuple(p.shape)}")
    if w is not None and (w.dtype != torch.float32 or p.dtype == torch.float32):
        raise HrError(-1, f"masters[{i}] is {w.dtype} beside a {p.dtype} parameter, want float32 beside 16 bits, or None")
    want = torch.float32 if e is None else torch.uint8
    if m.dtype != want or v.dtype != want:
        raise HrError(-1, f"m[{i}] and v[{i}] are {m.dtype} and {v.dtype}, want {want}" + (": exponents are None" if e is None else ""))
    shape = ((p.numel() + HR_ADAMW_BLOCK - 1) // HR_ADAMW_BLOCK, 2)
    if e is not None and (e.dtype != torch.uint8 or e.shape != shape):
        raise HrError(-1, f"exponents[{i}] is {e.dtype} {tuple(e.shape)}, want {torch.uint8} {shape}")


_numel, _get_device, _is_contiguous, _data_ptr = torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous, torch.Tensor.data_ptr
_F32, _U8 = torch.float32, torch.uint8


def _lists(n, **named):
    found = []
    for name, x in named.items():
        x = [None] * n if x is None else list(x)
        if len(x) != n:
            raise HrError(-1, f"{name} has {len(x)} entries, params {n}")
        found.append(x)
    return found


def adamw(params, grads, m, v, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, exponents=None, masters=None, grad_scale=None):
    """One step of AdamW over all tensors of the lists, in place.

    params: contiguous tensors on one device.  grads: tensors of their shapes, or None for a parameter that this step leaves alone.  m, v:
    moments (see ``adamw_state``), float32, or uint8 with their exponents.  masters: None, or a list with float32 copies of 16-bit parameters (or
    None for those that have none), which are updated in their place.  weight_decay: a number, or one for each tensor.  step: the number of
    this step, from 1 on, or an int64 tensor of one element on the device (for captured steps).  grad_scale: None, or a float32 tensor of one
    element on the device that all gradients are multiplied by."""
    params = list(params)
    n = len(params)
    grads, m, v, exponents, masters = _lists(n, grads=grads, m=m, v=v, exponents=exponents, masters=masters)
    decay = _lists(n, weight_decay=weight_decay)[0] if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
    if not n:
        return
    if not isinstance(params[0], torch.Tensor) or not params[0].is_cuda:
        raise HrError(-1, "params[0] must be a device tensor")
    dev = params[0].device
    device_step = scale = None
    if isinstance(step, torch.Tensor):
        device_step, step = _like(step, "step", torch.int64, step.shape, dev), 0
        if device_step.numel() != 1:
            raise HrError(-1, f"step has {device_step.numel()} elements, want 1")
    if grad_scale is not None:
        scale = _like(grad_scale, "grad_scale", torch.float32, grad_scale.shape if isinstance(grad_scale, torch.Tensor) else (), dev)
        if scale.numel() != 1:
            raise HrError(-1, f"grad_scale has {scale.numel()} elements, want 1")
    if any(g is None for g in grads):
        kept = [i for i, g in enumerate(grads) if g is not None]
        params, grads, m, v, exponents, masters, decay = ([x[i] for i in kept] for x in (params, grads, m, v, exponents, masters, decay))
        n = len(params)
    # (hundreds of tensors: what is asked of each is asked of whole lists, by functions that are not Python's)
    has_e, has_w = [e for e in exponents if e is not None], [w for w in masters if w is not None]
    try:
        sizes, kinds, shapes = list(map(_numel, params)), [p.dtype for p in params], [p.shape for p in params]
        wants = [_F32] * n if not has_e else [_F32 if e is None else _U8 for e in exponents]
        fine = (set(map(_get_device, chain(params, grads, m, v, has_e, has_w))) <= {dev.index} and all(map(_is_contiguous, chain(params, m, v, has_e, has_w)))
                and [g.shape for g in grads] == shapes and list(map(_numel, m)) == sizes and list(map(_numel, v)) == sizes
                and [t.dtype for t in m] == wants and [t.dtype for t in v] == wants
                and (not has_e or [(e.dtype, *e.shape) for e in has_e] == [(_U8, (k + HR_ADAMW_BLOCK - 1) // HR_ADAMW_BLOCK, 2) for k, e in zip(sizes, exponents) if e is not None])
                and (not has_w or [(w.dtype, w.numel(), False) for w in has_w] == [(_F32, k, d is _F32) for k, d, w in zip(sizes, kinds, masters) if w is not None]))
        ptypes, gtypes = [_DTYPE[d] for d in kinds], [_DTYPE[g.dtype] for g in grads]
    except (AttributeError, KeyError, TypeError):
        fine = False
    if not fine:
        for i, x in enumerate(zip(params, grads, masters, m, v, exponents)):
            _refuse(i, *x, dev)
    if not all(map(_is_contiguous, grads)):
        grads = [g.contiguous() for g in grads]
    at = [list(map(_data_ptr, x)) for x in (params, grads, m, v)]
    wat, eat = ([0 if t is None else t.data_ptr() for t in x] if has else [0] * n for x, has in ((masters, has_w), (exponents, has_e)))
    places = at[0] + at[2] + at[3] + (wat if has_w else []) + (eat if has_e else [])
    if 0 in sizes or 0 < len(has_w) < n or 0 < len(has_e) < n:           # (addresses of nothing are no places)
        places = [x for x, k in zip(places, sizes * 5) if k and x]
    if len(set(places)) != len(places):
        raise HrError(-1, "a tensor is in the lists twice")
    table = _tables(n).pack(*chain.from_iterable(zip(at[0], at[1], wat, at[2], at[3], eat, sizes, decay, ptypes, gtypes)))
    beta1, beta2 = betas
    if dev.index == _current_device():
        _check(lib.hr_adamw(table, n, lr, beta1, beta2, eps, step, _at(device_step), _at(scale), _raw_stream(dev.index)))
    else:
        with torch.cuda.device(dev):
            _check(lib.hr_adamw(table, n, lr, beta1, beta2, eps, step, _at(device_step), _at(scale), _raw_stream(dev.index)))
    torch.autograd.graph.increment_version(list(chain(params, m, v, has_e, has_w)))


@_on_device
def adamw_moments(m, v, exponents):
    """The numbers that moments in 8 bits stand for: (m, v) in float32, in the shape of m."""
    dev = m.device if isinstance(m, torch.Tensor) else None
    if dev is None or not m.is_cuda:
        raise HrError(-1, "m must be a device tensor")
    m = _like(m, "m", torch.uint8, m.shape, dev)
    v = _like(v, "v", torch.uint8, m.shape, dev)
    n = m.numel()
    exponents = _like(exponents, "exponents", torch.uint8, ((n + HR_ADAMW_BLOCK - 1) // HR_ADAMW_BLOCK, 2), dev)
    fm, fv = (torch.empty(m.shape, dtype=torch.float32, device=dev) for _ in range(2))
    _check(lib.hr_adamw_moments(m.data_ptr(), v.data_ptr(), exponents.data_ptr(), n, fm.data_ptr(), fv.data_ptr(), _raw_stream(dev.index)))
    return fm, fv
