"""Operators on device tensors: rows routed to experts, and layers in 4 bits.

A population's variants can serve together, each row going to the few of them
that a router chooses (mixture.py does so); the same calls run any experts held
as one tensor of weight matrices.  This module marshals arguments of the
library's calls (include/gevo.h, which states the mathematics): outputs come
from torch's allocator, work goes to the tensors' device on torch's current
stream, so calls can be captured into a graph.  Tensors are float32 or
bfloat16; rows may be strided, a last dimension that is not contiguous is
copied first.  A wrong argument raises GevoError and launches nothing.

These calls are not recorded by autograd: an output does not ask for a
gradient, whatever its inputs do.  Gradients are the calls named backward,
whose results the caller hands on (logits.backward(route_backward(...))).

    weights, ids = route(logits, top_k)              # [T][k] each
    plan = route_plan(ids, n_experts)                # slots sorted by expert
    rows = expert_forward(x, w, plan, bias, relu=True)       # [T k][N], sorted
    y = expert_combine(rows, plan, weights)          # [T][N]

and backward: expert_combine_backward, expert_backward, route_backward.
    q = mx4_quantize(w)                              # 4.25 bits a value
    y = mx4_matmul(mx4_quantize(x), q)               # every matrix, or routed with plan=
"""
from __future__ import annotations

import ctypes
import functools
import operator

import torch

from . import GEVO_ABI_VERSION, GevoError, _check, lib

SCORES = {"softmax": 0, "sigmoid": 1}
DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_u32, _i64, _int = ctypes.c_uint32, ctypes.c_int64, ctypes.c_int


class RouteConfig(ctypes.Structure):
    _fields_ = [("abi_version", _u32), ("E", _u32), ("k", _u32), ("T", _i64), ("dtype", _int), ("score", _int),
                ("logits_stride", _i64), ("groups", _u32), ("top_groups", _u32), ("group_top", _u32),
                ("renorm", _u32), ("scale", ctypes.c_float)]


class ExpertConfig(ctypes.Structure):
    _fields_ = [("abi_version", _u32), ("dtype", _int), ("out_dtype", _int), ("E", _u32), ("k", _u32), ("N", _u32),
                ("K", _u32), ("T", _i64), ("x_stride", _i64), ("w_stride_e", _i64), ("w_stride_n", _i64),
                ("y_stride", _i64), ("sorted_rows", _u32), ("relu", _u32)]


class CombineConfig(ctypes.Structure):
    _fields_ = [("abi_version", _u32), ("dtype", _int), ("out_dtype", _int), ("k", _u32), ("N", _u32), ("T", _i64),
                ("rows_stride", _i64), ("y_stride", _i64)]


class Mx4Config(ctypes.Structure):
    _fields_ = [("abi_version", _u32), ("out_dtype", _int), ("P", _u32), ("N", _u32), ("K", _u32), ("M", _i64),
                ("a_each", _u32), ("k", _u32), ("sorted_rows", _u32), ("relu", _u32)]


def _rows(t, name, dims=2):
    """t with dims dimensions, of a type that the kernels take, its last one contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise GevoError(f"{name}: a tensor on the GPU")
    if t.dtype not in DTYPES:
        raise GevoError(f"{name}: float32 or bfloat16, not {t.dtype}")
    if t.dim() != dims:
        raise GevoError(f"{name}: {dims} dimensions, not {t.dim()}")
    return t if t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


def _flat(t, name, dtype, shape, device):
    """t as a contiguous tensor of one type and shape."""
    if not (isinstance(t, torch.Tensor) and t.device == device):
        raise GevoError(f"{name}: a tensor on {device}")
    if t.dtype != dtype or t.shape != shape:
        raise GevoError(f"{name}: {dtype} of shape {tuple(shape)}, not {t.dtype} of {tuple(t.shape)}")
    return t if t.is_contiguous() else t.contiguous()


# New contiguous tensors.  (empty_strided parses its arguments in 0.6 of empty's
# time: an output costs 1.0 us so, 1.7 by empty.)
def _new(shape, dtype, device):
    strides, n = [], 1
    for size in reversed(shape):
        strides.append(n)
        n *= size
    return torch.empty_strided(shape, strides[::-1], dtype=dtype, device=device)


def _new_rows(rows, columns, dtype, device):
    return torch.empty_strided((rows, columns), (columns, 1), dtype=dtype, device=device)


def _new_flat(n, dtype, device):
    return torch.empty_strided((n,), (1,), dtype=dtype, device=device)


def _stride(t):
    """Elements between t's rows; a row's length where there is one row or none."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[-1]


def _out_dtype(dtype, default):
    if dtype is None:
        return default
    if not isinstance(dtype, torch.dtype) or dtype not in DTYPES:
        raise GevoError(f"out_dtype: float32 or bfloat16, not {dtype}")
    return dtype


# (the pointer of torch's current stream, without the object around it)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_entries = {}


def _call(name, device, *args):
    """The library's call `name` on the device's current stream."""
    entry = _entries.get(name)
    if entry is None:
        entry = _entries[name] = getattr(lib(), name)
    index = device.index
    if index == _current_device():
        rc = entry(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = entry(*args, _raw_stream(index))
    if rc:
        _check(rc, name)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _u32_ok(name, value):
    """value, which the library takes in 32 bits (ctypes would drop the others)."""
    if not 0 <= value < 1 << 32:
        raise GevoError(f"{name}: {value} does not fit 32 bits")
    return value


# Numbers of the caller's as plain ones, read at the call: a tensor or an array
# of one value can change, and would be kept by its identity below.
def _index(name, value):
    try:
        return operator.index(value)
    except (TypeError, ValueError, RuntimeError):
        raise GevoError(f"{name}: an integer, not {value!r}") from None


def _number(name, value):
    try:
        return ctypes.c_float(value).value + 0.0     # (-0 and 0 are one key)
    except (TypeError, ValueError, RuntimeError, OverflowError):
        raise GevoError(f"{name}: a number, not {value!r}") from None


# The configurations of calls, by their values, which are plain numbers: a program
# repeats a few, and the library reads them during the call alone.
def _config(cls):
    def make(*values):
        for (name, kind), value in zip(cls._fields_[1:], values):
            if kind is _u32:
                _u32_ok(name, value)
        return ctypes.byref(cls(GEVO_ABI_VERSION, *values))
    return functools.lru_cache(maxsize=1024)(make)


_route_cfg, _expert_cfg = _config(RouteConfig), _config(ExpertConfig)
_combine_cfg, _mx4_cfg = _config(CombineConfig), _config(Mx4Config)


@functools.lru_cache(maxsize=1024)
def _plan_bytes(slots, n_experts):
    nbytes = ctypes.c_size_t()
    _u32_ok("n_experts", n_experts)
    _check(lib().gevo_route_plan_bytes(slots, n_experts, ctypes.byref(nbytes)), "gevo_route_plan_bytes")
    return nbytes.value


class RoutePlan:
    """A routing's slots sorted by expert: order [T k], pos [T][k] and offsets
    [E + 1], int32 (gevo_route_plan)."""

    __slots__ = ("order", "pos", "offsets")

    def __init__(self, order, pos, offsets):
        if not (isinstance(pos, torch.Tensor) and pos.is_cuda and pos.dim() == 2):
            raise GevoError("pos: a tensor [T][k] on the GPU")
        if not (isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.numel() >= 2):
            raise GevoError("offsets: a tensor [E + 1]")
        self.pos = _flat(pos, "pos", torch.int32, pos.shape, pos.device)
        self.order = _flat(order, "order", torch.int32, (pos.numel(),), pos.device)
        self.offsets = _flat(offsets, "offsets", torch.int32, offsets.shape, pos.device)

    @property
    def n_experts(self) -> int:
        return self.offsets.numel() - 1


def _plan_of(plan, device):
    if not (isinstance(plan, RoutePlan) and plan.pos.device == device):
        raise GevoError(f"plan: a RoutePlan on {device}")
    return plan


def _route_config(logits, k, score, groups, top_groups, group_top, renorm, scale):
    if not isinstance(score, str) or score not in SCORES:
        raise GevoError(f"score: one of {sorted(SCORES)}, not {score!r}")
    if not type(k) is type(groups) is type(top_groups) is type(group_top) is int:
        k, groups = _index("top_k", k), _index("groups", groups)
        top_groups, group_top = _index("top_groups", top_groups), _index("group_top", group_top)
    if min(k, groups, top_groups, group_top) < 1:
        raise GevoError("top_k, groups, top_groups and group_top: at least 1")
    T, E = logits.shape
    if k > E:
        raise GevoError(f"top_k: at most the {E} experts, not {k}")
    scale = scale + 0.0 if type(scale) is float else _number("scale", scale)
    return _route_cfg(E, k, T, DTYPES[logits.dtype], SCORES[score], _stride(logits) if T > 1 else E, groups,
                      top_groups, group_top, 1 if renorm else 0, scale)


def route(logits, top_k, *, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """weights [T][k] float32 and ids [T][k] int32 of each row's k experts of
    logits [T][E] (gevo_route)."""
    logits = _rows(logits, "logits")
    dev = logits.device
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, logits.shape[1:], dev)
    if logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]:
        logits = logits.contiguous()                 # rows that overlap (expanded)
    if type(top_k) is not int:
        top_k = _index("top_k", top_k)
    cfg = _route_config(logits, top_k, score, groups, top_groups, group_top, renorm, scale)
    T = logits.shape[0]
    weights, ids = _new_rows(T, top_k, torch.float32, dev), _new_rows(T, top_k, torch.int32, dev)
    _call("gevo_route", dev, cfg, logits.data_ptr(), _ptr(bias), weights.data_ptr(), ids.data_ptr())
    return weights, ids


def route_backward(logits, ids, dweights, *, score="softmax", renorm=True, scale=1.0):
    """Gradient with respect to the logits, in their type, of route's weights
    with gradient dweights [T][k] and choice ids (gevo_route_backward)."""
    logits = _rows(logits, "logits")
    dev = logits.device
    if not (isinstance(ids, torch.Tensor) and ids.dim() == 2):
        raise GevoError("ids: a tensor [T][k]")
    shape = (logits.shape[0], ids.shape[1])
    ids = _flat(ids, "ids", torch.int32, shape, dev)
    dweights = _flat(dweights, "dweights", torch.float32, shape, dev)
    if shape[0] > 1 and logits.stride(0) < logits.shape[1]:
        logits = logits.contiguous()
    cfg = _route_config(logits, shape[1], score, 1, 1, 1, renorm, scale)
    out = _new_rows(*logits.shape, logits.dtype, dev)
    _call("gevo_route_backward", dev, cfg, logits.data_ptr(), ids.data_ptr(), dweights.data_ptr(), out.data_ptr())
    return out


def route_plan(ids, n_experts) -> RoutePlan:
    """The slots of ids [T][k] sorted by expert (gevo_route_plan)."""
    if not (isinstance(ids, torch.Tensor) and ids.is_cuda and ids.dim() == 2):
        raise GevoError("ids: a tensor [T][k] on the GPU")
    if type(n_experts) is not int:
        n_experts = _index("n_experts", n_experts)
    if n_experts < 1:
        raise GevoError("n_experts: at least 1")
    dev = ids.device
    ids = _flat(ids, "ids", torch.int32, ids.shape, dev)
    n = ids.numel()
    nbytes = _plan_bytes(n, n_experts)
    ws = _new_flat(nbytes, torch.uint8, dev) if nbytes else None
    plan = RoutePlan.__new__(RoutePlan)
    plan.order = _new_flat(n, torch.int32, dev)
    plan.pos = _new_rows(*ids.shape, torch.int32, dev)
    plan.offsets = _new_flat(n_experts + 1, torch.int32, dev)
    _call("gevo_route_plan", dev, n, n_experts, ids.data_ptr(), _ptr(ws), nbytes, plan.order.data_ptr(),
          plan.pos.data_ptr(), plan.offsets.data_ptr())
    return plan


def _expert_setup(x, w, plan, sorted_rows, y_stride, relu, out_dtype):
    w = _rows(w, "w", 3)
    dev = x.device
    _plan_of(plan, dev)
    if w.device != dev or w.dtype != x.dtype:
        raise GevoError(f"w: {x.dtype} on {dev}")
    (T, k), (E, N, K) = plan.pos.shape, w.shape
    if E != plan.n_experts:
        raise GevoError(f"w: {plan.n_experts} experts as the plan has, not {E}")
    rows = T * k if sorted_rows else T
    if x.shape != (rows, K):
        raise GevoError(f"x: shape {(rows, K)}, not {tuple(x.shape)}")
    if (N > 1 and w.stride(1) < K) or (E > 1 and w.stride(0) < (N - 1) * w.stride(1) + K):
        w = w.contiguous()                           # overlapping or transposed matrices
    if rows > 1 and x.stride(0) < K:
        x = x.contiguous()
    wn = w.stride(1) if N > 1 else K
    we = w.stride(0) if E > 1 else (N - 1) * wn + K
    cfg = _expert_cfg(DTYPES[x.dtype], DTYPES[out_dtype], E, k, N, K, T, _stride(x), we, wn, y_stride or N,
                      1 if sorted_rows else 0, 1 if relu else 0)
    return x, w, cfg, dev


def expert_forward(x, w, plan, bias=None, *, relu=False, sorted_rows=False, out_dtype=None):
    """Rows [T k][N], sorted by expert: act(x[row] w[e]^T + bias[e]) with w
    [E][N][K], bias [E][N] float32 (gevo_expert_forward).  x is [T][K], or with
    sorted_rows the sorted rows of a layer before, [T k][K].  Rows of slots
    without an expert (from plan.offsets[-1] on) hold nothing."""
    x = _rows(x, "x")
    out_dtype = _out_dtype(out_dtype, x.dtype)
    x, w, cfg, dev = _expert_setup(x, w, plan, sorted_rows, 0, relu, out_dtype)
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, w.shape[:2], dev)
    out = _new_rows(plan.pos.numel(), w.shape[1], out_dtype, dev)
    _call("gevo_expert_forward", dev, cfg, x.data_ptr(), w.data_ptr(), _ptr(bias), plan.order.data_ptr(),
          plan.offsets.data_ptr(), out.data_ptr())
    return out


def expert_backward(dy, x, w, plan, *, sorted_rows=False, relu_input=False, need_dx=True, need_dw=True):
    """(dx [T k][K] in x's type, dw [E][N][K] float32, db [E][N] float32) of the
    product with gradient dy [T k][N] (gevo_expert_backward); None where not
    needed.  relu_input: x is a ReLU's output, and dx the gradient before it.
    expert_combine(dx, plan) adds the sorted rows up to a gradient of x [T][K]."""
    dy, x = _rows(dy, "dy"), _rows(x, "x")
    n = plan.pos.numel() if isinstance(plan, RoutePlan) else 0
    if n > 1 and dy.stride(0) < dy.shape[1]:
        dy = dy.contiguous()
    x, w, cfg, dev = _expert_setup(x, w, plan, sorted_rows, _stride(dy), relu_input, dy.dtype)
    if dy.dtype != x.dtype or dy.device != dev or dy.shape != (n, w.shape[1]):
        raise GevoError(f"dy: {x.dtype} of shape {(n, w.shape[1])} on {dev}, not {dy.dtype} of {tuple(dy.shape)}")
    (E, N, K), dw, db = w.shape, None, None
    dx = _new_rows(n, K, x.dtype, dev) if need_dx else None
    if need_dw:
        dw, db = _new((E, N, K), torch.float32, dev), _new_rows(E, N, torch.float32, dev)
    _call("gevo_expert_backward", dev, cfg, _ptr(dy), _ptr(x), _ptr(w), _ptr(plan.order),
          _ptr(plan.offsets), _ptr(dx), _ptr(dw), _ptr(db))
    return dx, dw, db


def _combine_setup(rows, plan, weights):
    rows = _rows(rows, "rows")
    dev = rows.device
    _plan_of(plan, dev)
    n = plan.pos.numel()
    if rows.shape[0] != n:
        raise GevoError(f"rows: {n} of them, not {rows.shape[0]}")
    if n > 1 and rows.stride(0) < rows.shape[1]:
        rows = rows.contiguous()
    if weights is not None:
        weights = _flat(weights, "weights", torch.float32, plan.pos.shape, dev)
    return rows, weights, dev


def expert_combine(rows, plan, weights=None, *, out_dtype=None):
    """y [T][N]: each row's slots of the sorted rows, added up with weights
    [T][k] (None: ones) in float32 and rounded once (gevo_expert_combine)."""
    rows, weights, dev = _combine_setup(rows, plan, weights)
    out_dtype = _out_dtype(out_dtype, rows.dtype)
    (T, k), N = plan.pos.shape, rows.shape[1]
    cfg = _combine_cfg(DTYPES[rows.dtype], DTYPES[out_dtype], k, N, T, _stride(rows), N)
    y = _new_rows(T, N, out_dtype, dev)
    _call("gevo_expert_combine", dev, cfg, rows.data_ptr(), plan.pos.data_ptr(), _ptr(weights), y.data_ptr())
    return y


def expert_combine_backward(dy, rows, plan, weights=None):
    """(drows [T k][N] sorted, dweights [T][k] float32) of expert_combine with
    gradient dy [T][N], in the rows' type (gevo_expert_combine_backward)."""
    rows, weights, dev = _combine_setup(rows, plan, weights)
    dy = _rows(dy, "dy")
    (T, k), N = plan.pos.shape, rows.shape[1]
    if dy.dtype != rows.dtype or dy.device != dev or dy.shape != (T, N):
        raise GevoError(f"dy: {rows.dtype} of shape {(T, N)} on {dev}, not {dy.dtype} of {tuple(dy.shape)}")
    if T > 1 and dy.stride(0) < N:
        dy = dy.contiguous()
    dtype = DTYPES[rows.dtype]
    cfg = _combine_cfg(dtype, dtype, k, N, T, _stride(rows), _stride(dy))
    drows, dweights = _new_rows(T * k, N, rows.dtype, dev), _new_rows(T, k, torch.float32, dev)
    _call("gevo_expert_combine_backward", dev, cfg, dy.data_ptr(), rows.data_ptr(), plan.pos.data_ptr(),
          _ptr(weights), drows.data_ptr(), dweights.data_ptr())
    return drows, dweights


class Mx4:
    """Rows in microscaled 4-bit floating point: codes [..., rows, Kp / 2] and
    scales [..., rows, Kp / 32] (uint8, Kp = K rounded up to 128; gevo.h states
    the layout) of `k` values a row."""

    __slots__ = ("codes", "scales", "k")

    def __init__(self, codes, scales, k):
        k = _index("k", k)
        if not (1 <= k < 1 << 32 and isinstance(codes, torch.Tensor) and codes.is_cuda and codes.dim() >= 2):
            raise GevoError("codes: a tensor [..., rows, Kp / 2] on the GPU")
        kp = (k + 127) // 128 * 128
        if codes.shape[-1] != kp // 2:
            raise GevoError(f"codes: rows of {kp // 2} bytes for {k} values, not {codes.shape[-1]}")
        self.codes = _flat(codes, "codes", torch.uint8, codes.shape, codes.device)
        self.scales = _flat(scales, "scales", torch.uint8, (*codes.shape[:-1], kp // 32), codes.device)
        self.k = k

    @property
    def shape(self):
        return (*self.codes.shape[:-1], self.k)

    def dequantize(self, dtype=torch.float32):
        """The values as a tensor of self.shape (gevo_mx4_dequantize)."""
        dtype = _out_dtype(dtype, torch.float32)
        k, dev = self.k, self.codes.device
        out = _new(self.shape, dtype, dev)
        _call("gevo_mx4_dequantize", dev, DTYPES[dtype], out.numel() // k, k, self.codes.data_ptr(),
              self.scales.data_ptr(), out.data_ptr(), k)
        return out


def mx4_quantize(x) -> Mx4:
    """The rows of x [..., rows, K] in 4 bits, 32 values of a row to a scale
    (gevo_mx4_quantize)."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() >= 2 and x.shape[-1] >= 1):
        raise GevoError("x: a tensor [..., rows, K] on the GPU")
    if x.dtype not in DTYPES:
        raise GevoError(f"x: float32 or bfloat16, not {x.dtype}")
    k = _u32_ok("K", x.shape[-1])
    if x.dim() > 2 or (k > 1 and x.stride(-1) != 1) or (x.shape[0] > 1 and x.stride(0) < k):
        x = x.contiguous()
    kp = (k + 127) // 128 * 128
    lead, dev = x.shape[:-1], x.device
    q = Mx4.__new__(Mx4)
    q.codes, q.scales = _new((*lead, kp // 2), torch.uint8, dev), _new((*lead, kp // 32), torch.uint8, dev)
    q.k = k
    _call("gevo_mx4_quantize", dev, DTYPES[x.dtype], x.numel() // k, k, x.data_ptr(),
          k if x.dim() > 2 else _stride(x), q.codes.data_ptr(), q.scales.data_ptr())
    return q


def mx4_matmul(a, b, *, bias=None, relu=False, plan=None, sorted_rows=False, out_dtype=torch.float32):
    """act(a b_p^T + bias[p]) of 4-bit rows and P 4-bit matrices b [P][N][K]
    (gevo_mx4_matmul).  Without a plan [P][M][N], a being [M][K] for every p or
    [P][M][K]; with one the sorted rows [T k][N], a being [T][K] or, with
    sorted_rows, [T k][K]."""
    if not (isinstance(a, Mx4) and isinstance(b, Mx4)):
        raise GevoError("a, b: Mx4")
    ac, bc = a.codes, b.codes
    dev = ac.device
    out_dtype = _out_dtype(out_dtype, torch.float32)
    if bc.dim() != 3 or bc.device != dev or a.k != b.k:
        raise GevoError(f"b: [P][N][{a.k}] on {dev}, not {b.shape}")
    P, N, K = bc.shape[0], bc.shape[1], b.k
    if P < 1 or N < 1:
        raise GevoError(f"b: [P][N][K], not {b.shape}")
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, (P, N), dev)
    k, order, offsets, each = 1, None, None, ac.dim() == 3
    if plan is None:
        if not (ac.dim() == 2 or (each and ac.shape[0] == P)):
            raise GevoError(f"a: [M][K] or [{P}][M][K], not {a.shape}")
        if sorted_rows:
            raise GevoError("sorted_rows: with a plan")
        M = ac.shape[-2]
        shape = (P, M, N)
    else:
        _plan_of(plan, dev)
        if plan.n_experts != P:
            raise GevoError(f"b: {plan.n_experts} experts as the plan has, not {P}")
        (M, k), order, offsets = plan.pos.shape, plan.order.data_ptr(), plan.offsets.data_ptr()
        if a.shape != (M * k if sorted_rows else M, K):
            raise GevoError(f"a: shape {(M * k if sorted_rows else M, K)}, not {a.shape}")
        shape = (M * k, N)
    out = _new(shape, out_dtype, dev)
    cfg = _mx4_cfg(DTYPES[out_dtype], P, N, K, M, 1 if each else 0, k, 1 if sorted_rows else 0, 1 if relu else 0)
    _call("gevo_mx4_matmul", dev, cfg, ac.data_ptr(), a.scales.data_ptr(), bc.data_ptr(), b.scales.data_ptr(),
          _ptr(bias), order, offsets, out.data_ptr())
    return out
