"""Operators on device tensors: rows routed to experts, and layers in 4 bits.

A population's variants can serve together, each row going to the few of them
that a router chooses (mixture.py does so); the same calls run any experts held
as one tensor of weight matrices.  This module marshals arguments of the
library's calls (include/gevo.h, which states the mathematics): outputs come
from torch's allocator, work goes to the tensors' device on torch's current
stream, so calls can be captured into a graph.  Tensors are float32 or
bfloat16; rows may be strided, a last dimension that is not contiguous is
copied first.  A wrong argument raises GevoError and launches nothing.

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


def _need(ok, what):
    if not ok:
        raise GevoError(what)


def _rows(t, name, dims=2):
    """t with dims dimensions, of a type that the kernels take, its last one contiguous."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda, f"{name}: a tensor on the GPU")
    _need(t.dtype in DTYPES, f"{name}: float32 or bfloat16, not {t.dtype}")
    _need(t.dim() == dims, f"{name}: {dims} dimensions, not {t.dim()}")
    return t if t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


def _flat(t, name, dtype, shape, device):
    """t as a contiguous tensor of one type and shape."""
    _need(isinstance(t, torch.Tensor) and t.device == device, f"{name}: a tensor on {device}")
    _need(t.dtype == dtype and tuple(t.shape) == tuple(shape), f"{name}: {dtype} of shape {tuple(shape)}, not "
          f"{t.dtype} of {tuple(t.shape)}")
    return t if t.is_contiguous() else t.contiguous()


def _stride(t, dim=0):
    """Elements between t's rows; at least a row's length where there is one row or none."""
    return max(t.stride(dim), t.shape[-1]) if t.shape[dim] > 1 else t.shape[-1]


def _out_dtype(dtype, default):
    dtype = default if dtype is None else dtype
    _need(dtype in DTYPES, f"out_dtype: float32 or bfloat16, not {dtype}")
    return dtype


def _call(name, device, *args):
    """The library's call `name` on the device's current stream."""
    fn = getattr(lib(), name)
    if device.index == torch.cuda.current_device():
        rc = fn(*args, torch.cuda.current_stream(device).cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, torch.cuda.current_stream(device).cuda_stream)
    if rc:
        _check(rc, name)


def _ptr(t):
    return None if t is None else t.data_ptr()


class RoutePlan:
    """A routing's slots sorted by expert: order [T k], pos [T][k] and offsets
    [E + 1], int32 (gevo_route_plan)."""

    __slots__ = ("order", "pos", "offsets")

    def __init__(self, order, pos, offsets):
        _need(isinstance(pos, torch.Tensor) and pos.is_cuda and pos.dim() == 2, "pos: a tensor [T][k] on the GPU")
        _need(isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.numel() >= 2,
              "offsets: a tensor [E + 1]")
        self.pos = _flat(pos, "pos", torch.int32, pos.shape, pos.device)
        self.order = _flat(order, "order", torch.int32, (pos.numel(),), pos.device)
        self.offsets = _flat(offsets, "offsets", torch.int32, offsets.shape, pos.device)

    @property
    def n_experts(self) -> int:
        return self.offsets.numel() - 1


def _route_config(logits, k, score, groups, top_groups, group_top, renorm, scale):
    _need(score in SCORES, f"score: one of {sorted(SCORES)}, not {score!r}")
    T, E = logits.shape
    _need(min(k, groups, top_groups, group_top) >= 1, "top_k, groups, top_groups and group_top: at least 1")
    return RouteConfig(GEVO_ABI_VERSION, E, k, T, DTYPES[logits.dtype], SCORES[score], _stride(logits), groups,
                       top_groups, group_top, 1 if renorm else 0, scale)


def route(logits, top_k, *, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """weights [T][k] float32 and ids [T][k] int32 of each row's k experts of
    logits [T][E] (gevo_route)."""
    logits = _rows(logits, "logits")
    dev = logits.device
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, logits.shape[1:], dev)
    cfg = _route_config(logits, top_k, score, groups, top_groups, group_top, renorm, scale)
    weights = torch.empty((logits.shape[0], top_k), dtype=torch.float32, device=dev)
    ids = torch.empty((logits.shape[0], top_k), dtype=torch.int32, device=dev)
    _call("gevo_route", dev, ctypes.byref(cfg), _ptr(logits), _ptr(bias), _ptr(weights), _ptr(ids))
    return weights, ids


def route_backward(logits, ids, dweights, *, score="softmax", renorm=True, scale=1.0):
    """Gradient with respect to the logits, in their type, of route's weights
    with gradient dweights [T][k] and choice ids (gevo_route_backward)."""
    logits = _rows(logits, "logits")
    dev = logits.device
    _need(isinstance(ids, torch.Tensor) and ids.dim() == 2, "ids: a tensor [T][k]")
    shape = (logits.shape[0], ids.shape[1])
    ids = _flat(ids, "ids", torch.int32, shape, dev)
    dweights = _flat(dweights, "dweights", torch.float32, shape, dev)
    cfg = _route_config(logits, shape[1], score, 1, 1, 1, renorm, scale)
    out = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    _call("gevo_route_backward", dev, ctypes.byref(cfg), _ptr(logits), _ptr(ids), _ptr(dweights), _ptr(out))
    return out


def route_plan(ids, n_experts) -> RoutePlan:
    """The slots of ids [T][k] sorted by expert (gevo_route_plan)."""
    _need(isinstance(ids, torch.Tensor) and ids.is_cuda and ids.dim() == 2, "ids: a tensor [T][k] on the GPU")
    _need(n_experts >= 1, "n_experts: at least 1")
    dev = ids.device
    ids = _flat(ids, "ids", torch.int32, ids.shape, dev)
    n = ids.numel()
    nbytes = ctypes.c_size_t()
    _check(lib().gevo_route_plan_bytes(n, n_experts, ctypes.byref(nbytes)), "gevo_route_plan_bytes")
    ws = torch.empty(nbytes.value, dtype=torch.uint8, device=dev)
    order = torch.empty(n, dtype=torch.int32, device=dev)
    pos = torch.empty(ids.shape, dtype=torch.int32, device=dev)
    offsets = torch.empty(n_experts + 1, dtype=torch.int32, device=dev)
    _call("gevo_route_plan", dev, n, n_experts, _ptr(ids), _ptr(ws), nbytes.value, _ptr(order), _ptr(pos),
          _ptr(offsets))
    return RoutePlan(order, pos, offsets)


def _expert_setup(x, w, plan, sorted_rows, y_stride, relu, out_dtype):
    x, w = _rows(x, "x"), _rows(w, "w", 3)
    dev = x.device
    _need(isinstance(plan, RoutePlan) and plan.pos.device == dev, f"plan: a RoutePlan on {dev}")
    _need(w.device == dev and w.dtype == x.dtype, f"w: {x.dtype} on {dev}")
    (T, k), (E, N, K) = plan.pos.shape, w.shape
    _need(E == plan.n_experts, f"w: {plan.n_experts} experts as the plan has, not {E}")
    rows = T * k if sorted_rows else T
    _need(tuple(x.shape) == (rows, K), f"x: shape {(rows, K)}, not {tuple(x.shape)}")
    if (N > 1 and w.stride(1) < K) or (E > 1 and w.stride(0) < (N - 1) * w.stride(1) + K):
        w = w.contiguous()                           # overlapping or transposed matrices
    if rows > 1 and x.stride(0) < K:
        x = x.contiguous()
    wn = w.stride(1) if N > 1 else K
    we = w.stride(0) if E > 1 else (N - 1) * wn + K
    cfg = ExpertConfig(GEVO_ABI_VERSION, DTYPES[x.dtype], DTYPES[out_dtype or x.dtype], E, k, N, K, T, _stride(x), we,
                       wn, y_stride or N, 1 if sorted_rows else 0, 1 if relu else 0)
    return x, w, cfg, dev


def expert_forward(x, w, plan, bias=None, *, relu=False, sorted_rows=False, out_dtype=None):
    """Rows [T k][N], sorted by expert: act(x[row] w[e]^T + bias[e]) with w
    [E][N][K], bias [E][N] float32 (gevo_expert_forward).  x is [T][K], or with
    sorted_rows the sorted rows of a layer before, [T k][K].  Rows of slots
    without an expert (from plan.offsets[-1] on) hold nothing."""
    out_dtype = _out_dtype(out_dtype, x.dtype if isinstance(x, torch.Tensor) else None)
    x, w, cfg, dev = _expert_setup(x, w, plan, sorted_rows, 0, relu, out_dtype)
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, w.shape[:2], dev)
    out = torch.empty((plan.pos.numel(), w.shape[1]), dtype=out_dtype, device=dev)
    _call("gevo_expert_forward", dev, ctypes.byref(cfg), _ptr(x), _ptr(w), _ptr(bias), _ptr(plan.order),
          _ptr(plan.offsets), _ptr(out))
    return out


def expert_backward(dy, x, w, plan, *, sorted_rows=False, relu_input=False, need_dx=True, need_dw=True):
    """(dx [T k][K] in x's type, dw [E][N][K] float32, db [E][N] float32) of the
    product with gradient dy [T k][N] (gevo_expert_backward); None where not
    needed.  relu_input: x is a ReLU's output, and dx the gradient before it.
    expert_combine(dx, plan) adds the sorted rows up to a gradient of x [T][K]."""
    dy = _rows(dy, "dy")
    n = plan.pos.numel() if isinstance(plan, RoutePlan) else 0
    if n > 1 and dy.stride(0) < dy.shape[1]:
        dy = dy.contiguous()
    x, w, cfg, dev = _expert_setup(x, w, plan, sorted_rows, _stride(dy), relu_input, None)
    _need(dy.dtype == x.dtype and dy.device == dev and tuple(dy.shape) == (n, w.shape[1]),
          f"dy: {x.dtype} of shape {(n, w.shape[1])} on {dev}, not {dy.dtype} of {tuple(dy.shape)}")
    dx = torch.empty((n, w.shape[2]), dtype=x.dtype, device=dev) if need_dx else None
    dw = torch.empty(w.shape, dtype=torch.float32, device=dev) if need_dw else None
    db = torch.empty(w.shape[:2], dtype=torch.float32, device=dev) if need_dw else None
    _call("gevo_expert_backward", dev, ctypes.byref(cfg), _ptr(dy), _ptr(x), _ptr(w), _ptr(plan.order),
          _ptr(plan.offsets), _ptr(dx), _ptr(dw), _ptr(db))
    return dx, dw, db


def _combine_setup(rows, plan, weights):
    rows = _rows(rows, "rows")
    dev = rows.device
    _need(isinstance(plan, RoutePlan) and plan.pos.device == dev, f"plan: a RoutePlan on {dev}")
    _need(rows.shape[0] == plan.pos.numel(), f"rows: {plan.pos.numel()} of them, not {rows.shape[0]}")
    if rows.shape[0] > 1 and rows.stride(0) < rows.shape[1]:
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
    cfg = CombineConfig(GEVO_ABI_VERSION, DTYPES[rows.dtype], DTYPES[out_dtype], k, N, T, _stride(rows), N)
    y = torch.empty((T, N), dtype=out_dtype, device=dev)
    _call("gevo_expert_combine", dev, ctypes.byref(cfg), _ptr(rows), _ptr(plan.pos), _ptr(weights), _ptr(y))
    return y


def expert_combine_backward(dy, rows, plan, weights=None):
    """(drows [T k][N] sorted, dweights [T][k] float32) of expert_combine with
    gradient dy [T][N], in the rows' type (gevo_expert_combine_backward)."""
    rows, weights, dev = _combine_setup(rows, plan, weights)
    dy = _rows(dy, "dy")
    (T, k), N = plan.pos.shape, rows.shape[1]
    _need(dy.dtype == rows.dtype and dy.device == dev and tuple(dy.shape) == (T, N),
          f"dy: {rows.dtype} of shape {(T, N)} on {dev}, not {dy.dtype} of {tuple(dy.shape)}")
    if T > 1 and 0 < dy.stride(0) < N:
        dy = dy.contiguous()
    if T > 1 and dy.stride(0) == 0:                  # one gradient for every row (expanded)
        dy = dy.contiguous()
    cfg = CombineConfig(GEVO_ABI_VERSION, DTYPES[rows.dtype], DTYPES[rows.dtype], k, N, T, _stride(rows), _stride(dy))
    drows = torch.empty((T * k, N), dtype=rows.dtype, device=dev)
    dweights = torch.empty((T, k), dtype=torch.float32, device=dev)
    _call("gevo_expert_combine_backward", dev, ctypes.byref(cfg), _ptr(dy), _ptr(rows), _ptr(plan.pos),
          _ptr(weights), _ptr(drows), _ptr(dweights))
    return drows, dweights


class Mx4:
    """Rows in microscaled 4-bit floating point: codes [..., rows, Kp / 2] and
    scales [..., rows, Kp / 32] (uint8, Kp = K rounded up to 128; gevo.h states
    the layout) of `k` values a row."""

    __slots__ = ("codes", "scales", "k")

    def __init__(self, codes, scales, k):
        kp = (k + 127) // 128 * 128
        _need(k >= 1 and isinstance(codes, torch.Tensor) and codes.is_cuda and codes.dim() >= 2,
              "codes: a tensor [..., rows, Kp / 2] on the GPU")
        _need(codes.shape[-1] == kp // 2, f"codes: rows of {kp // 2} bytes for {k} values, not {codes.shape[-1]}")
        self.codes = _flat(codes, "codes", torch.uint8, codes.shape, codes.device)
        self.scales = _flat(scales, "scales", torch.uint8, (*codes.shape[:-1], kp // 32), codes.device)
        self.k = k

    @property
    def shape(self):
        return (*self.codes.shape[:-1], self.k)

    def dequantize(self, dtype=torch.float32):
        """The values as a tensor of self.shape (gevo_mx4_dequantize)."""
        dtype = _out_dtype(dtype, torch.float32)
        out = torch.empty(self.shape, dtype=dtype, device=self.codes.device)
        _call("gevo_mx4_dequantize", self.codes.device, DTYPES[dtype], out.numel() // self.k, self.k,
              _ptr(self.codes), _ptr(self.scales), _ptr(out), self.k)
        return out


def mx4_quantize(x) -> Mx4:
    """The rows of x [..., rows, K] in 4 bits, 32 values of a row to a scale
    (gevo_mx4_quantize)."""
    _need(isinstance(x, torch.Tensor) and x.is_cuda and x.dim() >= 2 and x.shape[-1] >= 1,
          "x: a tensor [..., rows, K] on the GPU")
    _need(x.dtype in DTYPES, f"x: float32 or bfloat16, not {x.dtype}")
    k = x.shape[-1]
    if x.dim() > 2 or (k > 1 and x.stride(-1) != 1) or (x.shape[0] > 1 and x.stride(0) < k):
        x = x.contiguous()
    rows = x.numel() // k
    kp = (k + 127) // 128 * 128
    stride = k if x.dim() > 2 else _stride(x)
    codes = torch.empty((*x.shape[:-1], kp // 2), dtype=torch.uint8, device=x.device)
    scales = torch.empty((*x.shape[:-1], kp // 32), dtype=torch.uint8, device=x.device)
    _call("gevo_mx4_quantize", x.device, DTYPES[x.dtype], rows, k, _ptr(x), stride, _ptr(codes), _ptr(scales))
    return Mx4(codes, scales, k)


def mx4_matmul(a, b, *, bias=None, relu=False, plan=None, sorted_rows=False, out_dtype=torch.float32):
    """act(a b_p^T + bias[p]) of 4-bit rows and P 4-bit matrices b [P][N][K]
    (gevo_mx4_matmul).  Without a plan [P][M][N], a being [M][K] for every p or
    [P][M][K]; with one the sorted rows [T k][N], a being [T][K] or, with
    sorted_rows, [T k][K]."""
    _need(isinstance(a, Mx4) and isinstance(b, Mx4), "a, b: Mx4")
    dev = a.codes.device
    out_dtype = _out_dtype(out_dtype, torch.float32)
    _need(len(b.shape) == 3 and b.codes.device == dev and a.k == b.k, f"b: [P][N][{a.k}] on {dev}, not {b.shape}")
    P, N, K = b.shape
    if bias is not None:
        bias = _flat(bias, "bias", torch.float32, (P, N), dev)
    k, order, offsets, each = 1, None, None, len(a.shape) == 3
    if plan is None:
        _need(len(a.shape) == 2 or a.shape[0] == P, f"a: [M][K] or [{P}][M][K], not {a.shape}")
        _need(not sorted_rows, "sorted_rows: with a plan")
        M = a.shape[-2]
        shape = (P, M, N)
    else:
        _need(isinstance(plan, RoutePlan) and plan.pos.device == dev, f"plan: a RoutePlan on {dev}")
        _need(plan.n_experts == P, f"b: {plan.n_experts} experts as the plan has, not {P}")
        (M, k), order, offsets = plan.pos.shape, plan.order, plan.offsets
        rows = M * k if sorted_rows else M
        _need(tuple(a.shape) == (rows, K), f"a: shape {(rows, K)}, not {a.shape}")
        shape = (M * k, N)
    out = torch.empty(shape, dtype=out_dtype, device=dev)
    cfg = Mx4Config(GEVO_ABI_VERSION, DTYPES[out_dtype], P, N, K, M, 1 if each else 0, k, 1 if sorted_rows else 0,
                    1 if relu else 0)
    _call("gevo_mx4_matmul", dev, ctypes.byref(cfg), _ptr(a.codes), _ptr(a.scales), _ptr(b.codes), _ptr(b.scales),
          _ptr(bias), _ptr(order), _ptr(offsets), _ptr(out))
    return out
