"""The routed and 4-bit operators against their 64-bit definitions
(oracle/operators.py), at the sizes, masks, strides and orders where they can go
wrong.

Tolerances.  A sum of n products in binary32 in any order, each addition off by
at most half a step (2^-24) of a partial sum, is off by at most (n + 2) 2^-24
times the sum of the terms' magnitudes; matrix instructions may drop what lies
below a step instead of rounding, so a whole step (2^-23) is allowed.  An
output in bf16 is half a step (2^-8 relative) further.  Scores and weights
(exp, sums of E terms, a quotient) get 32 steps of 2^-24 relative plus that
sum's."""
import zlib

import numpy as np
import pytest

from oracle import operators as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2310_10211_amd as g                     # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _np(t):
    return t.detach().double().cpu().numpy()


def _rng(*seed):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(seed).encode()))


def _randn(gen, *shape, dtype="f32", by=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * by).to(DT[dtype])


def _close(got, want, mag, n, dtype, what=""):
    tol = (n + 2) * 2.0 ** -23 * mag + HALF[dtype] * np.abs(want) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - want) / tol)))


# --------------------------------------------------------------------- route
ROUTES = [
    # T, E, k, dtype, options
    (1, 1, 1, "f32", {}), (1, 64, 6, "f32", {}), (5, 3, 3, "bf16", dict(renorm=False)),
    (33, 17, 4, "f32", dict(score="sigmoid")), (70, 64, 16, "bf16", dict(scale=2.5)),
    (65, 65, 2, "f32", dict(renorm=False)), (40, 128, 8, "f32", dict(bias=True)),
    (257, 256, 8, "f32", dict(score="sigmoid", bias=True, groups=8, top_groups=4, group_top=2, scale=2.5)),
    (50, 256, 17, "bf16", dict(bias=True)), (30, 257, 5, "f32", dict(score="sigmoid", renorm=False)),
    (20, 513, 64, "f32", {}), (19, 1024, 4, "bf16", dict(renorm=False)), (9, 2048, 3, "f32", dict(bias=True)),
    (25, 96, 5, "f32", dict(groups=32, top_groups=7)), (25, 96, 3, "bf16", dict(groups=3, top_groups=2, group_top=2)),
    (13, 64, 2, "f32", dict(groups=64, top_groups=5, group_top=2, bias=True)),
    (13, 128, 2, "f32", dict(groups=16, top_groups=1, score="sigmoid", group_top=2)),
]


def _route_case(T, E, k, dtype, how, masked=0.2):
    gen = _rng("route", T, E, k)
    logits = _randn(gen, T, E, dtype=dtype, by=2.0)
    if masked and E > k:
        logits = logits.masked_fill(torch.rand(T, E, generator=gen, device="cuda") < masked, float("-inf"))
    how = dict(how)
    if how.pop("bias", False):
        how["bias"] = _randn(gen, E, by=0.2)
    return logits, how


def _oracle_how(how):
    return {k: _np(v) if isinstance(v, torch.Tensor) else v for k, v in how.items()}


def _check_route(logits, k, how):
    w, ids = g.route(logits, k, **how)
    rw, rids = ref.route(_np(logits), k, **_oracle_how(how))
    assert np.array_equal(ids.cpu().numpy(), rids)
    tol = (32 + logits.shape[1]) * 2.0 ** -24 * np.abs(rw) + 1e-37
    assert np.array_equal(np.isnan(_np(w)), np.isnan(rw))
    d = np.abs(_np(w) - rw)
    assert (d[~np.isnan(rw)] <= tol[~np.isnan(rw)]).all(), np.nanmax(d / tol)
    return w, ids


@pytest.mark.parametrize("T,E,k,dtype,how", ROUTES)
def test_route(T, E, k, dtype, how):
    print(f"[gpu] route {T} {E} {k} {dtype} {how}", flush=True)
    logits, how = _route_case(T, E, k, dtype, how)
    _check_route(logits, k, how)


def test_route_strided_rows():
    gen = _rng("strided")
    wide = _randn(gen, 20, 50)
    _check_route(wide[:, 3:44], 5, {})
    _check_route(wide[::2, :41], 5, dict(score="sigmoid"))
    _check_route(wide.t(), 5, {})                                 # last dimension not contiguous


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,groups", [(16, 4, 1), (256, 4, 8), (300, 17, 4)])
def test_route_rows_with_little_or_nothing_to_choose(score, E, k, groups):
    inf = float("inf")
    logits = torch.zeros(10, E, device="cuda")
    logits[0] = -inf                                              # nothing left
    logits[1] = -inf
    logits[1, E - 1] = -5.0                                       # fewer than k
    logits[2, 3] = float("nan")
    logits[3] = torch.finfo(torch.float32).min                    # the type's lowest value is a logit like others
    logits[4, 1:] = torch.finfo(torch.float32).min
    logits[5, 2] = inf
    logits[6] = 1e30
    logits[7] = -100.0                                            # scores underflow, their ratios do not
    logits[7, 5] = -101.0
    logits[8, :: 2] = -inf
    logits[9] = torch.linspace(-80, 80, E, device="cuda")
    for bias in (None, torch.zeros(E, device="cuda")):
        for renorm in (True, False):
            _check_route(logits, k, dict(score=score, groups=groups, top_groups=max(1, groups // 2), bias=bias,
                                         renorm=renorm))
    bias = torch.zeros(E, device="cuda")
    bias[0], bias[1], bias[2] = -inf, inf, 3.0
    _check_route(logits, k, dict(score=score, bias=bias))
    bias[4] = float("nan")
    w, ids = g.route(logits, k, score=score, bias=bias)
    assert (ids == -1).all() and w.isnan().sum() >= 9 * k


def test_route_orders_keys_closer_than_a_binary32_step():
    """Biases put keys within 1e-9 to 1e-7 of each other: their order is that of
    64-bit scores, for choices and for groups."""
    gen = _rng("near")
    for score in ("softmax", "sigmoid"):
        logits = _randn(gen, 300, 64)
        rows = []
        for t in range(300):
            l = _np(logits[t])
            s = ref.scores(l, score)
            rows.append((0.5 - s).astype(np.float32))             # key = s + bias = 0.5 to the bias's rounding
        for t in range(0, 300, 15):
            how = dict(score=score, bias=torch.tensor(rows[t], device="cuda"))
            _check_route(logits[t:t + 1], 6, how)
            _check_route(logits[t:t + 1], 6, dict(how, groups=8, top_groups=3, group_top=2))
        _check_route(logits, 6, dict(score=score, bias=torch.tensor(rows[0], device="cuda")))
    _check_route(torch.ones(9, 96, device="cuda"), 7, dict(bias=torch.zeros(96, device="cuda")))      # all equal


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 1, 1, "f32"), (37, 33, 4, "f32"), (20, 64, 2, "bf16"), (65, 130, 17, "f32"),
                                         (11, 700, 8, "bf16"), (5, 2048, 64, "f32")])
def test_route_backward(score, renorm, T, E, k, dtype):
    logits, _ = _route_case(T, E, k, dtype, {}, masked=0)
    gen = _rng("back", T, E)
    ids = torch.rand(T, E, generator=gen, device="cuda").topk(k, 1).indices.int()
    if k > 2:
        ids[0, 0] = -1                                            # a slot without an expert
        ids[-1, 1] = ids[-1, 0]                                   # an expert twice
        ids[T // 2] = -1                                          # a row without any
        ids[T // 3, 2] = E                                        # outside
    dw = _randn(gen, T, k)
    how = dict(score=score, renorm=renorm, scale=1.5)
    got = _np(g.route_backward(logits, ids, dw, **how))
    want = ref.route_backward(_np(logits), ids.cpu().numpy(), _np(dw), **how)
    # terms: each gradient times its weight, and the weight times the sum of all of them
    w = np.abs(ref.route_weights(_np(logits), ids.cpu().numpy(), **how))
    mag = (w * np.abs(_np(dw))).sum(1, keepdims=True) + (np.abs(_np(dw)).max(1, keepdims=True) * w).max(1, keepdims=True)
    tol = (64 + E + k) * 2.0 ** -24 * mag + HALF[dtype] * np.abs(want) + 1e-37
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 64), (63, 3, 5), (300, 7, 100), (2048, 1, 2048), (683, 3, 7),
                                   (5000, 2, 33), (3000, 8, 2048), (0, 2, 4)])
def test_route_plan(T, k, E):
    import ctypes
    gen = _rng("plan", T, E)
    ids = torch.randint(-1, E + 1, (T, k), generator=gen, device="cuda", dtype=torch.int32)   # -1 and E: no expert
    if T > 100:
        ids[T // 3: T // 2] = E // 2                              # a run of one expert
    order, pos, off = ref.plan(ids.cpu().numpy(), E)
    p = g.route_plan(ids, E)
    assert np.array_equal(p.offsets.cpu().numpy(), off)
    assert np.array_equal(p.pos.cpu().numpy(), pos)
    assert np.array_equal(p.order.cpu().numpy()[:len(order)], order)
    # entries behind the last filled slot are left as they were
    n = ctypes.c_size_t()
    g.lib().gevo_route_plan_bytes(T * k, E, ctypes.byref(n))
    ws, o = torch.empty(n.value, dtype=torch.uint8, device="cuda"), torch.full((T * k,), 77, dtype=torch.int32, device="cuda")
    pos2, off2 = torch.empty_like(ids), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    assert g.lib().gevo_route_plan(T * k, E, ids.data_ptr(), ws.data_ptr(), n.value, o.data_ptr(), pos2.data_ptr(),
                                   off2.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert (o[len(order):] == 77).all() and torch.equal(pos2, p.pos)


# ------------------------------------------------------------------- experts
def _routed(T, k, E, seed, some_missing=True, only=None):
    gen = _rng("routed", T, k, E, seed)
    ids = torch.randint(0, E, (T, k), generator=gen, device="cuda", dtype=torch.int32)
    if only is not None:
        ids[:] = torch.tensor(only, device="cuda", dtype=torch.int32)[ids.long() % len(only)]
    if some_missing and T * k > 2:
        ids.view(-1)[1] = -1
    return gen, ids, g.route_plan(ids, E)


EXPERTS = [
    # T, k, E, N, K, dtype, out, only (experts with rows)
    (1, 1, 1, 1, 1, "f32", "f32", None), (1, 8, 64, 100, 72, "bf16", "bf16", None), (3, 2, 5, 17, 33, "bf16", "f32", None),
    (2, 2, 3, 40, 130, "f32", "bf16", None), (40, 2, 3, 70, 64, "bf16", "f32", None),
    (300, 2, 3, 257, 96, "bf16", "bf16", None), (300, 2, 4, 260, 50, "f32", "f32", None),
    (500, 1, 2, 300, 137, "bf16", "f32", None), (150, 3, 70, 24, 40, "bf16", "f32", None),
    (400, 4, 130, 33, 16, "f32", "f32", [5, 129]), (260, 2, 9, 512, 256, "bf16", "bf16", [3]),
    (500, 1, 2, 302, 138, "bf16", "bf16", None), (300, 2, 3, 34, 70, "bf16", "f32", None), (400, 2, 3, 6, 10, "bf16", "f32", None),
    (300, 1, 2, 3, 2, "f32", "f32", None), (260, 1, 1, 65, 129, "bf16", "f32", None),
    (1500, 2, 4, 10, 784, "f32", "f32", None), (700, 2, 6, 64, 1000, "bf16", "f32", [0, 5]),
]


@pytest.mark.parametrize("T,k,E,N,K,dtype,out,only", EXPERTS)
@pytest.mark.parametrize("sorted_rows", [False, True])
def test_expert_forward(T, k, E, N, K, dtype, out, only, sorted_rows):
    print(f"[gpu] expert_forward {T} {k} {E} {N} {K} {dtype} {out} {only} {sorted_rows}", flush=True)
    gen, ids, plan = _routed(T, k, E, N, only=only)
    x = _randn(gen, T * k if sorted_rows else T, K, dtype=dtype)
    w = _randn(gen, E, N, K, dtype=dtype)
    b = _randn(gen, E, N)
    order, _, off = ref.plan(ids.cpu().numpy(), E)
    n = off[-1]
    for bias, relu in ((b, True), (None, False)):
        y = g.expert_forward(x, w, plan, bias, relu=relu, sorted_rows=sorted_rows, out_dtype=DT[out])
        want, mag = ref.expert_rows(_np(x), _np(w), None if bias is None else _np(bias), order, off, k, sorted_rows, relu)
        _close(_np(y)[:n], want, mag, K, out, (relu,))


@pytest.mark.parametrize("T,k,E,N,K,dtype,out,only", EXPERTS)
def test_expert_backward(T, k, E, N, K, dtype, out, only):
    print(f"[gpu] expert_backward {T} {k} {E} {N} {K} {dtype} {only}", flush=True)
    gen, ids, plan = _routed(T, k, E, N, only=only)
    order, _, off = ref.plan(ids.cpu().numpy(), E)
    n = off[-1]
    for sorted_rows, relu_input in ((False, True), (True, False)):
        x = _randn(gen, T * k if sorted_rows else T, K, dtype=dtype)
        w, dy = _randn(gen, E, N, K, dtype=dtype), _randn(gen, T * k, N, dtype=dtype)
        if relu_input:
            x = x.clamp(min=0)
        got = g.expert_backward(dy, x, w, plan, sorted_rows=sorted_rows, relu_input=relu_input)
        want, mag = ref.expert_grads(_np(dy), _np(x), _np(w), order, off, k, sorted_rows, relu_input)
        most = int(np.max(off[1:] - off[:-1]))
        _close(_np(got[0])[:n], want[0], mag[0], N, dtype, "dx")
        _close(_np(got[1]), want[1], mag[1], most, "f32", "dw")
        _close(_np(got[2]), want[2], mag[2], most, "f32", "db")
        again = g.expert_backward(dy, x, w, plan, sorted_rows=sorted_rows, relu_input=relu_input, need_dx=False)
        assert again[0] is None and torch.equal(again[1], got[1]) and torch.equal(again[2], got[2])
        again = g.expert_backward(dy, x, w, plan, sorted_rows=sorted_rows, relu_input=relu_input, need_dw=False)
        assert again[1] is None and torch.equal(again[0][:n], got[0][:n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_experts_with_strides_and_odd_addresses(dtype):
    T, k, E, N, K = 200, 2, 3, 48, 64
    gen, ids, plan = _routed(T, k, E, 1)
    order, _, off = ref.plan(ids.cpu().numpy(), E)
    n = off[-1]
    xw = _randn(gen, T, K + 9, dtype=dtype)
    ww = _randn(gen, E, N + 2, K + 7, dtype=dtype)
    dyw = _randn(gen, T * k, N + 5, dtype=dtype)
    for x, w, dy in ((xw[:, :K], ww[:, :N, :K], dyw[:, :N]), (xw[:, 1:K + 1], ww[:, 1:N + 1, 3:K + 3], dyw[:, 3:N + 3]),
                     (xw[:, 8:K + 8], ww[:, 2:, 7:], dyw[:, 5:])):
        y = g.expert_forward(x, w, plan, out_dtype=torch.float32)
        want, mag = ref.expert_rows(_np(x), _np(w), None, order, off, k)
        _close(_np(y)[:n], want, mag, K, "f32")
        got = g.expert_backward(dy, x, w, plan)
        want, mag = ref.expert_grads(_np(dy), _np(x), _np(w), order, off, k)
        for a, b, m, c, d in zip(got, want, mag, (N, T * k, T * k), (dtype, "f32", "f32")):
            _close(_np(a)[:len(b)], b, m, c, d)
    wt = _randn(gen, E, K, N, dtype=dtype).transpose(1, 2)           # [N][K] whose inner dimension is not contiguous
    y = g.expert_forward(xw[:, :K], wt, plan, out_dtype=torch.float32)
    want, mag = ref.expert_rows(_np(xw[:, :K]), _np(wt), None, order, off, k)
    _close(_np(y)[:n], want, mag, K, "f32")
    one = xw[:1, :K].expand(T, K)                                    # one row for all
    y = g.expert_forward(one, ww[:, :N, :K], plan, out_dtype=torch.float32)
    want, mag = ref.expert_rows(_np(one), _np(ww[:, :N, :K]), None, order, off, k)
    _close(_np(y)[:n], want, mag, K, "f32")


def test_experts_without_rows_and_rows_behind_the_last():
    import ctypes
    from paper_2310_10211_amd import operators as o
    E, N, K, T, k = 4, 40, 48, 300, 2
    ids = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    plan = g.route_plan(ids, E)
    x, w = torch.randn(T, K, device="cuda"), torch.randn(E, N, K, device="cuda")
    dx, dw, db = g.expert_backward(torch.randn(T * k, N, device="cuda"), x, w, plan)
    assert (dw == 0).all() and (db == 0).all()
    y = g.expert_combine(torch.full((T * k, N), float("nan"), device="cuda"), plan, torch.rand(T, k, device="cuda"))
    assert (y == 0).all()                                            # no slot has a row: none is read
    for T2 in (300, 5):                                              # tiles, and few rows
        ids = torch.randint(-1, E, (T2, k), device="cuda", dtype=torch.int32)
        ids[0] = -1
        plan = g.route_plan(ids, E)
        n = int(plan.offsets[-1])
        out = torch.full((T2 * k, N), 7.0, device="cuda")
        cfg = o.ExpertConfig(1, 0, 0, E, k, N, K, T2, K, N * K, K, N, 0, 0)
        st = torch.cuda.current_stream().cuda_stream
        assert g.lib().gevo_expert_forward(ctypes.byref(cfg), x.data_ptr(), w.data_ptr(), None, plan.order.data_ptr(),
                                           plan.offsets.data_ptr(), out.data_ptr(), st) == 0
        assert (out[n:] == 7).all() and torch.equal(out[:n], g.expert_forward(x[:T2], w, plan)[:n])
        dx = torch.full((T2 * k, K), 7.0, device="cuda")
        assert g.lib().gevo_expert_backward(ctypes.byref(cfg), out.data_ptr(), x.data_ptr(), w.data_ptr(),
                                            plan.order.data_ptr(), plan.offsets.data_ptr(), dx.data_ptr(), None, None,
                                            st) == 0
        assert (dx[n:] == 7).all()
    empty = g.route_plan(torch.empty((0, k), dtype=torch.int32, device="cuda"), E)
    assert g.expert_forward(x[:0], w, empty).shape == (0, N)
    dx, dw, db = g.expert_backward(torch.empty(0, N, device="cuda"), x[:0], w, empty)
    assert dx.shape == (0, K) and (dw == 0).all() and (db == 0).all()


def test_expert_plan_of_any_content_stays_inside():
    """Offsets and orders that no plan would hold read and write inside the arrays."""
    E, N, K, T, k = 3, 20, 24, 50, 2
    x, w = torch.randn(T, K, device="cuda"), torch.randn(E, N, K, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for off in ([0, 500, 20, 100], [-7, 10, 5, 90], [90, 40, 100, 1 << 30]):
        plan = g.RoutePlan(torch.full((T * k,), 1 << 20, **i32), torch.full((T, k), 1 << 20, **i32), torch.tensor(off, **i32))
        rows = g.expert_forward(x, w, plan)
        dx, dw, db = g.expert_backward(rows, x, w, plan, relu_input=True)
        y = g.expert_combine(rows, plan)
        drows, dwt = g.expert_combine_backward(y, rows, plan)
        assert (y == 0).all() and (dwt == 0).all()


def test_nan_and_inf_stay_in_their_expert():
    T, k, E, N, K = 200, 1, 4, 32, 64
    ids = (torch.arange(T, device="cuda", dtype=torch.int32) % E).view(T, 1)
    plan = g.route_plan(ids, E)
    x, w = torch.randn(T, K, device="cuda").bfloat16(), torch.randn(E, N, K, device="cuda").bfloat16()
    clean = g.expert_forward(x, w, plan, relu=True)
    x2, w2 = x.clone(), w.clone()
    x2[2, 5] = float("nan")                                          # expert 2, its first row
    w2[1, 3, 0] = float("inf")
    y = g.expert_forward(x2, w2, plan, relu=True)
    off = plan.offsets.tolist()
    assert y[off[2]].isnan().all()                                   # NaN passes a ReLU
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[off[2]] = False
    keep[off[1]:off[2], 3] = False
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("rows_dtype,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,k,E,N", [(1, 1, 1, 1), (7, 3, 5, 10), (130, 8, 64, 257), (33, 2, 4, 1024)])
def test_combine(rows_dtype, out, T, k, E, N):
    gen, ids, plan = _routed(T, k, E, 2)
    rows, wt = _randn(gen, T * k, N + 8, dtype=rows_dtype)[:, :N], torch.rand(T, k, generator=gen, device="cuda")
    pos = plan.pos.cpu().numpy()
    r = np.where((pos >= 0)[..., None], _np(rows)[np.maximum(pos, 0)], 0.0)
    for weights in (wt, None):
        wn = np.ones((T, k)) if weights is None else _np(weights)
        y = g.expert_combine(rows, plan, weights, out_dtype=DT[out])
        _close(_np(y), (r * wn[..., None]).sum(1), np.abs(r * wn[..., None]).sum(1), k, out)
        if rows_dtype == out:
            dy = _randn(gen, T, N + 3, dtype=out)[:, :N]
            drows, dw = g.expert_combine_backward(dy, rows, plan, weights)
            want = (r * _np(dy)[:, None]).sum(2)
            _close(_np(dw), want, np.abs(r * _np(dy)[:, None]).sum(2), N, "f32")
            d = wn[..., None] * _np(dy)[:, None]
            _close(_np(drows)[pos[pos >= 0]], d[pos >= 0], np.abs(d[pos >= 0]), 0, out)
    nan = torch.full((T, k), float("nan"), device="cuda")
    assert g.expert_combine(rows, plan, nan).isnan().all()           # a row that could not be routed says so


# ------------------------------------------------------------------ 4 bits
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 31), (5, 32), (4, 33), (2, 127), (7, 128), (2, 129), (3, 1000), (1, 5000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mx4_quantize(rows, K, dtype):
    gen = _rng("mx4", rows, K)
    x = _randn(gen, rows, K + 3, dtype=dtype)
    x = x * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=gen, device="cuda").float()).to(x.dtype)
    for v in (x[:, :K], x[:, 3:], x[:, :K].contiguous()):
        q = g.mx4_quantize(v)
        values, codes, scales = ref.mx4_quantize(_np(v))
        assert np.array_equal(q.scales.cpu().numpy(), scales)
        assert np.array_equal(q.codes.cpu().numpy(), codes)
        for d in (torch.float32, torch.bfloat16):
            assert np.array_equal(_np(q.dequantize(d)), values)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mx4_quantize_edges(dtype):
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    x = torch.zeros(12, 64)
    x[1, :16] = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    x[2] = -x[1]
    x[3, 5], x[3, 40] = float("nan"), 1.0
    x[4, 5], x[4, 40] = float("inf"), 1.0
    x[5, 5], x[5, 40] = -float("inf"), 3.0
    x[6, :3] = torch.tensor([tiny, 2.0 ** -126, -2.0 ** -127])
    x[7, :3] = torch.tensor([3.3e38, -1e38, 1e37])
    x[8, :2] = torch.tensor([2.0 ** -124, 2.0 ** -130])
    x[9] = torch.linspace(-8, 8, 64)
    x[10] = torch.finfo(DT[dtype]).min
    x[11, ::2] = -0.0
    x = x.to(DT[dtype]).cuda()
    q = g.mx4_quantize(x)
    values, codes, scales = ref.mx4_quantize(_np(x))
    assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(q.codes.cpu().numpy(), codes)
    got = _np(q.dequantize())
    assert np.array_equal(got, values.astype(np.float32).astype(np.float64), equal_nan=True)


def test_mx4_quantize_many_dimensions_and_none():
    x = torch.randn(2, 3, 5, 70, device="cuda")
    q = g.mx4_quantize(x)
    assert q.shape == (2, 3, 5, 70) and torch.equal(q.dequantize()[1, 2], g.mx4_quantize(x[1, 2]).dequantize())
    assert g.mx4_quantize(x[:0]).dequantize().shape == (0, 3, 5, 70)
    assert torch.equal(g.mx4_quantize(x[0, 0].t()).dequantize(), g.mx4_quantize(x[0, 0].t().contiguous()).dequantize())


MX4 = [(1, 1, 1, 1), (1, 1, 40, 784), (3, 5, 17, 33), (2, 16, 16, 128), (2, 17, 70, 200), (1, 300, 300, 96),
       (3, 150, 257, 1000), (256, 1, 24, 64), (1, 129, 511, 4100)]


@pytest.mark.parametrize("P,M,N,K", MX4)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_mx4_matmul(P, M, N, K, out):
    print(f"[gpu] mx4_matmul {P} {M} {N} {K} {out}", flush=True)
    gen = _rng("mm", P, M, N, K)
    # scales that differ from block to block and row to row, so that one taken for another shows
    def q(*shape):
        x = _randn(gen, *shape)
        e = torch.randint(-4, 5, (*shape[:-1], (K + 31) // 32), generator=gen, device="cuda").float()
        return g.mx4_quantize(x * torch.exp2(e).repeat_interleave(32, -1)[..., :K])
    b, bias = q(P, N, K), _randn(gen, P, N)
    for a in (q(M, K), q(P, M, K)):
        av, bv = _np(a.dequantize()), _np(b.dequantize())
        for bi, relu in ((bias, True), (None, False)):
            y = g.mx4_matmul(a, b, bias=bi, relu=relu, out_dtype=DT[out])
            bn = 0 if bi is None else _np(bi)[:, None]
            want = av @ bv.transpose(0, 2, 1) + bn
            mag = np.abs(av) @ np.abs(bv).transpose(0, 2, 1) + np.abs(bn)
            _close(_np(y), np.maximum(want, 0) if relu else want, mag, K, out)


@pytest.mark.parametrize("T,k,E,N,K", [(1, 4, 9, 33, 100), (40, 2, 3, 30, 70), (400, 2, 3, 260, 300), (300, 3, 80, 16, 32)])
@pytest.mark.parametrize("sorted_rows", [False, True])
def test_mx4_matmul_routed(T, k, E, N, K, sorted_rows):
    gen, ids, plan = _routed(T, k, E, 3)
    a = g.mx4_quantize(_randn(gen, T * k if sorted_rows else T, K))
    b, bias = g.mx4_quantize(_randn(gen, E, N, K)), _randn(gen, E, N)
    order, _, off = ref.plan(ids.cpu().numpy(), E)
    y = g.mx4_matmul(a, b, bias=bias, plan=plan, sorted_rows=sorted_rows)
    want, mag = ref.expert_rows(_np(a.dequantize()), _np(b.dequantize()), _np(bias), order, off, k, sorted_rows)
    _close(_np(y)[:off[-1]], want, mag, K, "f32")


def test_mx4_nan_blocks():
    x = torch.randn(40, 128, device="cuda")
    w = g.mx4_quantize(torch.randn(1, 40, 128, device="cuda"))
    clean = g.mx4_matmul(g.mx4_quantize(x), w)
    few = g.mx4_matmul(g.mx4_quantize(x[:8]), w)
    x[3, 70] = float("inf")
    for y, c in ((g.mx4_matmul(g.mx4_quantize(x), w), clean), (g.mx4_matmul(g.mx4_quantize(x[:8]), w), few)):
        assert y[0, 3].isnan().all()
        keep = torch.arange(y.shape[1], device="cuda") != 3
        assert torch.equal(y[:, keep], c[:, keep])


def test_offsets_past_32_bits():
    """The last of three experts lies more than 4 GB into the weights."""
    E, N, K, T = 3, 16400, 65600, 20
    w = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    w[2, N - 300:] = torch.randn(300, K, device="cuda").bfloat16()
    x = torch.randn(T, K, device="cuda").bfloat16()
    for T2 in (2, 20):                                               # few rows, and tiles
        plan = g.route_plan(torch.full((T2, 1), 2, dtype=torch.int32, device="cuda"), E)
        y = g.expert_forward(x[:T2], w, plan, out_dtype=torch.float32)
        xs, ws = x[:T2].double(), w[2, N - 300:].double()
        want, mag = _np(xs @ ws.T), _np(xs.abs() @ ws.abs().T)
        _close(_np(y)[:, N - 300:], want, mag, K, "f32")
        assert (y[:, :N - 300] == 0).all()
    del w
    torch.cuda.empty_cache()


# ----------------------------------------------- used together, streams, graphs
def _layer(logits, x, w, b, dy, k):
    weights, ids = g.route(logits, k, score="sigmoid")
    plan = g.route_plan(ids, logits.shape[1])
    rows = g.expert_forward(x, w, plan, b, relu=True)
    y = g.expert_combine(rows, plan, weights)
    drows, dweights = g.expert_combine_backward(dy, rows, plan, weights)
    drows = drows * (rows > 0)                                       # through the ReLU
    dx, dw, db = g.expert_backward(drows, x, w, plan)
    dx = g.expert_combine(dx, plan)
    return y, dx, dw, db, g.route_backward(logits, ids, dweights, score="sigmoid")


def test_a_routed_layer_and_its_gradient_against_autograd():
    T, E, k, N, K = 60, 5, 2, 24, 40
    gen = _rng("layer")
    logits, x, w, b, dy = (_randn(gen, *s) for s in ((T, E), (T, K), (E, N, K), (E, N), (T, N)))
    y, dx, dw, db, dl = _layer(logits, x, w, b, dy, k)
    lv, xv, wv, bv = (t.double().cpu().requires_grad_(True) for t in (logits, x, w, b))
    s = torch.sigmoid(lv)
    top = lv.topk(k, 1).indices
    wt = s.gather(1, top)
    wt = wt / wt.sum(1, keepdim=True)
    h = torch.relu(torch.einsum("tk,enk->ten", xv, wv) + bv)
    want = (h.gather(1, top[..., None].expand(T, k, N)) * wt[..., None]).sum(1)
    grads = torch.autograd.grad((want * dy.double().cpu()).sum(), (xv, wv, bv, lv))
    for got, ref_ in zip((y, dx, dw, db, dl), (want, *grads)):
        # two chained sums of at most 120 terms each, on values of order 1 to 10
        assert (got.double().cpu() - ref_.detach()).abs().max() <= 2e-5 * max(1.0, float(ref_.detach().abs().max()))


@pytest.mark.parametrize("T", [4, 700])
def test_captured_and_replayed(T):
    E, k, N, K = 12, 3, 136, 72
    gen = _rng("graph", T)
    ins = [_randn(gen, *s) for s in ((T, E), (T, K), (E, N, K), (E, N), (T, N))]

    def both():
        q = g.mx4_quantize(ins[1])
        return (*_layer(*ins, k), g.mx4_matmul(q, g.mx4_quantize(ins[2]), bias=ins[3]), q.dequantize())
    both()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        both()
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        outs = both()
    for i in range(4):
        for t in ins:
            t.copy_(_randn(gen, *t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, both()):
            assert torch.equal(a, b), i
        torch.cuda.synchronize()


def test_two_streams_at_once():
    E, k, N, K, T = 12, 3, 136, 72, 2000
    gen = _rng("streams")
    sets = [[_randn(gen, *s) for s in ((T, E), (T, K), (E, N, K), (E, N), (T, N))] for _ in range(2)]
    want = [_layer(*s, k) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [None, None]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = _layer(*sets[i], k)
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refused_tensors():
    x, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    w, plan = torch.zeros(3, 5, 8, device="cuda"), g.route_plan(ids, 3)
    q, b = g.mx4_quantize(x), g.mx4_quantize(w)
    for call in (
            lambda: g.route(x.double(), 1), lambda: g.route(x[0], 1), lambda: g.route(x, 9), lambda: g.route(x, 0),
            lambda: g.route(x, 1, score="relu"), lambda: g.route(x, 1, groups=3), lambda: g.route(x, 1, top_groups=2),
            lambda: g.route(x, 1, group_top=3), lambda: g.route(x, 1, bias=x[0, :7]), lambda: g.route(x, 1, bias=x[0].cpu()),
            lambda: g.route(x, 1, scale=float("nan")), lambda: g.route(torch.zeros(2, 0, device="cuda"), 1),
            lambda: g.route_plan(ids.long(), 3), lambda: g.route_plan(ids, 0), lambda: g.route_plan(ids, 2049),
            lambda: g.route_backward(x, ids, x), lambda: g.route_backward(x, ids[:3], x[:3, :2]),
            lambda: g.expert_forward(x, w.bfloat16(), plan), lambda: g.expert_forward(x[:3], w, plan),
            lambda: g.expert_forward(x, w[:2], plan), lambda: g.expert_forward(x, w, plan, bias=w[0]),
            lambda: g.expert_forward(x, w, plan, sorted_rows=True), lambda: g.expert_forward(x, w, None),
            lambda: g.expert_forward(x, w, plan, out_dtype=torch.float16), lambda: g.expert_forward(x[:, :7], w, plan),
            lambda: g.expert_backward(x[:, :5], x, w, plan), lambda: g.expert_combine(x, plan, x[:, :2].double()),
            lambda: g.expert_combine(x, plan, x[:, :2]), lambda: g.expert_combine_backward(x, torch.zeros(8, 5, device="cuda"), plan),
            lambda: g.mx4_quantize(x.half()), lambda: g.mx4_quantize(x[0]), lambda: g.mx4_matmul(q, q),
            lambda: g.mx4_matmul(q, g.mx4_quantize(w[..., :7])), lambda: g.mx4_matmul(b, b, bias=w[0]),
            lambda: g.mx4_matmul(q, b, plan=g.route_plan(ids, 4)), lambda: g.mx4_matmul(q, b, sorted_rows=True),
            lambda: g.Mx4(q.codes, q.scales, 200), lambda: g.Mx4(q.codes, q.scales[:2], 8)):
        with pytest.raises(g.GevoError):
            call()


def test_refused_sizes():
    x, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    big = 1 << 32
    for call in (lambda: g.route(x, big + 1), lambda: g.route(x, 1, groups=big + 1),
                 lambda: g.route_plan(ids, big + 3),
                 lambda: g.mx4_quantize(torch.empty(1, 1, device="cuda").expand(0, big + 128))):
        with pytest.raises(g.GevoError):
            call()


# ------------------------------------------------- many row tiles, full steps
@pytest.mark.parametrize("T,k,E,N,K,dtype", [(2500, 1, 1, 700, 192, "bf16"), (2700, 3, 2, 300, 128, "f32"),
                                             (5000, 2, 3, 520, 200, "bf16"), (2300, 7, 5, 66, 256, "bf16")])
def test_experts_of_more_than_eight_row_tiles(T, k, E, N, K, dtype):
    """Tiles are taken eight rows of them at a time: every one once, at both ends of a group."""
    gen, ids, plan = _routed(T, k, E, 11)
    x, w, dy = _randn(gen, T, K, dtype=dtype), _randn(gen, E, N, K, dtype=dtype), _randn(gen, T * k, N, dtype=dtype)
    order, _, off = ref.plan(ids.cpu().numpy(), E)
    n = off[-1]
    y = g.expert_forward(x, w, plan, out_dtype=torch.float32)
    want, mag = ref.expert_rows(_np(x), _np(w), None, order, off, k)
    _close(_np(y)[:n], want, mag, K, "f32")
    got = g.expert_backward(dy, x, w, plan)
    want, mag = ref.expert_grads(_np(dy), _np(x), _np(w), order, off, k)
    most = int(np.max(off[1:] - off[:-1]))
    for a, b, m, c, d in zip(got, want, mag, (N, most, most), (dtype, "f32", "f32")):
        _close(_np(a)[:len(b)], b, m, c, d)


@pytest.mark.parametrize("P,M,N,K,each", [(2, 2500, 300, 512, False), (2, 2500, 300, 512, True), (1, 5000, 270, 768, False)])
def test_mx4_matmul_of_more_than_eight_row_tiles(P, M, N, K, each):
    gen = _rng("mx4 rows", P, M, each)
    a, b = g.mx4_quantize(_randn(gen, *((P, M, K) if each else (M, K)))), g.mx4_quantize(_randn(gen, P, N, K))
    av, bv = _np(a.dequantize()), _np(b.dequantize())
    y = g.mx4_matmul(a, b)
    _close(_np(y), av @ bv.transpose(0, 2, 1), np.abs(av) @ np.abs(bv).transpose(0, 2, 1), K, "f32")


@pytest.mark.parametrize("dtype,K", [("f32", 96), ("bf16", 192), ("bf16", 200)])
def test_rows_outside_x_read_zeros(dtype, K):
    """A sorted row whose slot no row of x has is a row of zeros: its output the bias, its part of dw nothing."""
    T, k, E, N = 300, 3, 2, 140
    gen, ids, plan = _routed(T, k, E, 12, some_missing=False)
    order = plan.order.clone()
    gone = torch.tensor([0, 5, 130, 131, 500, T * k - 1], device="cuda")
    order[gone] = torch.tensor([T * k, -1, 1 << 30, T * k + 7, -5, (1 << 31) - 1], dtype=torch.int32, device="cuda")
    odd = g.RoutePlan(order, plan.pos, plan.offsets)
    x, w, b = _randn(gen, T, K, dtype=dtype), _randn(gen, E, N, K, dtype=dtype), _randn(gen, E, N)
    y, whole = (g.expert_forward(x, w, p, b, out_dtype=torch.float32) for p in (odd, plan))
    expert = torch.searchsorted(plan.offsets[1:].contiguous(), gone.int(), right=True)
    assert torch.equal(y[gone], b[expert])
    keep = torch.ones(T * k, dtype=torch.bool, device="cuda")
    keep[gone] = False
    assert torch.equal(y[keep], whole[keep])
    dy = _randn(gen, T * k, N, dtype=dtype)
    dy0 = dy.clone()
    dy0[gone] = 0
    got, want = (g.expert_backward(d, x, w, p, need_dx=False)[1] for d, p in ((dy, odd), (dy0, plan)))
    # the same products, and zeros, in the same order
    assert torch.equal(got, want)


def test_offsets_past_32_bits_in_tiles():
    """The last of three experts lies more than 4 GB into the weights, rows enough for tiles."""
    E, N, K, T = 3, 16400, 65600, 300
    w = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    w[2, N - 300:] = torch.randn(300, K, device="cuda").bfloat16()
    x = torch.randn(T, K, device="cuda").bfloat16()
    plan = g.route_plan(torch.full((T, 1), 2, dtype=torch.int32, device="cuda"), E)
    y = g.expert_forward(x, w, plan, out_dtype=torch.float32)
    xs, ws = x.double(), w[2, N - 300:].double()
    _close(_np(y)[:, N - 300:], _np(xs @ ws.T), _np(xs.abs() @ ws.abs().T), K, "f32")
    assert (y[:, :N - 300] == 0).all()
    dy = torch.randn(T, N, device="cuda").bfloat16()
    dx = g.expert_backward(dy, x, w, plan, need_dw=False)[0]
    ds = dy[:, N - 300:].double()
    _close(_np(dx), _np(ds @ ws), _np(ds.abs() @ ws.abs()), N, "bf16")
    del w, dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,k,groups", [(64, 5, 1), (128, 8, 4), (256, 8, 8), (200, 20, 1), (512, 6, 1), (1000, 9, 8), (2048, 12, 1)])
def test_route_of_logits_that_agree_or_nearly(dtype, E, k, groups):
    """Equal logits in one lane and across lanes, and ones that differ in the last
    bits of a binary32, of both signs: the choice is the exact one."""
    gen = _rng("near logits", E)
    few = torch.randint(-3, 4, (24, E), generator=gen, device="cuda").float()         # many ties
    step = torch.randint(0, 40, (24, E), generator=gen, device="cuda").float()
    near = few + torch.where(few == 0, step * 1e-30, few * step * 2.0 ** -23)         # within 40 steps of each
    wide = _randn(gen, 24, E, by=3.0)
    wide[:, :: 3] = float("-inf")
    for l in (few, near, wide, near.abs(), -near.abs()):
        how = dict(groups=groups, top_groups=max(1, groups // 2))
        _check_route(l.to(DT[dtype]).contiguous(), k, how)
        _check_route(l.to(DT[dtype]).contiguous(), k, dict(how, score="sigmoid", renorm=False))
    bias = few[0] * 1e-3
    for score in ("softmax", "sigmoid"):
        _check_route(near[:6].to(DT[dtype]).contiguous(), k, dict(score=score, bias=bias, groups=groups,
                                                                  top_groups=max(1, groups // 2), group_top=2))
        _check_route(wide[:6].to(DT[dtype]).contiguous(), k, dict(score=score, bias=bias - 5.0))


def test_more_choices_than_experts_are_refused_before_their_memory():
    x = torch.zeros(4, 8, device="cuda")
    for k in (9, 1 << 31, (1 << 32) - 1):
        with pytest.raises(g.GevoError):
            g.route(x, k)


@pytest.mark.parametrize("T,E,N,K", [(3800, 1, 4096, 256), (9000, 2, 1100, 200)])
def test_large_tiles_captured_and_replayed(T, E, N, K):
    """Tiles whose memory on chip asks for an attribute of the kernel, inside a capture."""
    gen = _rng("large graph", T)
    x, w, dy = (_randn(gen, *s, dtype="bf16") for s in ((T, K), (E, N, K), (T, N)))
    ids = torch.randint(0, E, (T, 1), generator=gen, device="cuda", dtype=torch.int32)

    def both():
        plan = g.route_plan(ids, E)
        q = g.mx4_matmul(g.mx4_quantize(x), g.mx4_quantize(w), plan=plan, out_dtype=torch.bfloat16)
        return (g.expert_forward(x, w, plan, relu=True), *g.expert_backward(dy, x, w, plan), q)
    both()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = both()
    for i in range(3):
        for t in (x, w, dy):
            t.copy_(_randn(gen, *t.shape, dtype="bf16"))
        ids.copy_(torch.randint(0, E, (T, 1), generator=gen, device="cuda", dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, both()):
            assert torch.equal(a, b), i
        torch.cuda.synchronize()


def test_a_scale_that_changes_in_place():
    """A tensor's value is read at each call: a scale is not kept by its identity."""
    x = torch.randn(6, 9, device="cuda")
    dw = torch.randn(6, 2, device="cuda")
    for t in (torch.tensor(2.5), torch.tensor([2.5]), np.array(2.5)):
        for value in (2.5, 5.0, -0.0):
            t[...] = value
            w, ids = g.route(x, 2, scale=t)
            assert torch.equal(w, g.route(x, 2, scale=float(value))[0])
            assert torch.equal(g.route_backward(x, ids, dw, scale=t), g.route_backward(x, ids, dw, scale=float(value)))
    n = torch.tensor(9)
    a = g.route_plan(ids, n)
    n += 3
    assert a.n_experts == 9 and g.route_plan(ids, n).n_experts == 12


def _odd_plan(plan, T, k, gone):
    """The plan with `gone` of its sorted rows naming slots that no row of x has."""
    order = plan.order.clone()
    names = [T * k, -1, 1 << 30, (1 << 31) - 1, -(1 << 31), T * k + 7]
    order[gone] = torch.tensor([names[i % len(names)] for i in range(len(gone))], dtype=torch.int32, device="cuda")
    keep = torch.ones(T * k, dtype=torch.bool, device="cuda")
    keep[gone] = False
    return g.RoutePlan(order, plan.pos, plan.offsets), keep


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("T,k,E,N,K", [(20, 2, 5, 40, 96), (20, 2, 5, 33, 2100), (9, 1, 9, 16, 1027), (30, 3, 2, 70, 4)])
def test_few_rows_outside_x_read_zeros(kind, T, k, E, N, K):
    """The same where an expert has few rows, the contraction split over waves and not."""
    gen, ids, plan = _routed(T, k, E, 13, some_missing=False)
    gone = torch.tensor([0, 1, T * k // 2, T * k - 1], device="cuda")
    odd, keep = _odd_plan(plan, T, k, gone)
    x, w, b = _randn(gen, T, K), _randn(gen, E, N, K), _randn(gen, E, N)
    expert = torch.searchsorted(plan.offsets[1:].contiguous(), gone.int(), right=True)
    if kind == "mx4":
        xq, wq = g.mx4_quantize(x), g.mx4_quantize(w)
        run = lambda p, **how: g.mx4_matmul(xq, wq, bias=b, plan=p, **how)                      # noqa: E731
    else:
        run = lambda p, **how: g.expert_forward(x.to(DT[kind]), w.to(DT[kind]), p, b, **how)    # noqa: E731
    for relu in (False, True):
        for out in (torch.float32, torch.bfloat16):
            y, whole = (run(p, relu=relu, out_dtype=out) for p in (odd, plan))
            want = b[expert].clamp(min=0) if relu else b[expert]
            assert torch.equal(y[gone], want.to(out)), (relu, out)
            assert torch.equal(y[keep], whole[keep])


@pytest.mark.parametrize("dtype,K", [("f32", 96), ("f32", 3), ("bf16", 192), ("bf16", 200), ("bf16", 67)])
@pytest.mark.parametrize("T", [9, 300])
def test_a_row_outside_x_clears_its_gradient(dtype, K, T):
    """With relu_input a sorted row whose slot no row of x has was a row of zeros, of
    which none is > 0; row 0 of x, which lets everything pass, has no part in it."""
    k, E, N = 3, 2, 140
    gen, ids, plan = _routed(T, k, E, 14, some_missing=False)
    gone = torch.tensor([0, 3, T * k // 2, T * k - 1], device="cuda")
    odd, keep = _odd_plan(plan, T, k, gone)
    x, w, dy = _randn(gen, T, K, dtype=dtype), _randn(gen, E, N, K, dtype=dtype), _randn(gen, T * k, N, dtype=dtype)
    x[0] = 1.0
    got, whole = (g.expert_backward(dy, x, w, p, relu_input=True, need_dw=False)[0] for p in (odd, plan))
    assert (got[gone] == 0).all() and torch.equal(got[keep], whole[keep])
    got, whole = (g.expert_backward(dy, x, w, p, need_dw=False)[0] for p in (odd, plan))
    assert torch.equal(got, whole)                   # without it, dx does not read x


# A launch holds fewer than 2^32 work-items: rows past what one holds go out in several.
def _pieces(n, at=1 << 24):
    return [slice(r, min(n, r + at)) for r in range(0, n, at)]


def test_more_rows_than_a_launch_holds_route():
    T, E, k = (1 << 26) + 77, 17, 17                 # 64 lanes a row
    logits = torch.empty(T, E, dtype=torch.bfloat16, device="cuda").normal_(generator=_rng("launch"))
    w, ids = g.route(logits, k)
    for p in _pieces(T):
        a, b = g.route(logits[p], k)
        assert torch.equal(a, w[p]) and torch.equal(b, ids[p])
    got = g.route_backward(logits, ids, w)
    for p in _pieces(T):
        assert torch.equal(g.route_backward(logits[p], ids[p], w[p]), got[p])
    del logits, w, ids, got, a, b
    torch.cuda.empty_cache()


def test_more_rows_than_a_launch_holds_quantize():
    rows, K = (1 << 26) + 77, 3
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda").normal_(generator=_rng("launch", 2))
    q = g.mx4_quantize(x)
    y = q.dequantize(torch.bfloat16)
    for p in _pieces(rows):
        s = g.mx4_quantize(x[p])
        assert torch.equal(s.codes, q.codes[p]) and torch.equal(s.scales, q.scales[p])
        assert torch.equal(s.dequantize(torch.bfloat16), y[p])
    del x, q, y, s
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,k", [((1 << 24) + 19, 5), (1, (1 << 26) + 77)])
def test_more_rows_than_a_launch_holds_join_gradient(T, k):
    gen = _rng("launch", 3)
    n = T * k
    pos = (torch.arange(n, dtype=torch.int32, device="cuda") ^ 5).clamp(max=n - 1)
    pos[n - 8:] = torch.arange(n - 8, n, dtype=torch.int32, device="cuda")       # (a permutation up to its end)
    lone = torch.arange(n, device="cuda") ^ 5
    pos[(lone >= n - 8) & (torch.arange(n, device="cuda") < n - 8)] = -1
    pos[::1001] = -1
    plan = g.RoutePlan(torch.zeros(n, dtype=torch.int32, device="cuda"), pos.view(T, k),
                       torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    rows = torch.randn(n, 2, generator=gen, device="cuda")
    wt, dy = torch.rand(T, k, generator=gen, device="cuda"), torch.randn(T, 2, generator=gen, device="cuda")
    drows, dw = g.expert_combine_backward(dy, rows, plan, wt)
    have = pos >= 0
    at = pos.clamp(min=0).long()
    d = dy.repeat_interleave(k, 0)
    r = rows[at]
    want = torch.where(have, d[:, 0] * r[:, 0] + d[:, 1] * r[:, 1], 0.0)
    mag = (d * r).abs().sum(1)
    assert ((dw.view(-1) - want).abs() <= 8 * 2.0 ** -24 * mag).all()        # two products and a sum, rounded or fused
    assert torch.equal(drows[at[have]], (wt.view(-1, 1) * d)[have])
    del rows, drows, dw, d, r, want, mag, at, have, lone
    torch.cuda.empty_cache()


def test_more_columns_than_a_launch_holds_join():
    """2^34 and some outputs: rows of 2^20, most of whose slots have no row."""
    import ctypes
    from paper_2310_10211_amd import operators as o
    T, k, N, R = (1 << 14) + 3, 2, 1 << 20, 4
    rows = torch.randn(R, N, generator=_rng("launch", 4), device="cuda").bfloat16()
    pos = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    some = {0: (0, 1), 8191: (2, -1), 8192: (-1, 3), 16383: (1, 2), T - 1: (3, 0)}
    for t, p in some.items():
        pos[t] = torch.tensor(p, dtype=torch.int32, device="cuda")
    y = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    cfg = o.CombineConfig(1, 1, 1, k, N, T, N, N)
    assert g.lib().gevo_expert_combine(ctypes.byref(cfg), rows.data_ptr(), pos.data_ptr(), None, y.data_ptr(),
                                       torch.cuda.current_stream().cuda_stream) == 0
    for t in range(0, T, 1024):
        piece = y[t:t + 1024]
        here = torch.zeros(len(piece), dtype=torch.bool, device="cuda")
        for s, p in some.items():
            if t <= s < t + len(piece):
                here[s - t] = True
                want = sum((rows[i].float() for i in p if i >= 0), torch.zeros(N, device="cuda")).bfloat16()
                assert torch.equal(y[s], want)
        assert (piece[~here] == 0).all()
    del y, rows
    torch.cuda.empty_cache()


def test_more_small_tiles_than_a_launch_holds():
    """One expert of one weight on 2^30 and some slots: tiles of 64 rows would be more work-items than a launch takes."""
    T, k = 1025, 1 << 20
    ids = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    plan = g.route_plan(ids, 1)
    del ids
    x = torch.randn(T, 1, generator=_rng("launch", 5), device="cuda").bfloat16()
    w = torch.full((1, 1, 1), 0.5, dtype=torch.bfloat16, device="cuda")
    y = g.expert_forward(x, w, plan)
    assert torch.equal(y.view(T, k), (x * 0.5).expand(T, k))
    dx = g.expert_backward(y, x, w, plan, need_dw=False)[0]
    assert torch.equal(dx.view(T, k), (x * 0.25).expand(T, k))
    del plan, x, w, y, dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("E,k,groups", [(2000, 6, 8), (1030, 3, 2), (1500, 64, 60), (2048, 9, 64), (1100, 5, 55)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_over_many_experts_in_groups_of_any_size(E, k, groups, score):
    """Past 1,024 experts, groups that are a power of two of whole lanes and ones that
    pass through memory on chip, with keys that 32 bits order and that they do not."""
    print(f"[gpu] route {E} {k} {groups} {score}", flush=True)
    gen = _rng("many", E, groups)
    top = max(1, groups // 2)
    wide = _randn(gen, 9, E, by=2.0)
    wide[:, ::5] = float("-inf")
    bias = _randn(gen, E, by=0.2)
    _check_route(wide, k, dict(score=score, groups=groups, top_groups=top))
    _check_route(wide.bfloat16(), k, dict(score=score, groups=groups, top_groups=top, group_top=2, renorm=False))
    _check_route(wide, k, dict(score=score, groups=groups, top_groups=top, group_top=2, bias=bias, scale=2.5))
    l = _randn(gen, 3, E)
    for t in range(3):                               # key = s + bias = 0.5 to the bias's rounding
        near = torch.tensor((0.5 - ref.scores(_np(l[t]), score)).astype(np.float32), device="cuda")
        _check_route(l[t:t + 1], k, dict(score=score, groups=groups, top_groups=top, group_top=2, bias=near))


def test_route_over_many_experts_captured_and_replayed():
    gen = _rng("many graph")
    logits, bias = _randn(gen, 40, 2000), _randn(gen, 2000, by=0.2)
    run = lambda: g.route(logits, 6, bias=bias, groups=8, top_groups=3, group_top=2)    # noqa: E731
    run()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = run()
    for i in range(3):
        logits.copy_(_randn(gen, 40, 2000))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, run()):
            assert torch.equal(a, b), i
        torch.cuda.synchronize()


@pytest.mark.parametrize("E,groups", [(16, 8), (64, 8), (2000, 8)])
def test_route_groups_whose_sums_nearly_tie(E, groups):
    """Two groups of two keys with a bias in common, every rounding of 32 bits against
    the larger one: key halves that go to the even step below and above, and sums that do."""
    gen, T, gs = _rng("sums", E), 1 << 15, E // groups
    for base in (1.0, 16.0, 64.0):
        step = base * 2.0 ** -23
        j = 4 * torch.randint(0, 64, (T, 1), generator=gen, device="cuda") + 1
        r = torch.rand(T, 4, generator=gen, device="cuda", dtype=torch.float64)
        h = 0.5 + j.double() * step / 2 + (r - 0.5) * 2e-7
        logits, bias = torch.full((T, E), -30.0, device="cuda"), torch.zeros(E, device="cuda")
        for c, (e, add) in enumerate(((0, 256), (1, 1), (gs, 257), (gs + 1, 0))):
            logits[:, e] = torch.log(h / (1 - h))[:, c].float()
            bias[e] = base + add * step
        ids = g.route(logits, 1, score="sigmoid", bias=bias, groups=groups, top_groups=1, group_top=2)[1][:, 0].long()
        key = torch.sigmoid(logits.double()) + bias.double()
        sums = key[:, [0, gs]] + key[:, [1, gs + 1]]
        apart = (sums[:, 0] - sums[:, 1]).abs() > 1e-13        # (of a binary64's own rounding)
        assert apart.float().mean() > 0.99
        assert torch.equal(ids[apart], torch.where(sums[:, 0] > sums[:, 1], 0, gs)[apart])
