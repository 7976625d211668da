"""Routed and 4-bit operators without a GPU: what the library refuses, before
any HIP call, and the oracle's own definitions against closed forms, brute
force and differences."""
import ctypes
import math

import numpy as np
import pytest

from oracle import operators as ref

g = pytest.importorskip("paper_2310_10211_amd")
pytest.importorskip("torch")

OK, E_ARG, E_SHAPE, E_WORKSPACE, E_UNSUPPORTED = 0, -1, -2, -3, -6
P = 1 << 12                                          # stands for a device pointer; nothing reads it


def _lib():
    try:
        return g.lib()
    except ImportError as e:
        pytest.skip(str(e))


def _fill(cls, base, over):
    c = cls()
    for k, v in {**base, **over}.items():
        setattr(c, k, v)
    return ctypes.byref(c)


ROUTE = dict(abi_version=1, E=8, k=2, T=0, dtype=1, score=0, logits_stride=8, groups=2, top_groups=1, group_top=1,
             renorm=1, scale=1.0)


@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(abi_version=2), E_ARG), (dict(dtype=2), E_ARG), (dict(score=2), E_ARG),
    (dict(E=0), E_SHAPE), (dict(k=0), E_SHAPE), (dict(k=9), E_SHAPE), (dict(T=-1), E_SHAPE),
    (dict(logits_stride=7), E_SHAPE), (dict(groups=3), E_SHAPE), (dict(groups=0), E_SHAPE),
    (dict(top_groups=3), E_SHAPE), (dict(top_groups=0), E_SHAPE), (dict(group_top=3), E_ARG),
    (dict(group_top=0), E_ARG), (dict(renorm=2), E_ARG), (dict(scale=math.inf), E_ARG), (dict(scale=math.nan), E_ARG),
    (dict(E=2049, logits_stride=2049, groups=1), E_UNSUPPORTED),
    (dict(E=128, logits_stride=128, k=65), E_UNSUPPORTED),
    (dict(E=130, logits_stride=130, groups=65), E_UNSUPPORTED), (dict(T=1 << 30), E_UNSUPPORTED),
])
def test_route_refusals(over, code):
    from paper_2310_10211_amd.operators import RouteConfig
    assert _lib().gevo_route(_fill(RouteConfig, ROUTE, over), P, None, P, P, None) == code


def test_pointers_are_checked():
    from paper_2310_10211_amd import operators as o
    L = _lib()
    c = _fill(o.RouteConfig, ROUTE, dict(T=1))
    assert L.gevo_route(None, P, None, P, P, None) == E_ARG
    for bad in ((None, None, P, P), (P + 1, None, P, P), (P, P + 2, P, P), (P, None, None, P), (P, None, P, P + 1)):
        assert L.gevo_route(c, *bad, None) == E_ARG, bad
    for bad in ((None, P, P, P), (P, None, P, P), (P, P, P + 2, P), (P, P, P, P + 1)):
        assert L.gevo_route_backward(c, *bad, None) == E_ARG, bad
    e = _fill(o.ExpertConfig, EXPERT, dict(T=3))
    for bad in ((None, P, None, P, P, P), (P, P + 1, None, P, P, P), (P, P, P + 2, P, P, P), (P, P, None, None, P, P),
                (P, P, None, P, None, P), (P, P, None, P, P, None)):
        assert L.gevo_expert_forward(e, *bad, None) == E_ARG, bad
    for bad in ((None, P, P, P, P, P, P, P), (P, None, P, P, P, P, P, P), (P, P, None, P, P, P, P, P),
                (P, P, P, None, P, P, P, P), (P, P, P, P, None, P, P, P), (P, P, P, P, P, P, None, P)):
        assert L.gevo_expert_backward(e, *bad, None) == E_ARG, bad
    b = _fill(o.CombineConfig, COMBINE, dict(T=3))
    for bad in ((None, P, P, P), (P, None, P, P), (P, P, P + 1, P), (P, P, P, None)):
        assert L.gevo_expert_combine(b, *bad, None) == E_ARG, bad
    for bad in ((None, P, P, P, P, P), (P, None, P, P, P, P), (P, P, None, P, P, P), (P, P, P, P + 2, P, P)):
        assert L.gevo_expert_combine_backward(b, *bad, None) == E_ARG, bad
    m = _fill(o.Mx4Config, MX4, dict(M=3))
    for bad in ((None, P, P, P, None, None, None, P), (P + 8, P, P, P, None, None, None, P),
                (P, P + 2, P, P, None, None, None, P), (P, P, P, None, None, None, None, P),
                (P, P, P, P, P + 1, None, None, P), (P, P, P, P, None, None, P, P), (P, P, P, P, None, None, None, None)):
        assert L.gevo_mx4_matmul(m, *bad, None) == E_ARG, bad
    assert L.gevo_mx4_quantize(0, 2, 5, None, 5, P, P, None) == E_ARG
    assert L.gevo_mx4_quantize(0, 2, 5, P, 5, P + 4, P, None) == E_ARG
    assert L.gevo_mx4_dequantize(0, 2, 5, P, P + 1, P, 5, None) == E_ARG
    assert L.gevo_pop_layer_weights(None, 1, 0, P, P) == E_ARG


EXPERT = dict(abi_version=1, dtype=1, out_dtype=1, E=3, k=2, N=5, K=7, T=0, x_stride=7, w_stride_e=35, w_stride_n=7,
              y_stride=5, sorted_rows=0, relu=0)


@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(abi_version=0), E_ARG), (dict(dtype=3), E_ARG), (dict(out_dtype=-1), E_ARG),
    (dict(sorted_rows=2), E_ARG), (dict(relu=2), E_ARG), (dict(E=0), E_SHAPE), (dict(k=0), E_SHAPE),
    (dict(N=0), E_SHAPE), (dict(K=0), E_SHAPE), (dict(T=-1), E_SHAPE), (dict(x_stride=6), E_SHAPE),
    (dict(w_stride_n=6), E_SHAPE), (dict(w_stride_e=34), E_SHAPE), (dict(w_stride_e=0, E=1), OK),
    (dict(y_stride=4), E_SHAPE), (dict(E=2049), E_UNSUPPORTED), (dict(T=1 << 30), E_UNSUPPORTED),
    (dict(K=(1 << 20) + 1, x_stride=1 << 21, w_stride_n=1 << 21, w_stride_e=1 << 24), E_UNSUPPORTED),
])
def test_expert_refusals(over, code):
    from paper_2310_10211_amd.operators import ExpertConfig
    c = _fill(ExpertConfig, EXPERT, over)
    assert _lib().gevo_expert_forward(c, P, P, None, P, P, P, None) == code
    if code != OK:
        assert _lib().gevo_expert_backward(c, P, P, P, P, P, P, P, P, None) == code


COMBINE = dict(abi_version=1, dtype=0, out_dtype=1, k=2, N=5, T=0, rows_stride=5, y_stride=5)


@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(abi_version=7), E_ARG), (dict(dtype=2), E_ARG), (dict(k=0), E_SHAPE), (dict(N=0), E_SHAPE),
    (dict(T=-2), E_SHAPE), (dict(rows_stride=4), E_SHAPE), (dict(y_stride=4), E_SHAPE),
    (dict(T=1 << 30), E_UNSUPPORTED),
])
def test_combine_refusals(over, code):
    from paper_2310_10211_amd.operators import CombineConfig
    c = _fill(CombineConfig, COMBINE, over)
    assert _lib().gevo_expert_combine(c, P, P, P, P, None) == code
    assert _lib().gevo_expert_combine_backward(c, P, P, P, P, P, P, None) == code


MX4 = dict(abi_version=1, out_dtype=0, P=2, N=5, K=40, M=0, a_each=0, k=1, sorted_rows=0, relu=0)


@pytest.mark.parametrize("over,offsets,code", [
    (dict(), None, OK), (dict(abi_version=3), None, E_ARG), (dict(out_dtype=5), None, E_ARG),
    (dict(P=0), None, E_SHAPE), (dict(N=0), None, E_SHAPE), (dict(K=0), None, E_SHAPE), (dict(M=-1), None, E_SHAPE),
    (dict(k=0), P, E_SHAPE), (dict(a_each=1), P, E_SHAPE), (dict(a_each=1), None, OK), (dict(relu=3), None, E_ARG),
    (dict(P=3000), P, E_UNSUPPORTED), (dict(M=1 << 31), None, E_UNSUPPORTED),
])
def test_mx4_refusals(over, offsets, code):
    from paper_2310_10211_amd.operators import Mx4Config
    assert _lib().gevo_mx4_matmul(_fill(Mx4Config, MX4, over), P, P, P, P, None, P, offsets, P, None) == code


def test_quantize_and_plan_refusals():
    L = _lib()
    assert L.gevo_mx4_quantize(2, 2, 5, P, 5, P, P, None) == E_ARG
    assert L.gevo_mx4_quantize(0, -1, 5, P, 5, P, P, None) == E_SHAPE
    assert L.gevo_mx4_quantize(0, 2, 0, P, 5, P, P, None) == E_SHAPE
    assert L.gevo_mx4_quantize(0, 2, 5, P, 4, P, P, None) == E_SHAPE
    assert L.gevo_mx4_quantize(0, 2, (1 << 20) + 1, P, 1 << 21, P, P, None) == E_UNSUPPORTED
    assert L.gevo_mx4_quantize(0, 0, 5, None, 5, None, None, None) == OK
    n = ctypes.c_size_t()
    assert L.gevo_route_plan_bytes(10, 4, None) == E_ARG
    assert L.gevo_route_plan_bytes(-1, 4, ctypes.byref(n)) == E_SHAPE
    assert L.gevo_route_plan_bytes(10, 0, ctypes.byref(n)) == E_SHAPE
    assert L.gevo_route_plan_bytes(10, 2049, ctypes.byref(n)) == E_UNSUPPORTED
    assert L.gevo_route_plan_bytes(1 << 31, 4, ctypes.byref(n)) == E_UNSUPPORTED
    assert L.gevo_route_plan_bytes(100000, 300, ctypes.byref(n)) == OK and n.value > 0
    assert L.gevo_route_plan(100000, 300, P, P, n.value - 1, P, P, P, None) == E_WORKSPACE
    assert L.gevo_route_plan(100000, 300, P, P + 1, n.value, P, P, P, None) == E_WORKSPACE
    assert L.gevo_route_plan(100000, 300, None, P, n.value, P, P, P, None) == E_ARG
    assert L.gevo_route_plan(100000, 300, P, P, n.value, P, P, None, None) == E_ARG


def test_python_refuses_host_tensors():
    import torch
    _lib()
    x = torch.zeros(2, 4)
    for call in (lambda: g.route(x, 1), lambda: g.route_plan(x.int(), 4), lambda: g.mx4_quantize(x),
                 lambda: g.RoutePlan(x, x, x), lambda: g.Mx4(x, x, 4), lambda: g.expert_combine(x, None),
                 lambda: g.mx4_matmul(x, x), lambda: g.route_backward(x, x, x)):
        with pytest.raises(g.GevoError):
            call()


def test_sizes_past_32_bits_are_refused():
    from paper_2310_10211_amd import operators as o
    _lib()
    big = (1 << 32) + 1                              # 1 in its low 32 bits
    for call in (lambda: o._route_cfg(8, big, 4, 0, 0, 8, 1, 1, 1, 1, 1.0),
                 lambda: o._route_cfg(8, 2, 4, 0, 0, 8, big, 1, 1, 1, 1.0),
                 lambda: o._expert_cfg(0, 0, 3, 2, big, 8, 4, 8, 40, 8, big, 0, 0),
                 lambda: o._combine_cfg(0, 0, 2, big, 4, big, big), lambda: o._mx4_cfg(0, 3, 5, big, 4, 0, 1, 0, 0),
                 lambda: o._plan_bytes(8, big), lambda: o._route_cfg(8, -1, 4, 0, 0, 8, 1, 1, 1, 1, 1.0)):
        with pytest.raises(g.GevoError):
            call()
    assert o._route_cfg(8, 2, 4, 0, 0, 8, 1, 1, 1, 1, 1.0) is not None


def _route_config(scale=1.0, k=2, score="softmax", groups=1, top_groups=1, group_top=1):
    import torch
    from paper_2310_10211_amd import operators as o
    return o._route_config(torch.zeros(3, 8), k, score, groups, top_groups, group_top, True, scale)._obj


def test_configurations_hold_values_not_objects():
    """A tensor or an array that changes in place changes the next call."""
    import torch
    from paper_2310_10211_amd import operators as o
    _lib()
    for t in (torch.tensor(2.5), torch.tensor([2.5], dtype=torch.float64), np.array(2.5), np.float32(2.5)):
        assert _route_config(t).scale == 2.5
    t, a = torch.tensor(2.5), np.array(2.5)
    for value in (5.0, 0.0, -1.25):
        t.fill_(value)
        a[...] = value
        assert _route_config(t).scale == value and _route_config(a).scale == value
    k = torch.tensor(2)
    assert _route_config(k=k).k == 2
    k += 1
    assert _route_config(k=k).k == 3 and _route_config(k=np.int64(3)).k == 3 and _route_config(groups=np.int32(4)).groups == 4
    assert math.copysign(1, _route_config(0.0).scale) == math.copysign(1, _route_config(-0.0).scale)
    assert o._number("scale", 2) == 2.0 and o._index("k", True) == 1


def test_what_is_no_number_is_refused():
    import torch
    _lib()
    x = torch.zeros(2, 4)
    for bad in ([2.5], "2.5", None, np.zeros(2), torch.zeros(2), 1j, {}, 10 ** 400):
        with pytest.raises(g.GevoError):
            _route_config(bad)
    for bad in (2.0, "2", None, [2], np.zeros(2, int), torch.tensor(2.0)):
        for name in ("k", "groups", "top_groups", "group_top"):
            with pytest.raises(g.GevoError):
                _route_config(**{name: bad})
        with pytest.raises(g.GevoError):
            g.Mx4(x, x, bad)
    for bad in (["softmax"], None, 0, {}):
        with pytest.raises(g.GevoError):
            _route_config(score=bad)
    from paper_2310_10211_amd import operators as o
    for bad in ([], "float32", 0):
        with pytest.raises(g.GevoError):
            o._out_dtype(bad, torch.float32)


def test_products_of_more_tiles_than_a_launch_holds():
    """Refused on the host: a launch would drop the tiles past 2^32 work-items."""
    from paper_2310_10211_amd import operators as o
    L = _lib()
    top, wide = (1 << 31) - 1, 1 << 20
    for over in (dict(T=top, k=1, E=1, N=1, K=1, x_stride=1, w_stride_n=1, y_stride=1),
                 dict(T=1 << 24, k=1, N=wide, K=1, x_stride=1, w_stride_n=1, w_stride_e=wide, y_stride=wide)):
        for dtype in (0, 1):
            c = _fill(o.ExpertConfig, EXPERT, dict(over, dtype=dtype))
            assert L.gevo_expert_forward(c, P, P, None, P, P, P, None) == E_UNSUPPORTED
    c = _fill(o.ExpertConfig, EXPERT, dict(T=1 << 24, k=1, N=1, K=wide, x_stride=wide, w_stride_n=wide, w_stride_e=wide,
                                           y_stride=1))
    assert L.gevo_expert_backward(c, P, P, P, P, P, P, None, None, None) == E_UNSUPPORTED
    c = _fill(o.ExpertConfig, EXPERT, dict(E=2048, T=5, N=wide, K=wide, x_stride=wide, w_stride_n=wide,
                                           w_stride_e=1 << 40, y_stride=wide))
    assert L.gevo_expert_backward(c, P, P, P, P, P, None, P, P, None) == E_UNSUPPORTED
    for over in (dict(P=1, M=top, N=1), dict(P=1, M=1 << 24, N=wide)):
        assert L.gevo_mx4_matmul(_fill(o.Mx4Config, MX4, over), P, P, P, P, None, None, None, P, None) == E_UNSUPPORTED


def test_scores_of_labels_that_are_no_class():
    """A label outside the classes reads no logit: its loss is NaN, and it is a miss."""
    import torch
    from paper_2310_10211_amd.mixture import scores
    nan = math.nan
    logits = torch.tensor([[[1.0, 2.0, 0.0], [0.0, 2.0, 2.0]], [[1.0, 2.0, 0.0], [nan, 0.0, 1.0]]])
    for bad in (-1, 3, -(1 << 31), (1 << 31) - 1):
        loss, acc = scores(logits, torch.tensor([1, bad], dtype=torch.int32))
        assert loss.isnan().all() and acc.tolist() == [0.5, 0.5]
    loss, acc = scores(logits[:1], torch.tensor([1, 2]))
    want = (math.log(1 + math.exp(-1) + math.exp(-2)) + math.log(2 + math.exp(-2))) / 2
    assert abs(float(loss[0]) - want) < 1e-6 and acc.tolist() == [0.5]


# ------------------------------------------------------------- the oracle itself
def test_oracle_route_closed_forms():
    l = [math.log(4), math.log(1), math.log(3), -math.inf]
    w, ids = ref.route_row(l, 2, renorm=False)
    assert ids == [0, 2] and np.allclose(w, [0.5, 0.375])
    w, ids = ref.route_row(l, 2, scale=2.0)
    assert np.allclose(w, [2 * 4 / 7, 2 * 3 / 7])
    w, ids = ref.route_row(l, 4)
    assert ids == [0, 2, 1, -1] and w[3] == 0 and np.isclose(w.sum(), 1)
    assert ref.route_row([1.0, 1.0, 1.0], 2)[1] == [0, 1]                    # ties
    assert ref.route_row([0.0, 1.0, 0.0, 0.9], 1, groups=2, bias=[5.0, 0, 0, 0])[1] == [0]
    # groups of two: (2, 2) beats (3, 0) by two keys, not by one
    how = dict(groups=2, score="sigmoid", bias=[2.0, 2.0, 3.0, 0.0])
    assert ref.route_row([0.0] * 4, 1, group_top=2, **how)[1] == [0]
    assert ref.route_row([0.0] * 4, 1, group_top=1, **how)[1] == [2]
    assert np.isnan(ref.route_row([1.0, math.nan], 1)[0]).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_oracle_route_gradient_is_the_difference_quotient(score, renorm):
    rng = np.random.default_rng(3)
    l, dw = rng.normal(size=(3, 6)), rng.normal(size=(3, 3))
    ids = np.array([[1, 4, 0], [5, 5, 2], [3, -1, 0]])                        # one twice, one missing
    how = dict(score=score, renorm=renorm, scale=1.5)
    got = ref.route_backward(l, ids, dw, **how)
    h = 1e-6
    for t in range(3):
        for e in range(6):
            up, dn = l.copy(), l.copy()
            up[t, e] += h
            dn[t, e] -= h
            want = ((ref.route_weights(up, ids, **how) - ref.route_weights(dn, ids, **how)) * dw).sum() / (2 * h)
            assert abs(got[t, e] - want) < 1e-8, (t, e)


def test_oracle_quantizer():
    # every representable value maps to itself, halves go to the even index
    x = np.zeros((1, 32))
    x[0, :8], x[0, 8:16] = ref.E2M1, -ref.E2M1
    x[0, 16:24] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.5]
    v, codes, scales = ref.mx4_quantize(x)
    assert scales[0, 0] == 127 and (scales[0, 1:] == 0).all()
    assert np.array_equal(v[0, :16], x[0, :16])
    assert list(v[0, 16:24]) == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    assert codes[0, 0] == 0x10 and codes[0, 1] == 0x32 and codes[0, 4] & 15 == 8     # two a byte, -0 keeps its sign
    rng = np.random.default_rng(1)
    x = rng.normal(size=(4, 70))
    v, _, scales = ref.mx4_quantize(x)
    for r in range(4):
        for k in range(70):
            step = 2.0 ** (int(scales[r, k // 32]) - 127)
            grid = step * np.concatenate([ref.E2M1, -ref.E2M1])
            top = 6 * step
            assert abs(v[r, k] - x[r, k]) <= max(np.abs(grid - x[r, k]).min(), abs(x[r, k]) - top) + 1e-15


def test_oracle_expert_gradients_are_difference_quotients():
    rng = np.random.default_rng(5)
    x, w, b = rng.normal(size=(4, 3)), rng.normal(size=(3, 2, 3)), rng.normal(size=(3, 2))
    ids = np.array([[0, 2], [2, 2], [0, 1], [-1, 1]])
    order, pos, off = ref.plan(ids, 3)
    assert list(off) == [0, 2, 4, 7] and list(order) == [0, 4, 5, 7, 1, 2, 3] and pos[3, 0] == -1
    dy = rng.normal(size=(7, 2))
    (dx, dw, db), _ = ref.expert_grads(dy, x, w, order, off, 2)
    f = lambda x_, w_, b_: (ref.expert_rows(x_, w_, b_, order, off, 2)[0] * dy).sum()    # noqa: E731
    h = 1e-6
    for arr, grad, at in ((w, dw, (2, 1, 0)), (b, db, (0, 1)), (x, None, (1, 2))):
        up, dn = arr.copy(), arr.copy()
        up[at] += h
        dn[at] -= h
        args = [(up, dn) if a is arr else (a, a) for a in (x, w, b)]
        want = (f(*(a[0] for a in args)) - f(*(a[1] for a in args))) / (2 * h)
        got = grad[at] if grad is not None else sum(dx[r, 2] for r in range(7) if order[r] // 2 == 1)
        assert abs(got - want) < 1e-7
