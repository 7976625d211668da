"""Routed and 4-bit operators on a population's layers, as measurable cases.

A population's variants serve together as experts: a router sends every row to
a few of them (route, route_plan), their layers run on the rows they got
(expert_forward), the rows are joined with the router's weights
(expert_combine), and each of these has its backward pass.  Layers are also
held in microscaled 4-bit floating point (mx4_quantize, mx4_matmul), for every
variant on every row or for routed rows.

listed() names the cases, draw() gives more of the same ranges, prepare() makes
what a program has in hand, run() is one pass (own: the library's calls, else
the plain form), work() counts what a pass cannot do without, exact() computes
a pass in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _route(name, T, E, k, dtype, score, bias=False, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0,
           masked=0.0):
    return dict(name=name, op="route", T=T, E=E, k=k, dtype=dtype, score=score, bias=bias, groups=groups,
                top_groups=top_groups, group_top=group_top, renorm=renorm, scale=scale, masked=masked)


def _gate(name, T, E, k, N, dtype, score, renorm, scale=1.0):
    return dict(name=name, op="route", gradient=True, T=T, E=E, k=k, N=N, dtype=dtype, score=score, renorm=renorm,
                scale=scale)


def _experts(name, T, E, k, K, N, dtype, relu):
    return dict(name=name, op="experts", T=T, E=E, k=k, K=K, N=N, dtype=dtype, relu=relu)


def _experts_gradient(name, T, E, k, K, N, dtype, relu):
    return dict(_experts(name, T, E, k, K, N, dtype, relu), gradient=True)


def _quantize(name, rows, K, dtype):
    return dict(name=name, op="mx4_quantize", rows=rows, K=K, dtype=dtype)


def _matmul(name, P, M, N, K, out, relu, routed=0):
    return dict(name=name, op="mx4_matmul", P=P, M=M, N=N, K=K, out=out, relu=relu, routed=routed)


def listed():
    return [
        # one row's choice among 64 experts: launches and latency
        _route("route-one", 1, 64, 6, "f32", "softmax"),
        # a test split of 10,000 rows over a population of 1,024 variants, a quarter of them masked for each row
        _route("route-population", 10000, 1024, 4, "bf16", "softmax", renorm=False, masked=0.25),
        # a long prompt or training batch: sigmoid scores, a bias for balance, 4 of 8 groups
        _route("route-groups", 65536, 256, 8, "f32", "sigmoid", bias=True, groups=8, top_groups=4, group_top=2,
               scale=2.5),
        # the gate's training: through the join to the rows and the weights, and on to the logits
        _gate("gate-gradient", 8192, 128, 4, 1024, "bf16", "softmax", False),
        # one row through 8 of 64 experts' layer: weight traffic
        _experts("experts-one", 1, 64, 8, 2048, 1024, "bf16", False),
        # a batch through 4 of 64 experts, unevenly chosen
        _experts("experts-batch", 8192, 64, 4, 2048, 2048, "bf16", True),
        # full precision, a population's first layer, sizes that are no tile multiples
        _experts("experts-f32", 4999, 48, 2, 784, 257, "f32", True),
        # the training step of experts' weights on routed rows
        _experts_gradient("experts-gradient", 8192, 32, 2, 1024, 2048, "bf16", True),
        # the first layer of 64 variants of 784-512-... to 4 bits and back to the values that it holds
        _quantize("quantize-weights", 64 * 512, 784, "f32"),
        # activations of a batch, rows of odd length
        _quantize("quantize-rows", 2047, 1001, "bf16"),
        # the prediction workload's first layer in 4 bits: 64 variants over 10,000 rows
        _matmul("mx4-predict", 64, 10000, 512, 784, "bf16", True),
        # one row through that layer of 256 variants: weight traffic
        _matmul("mx4-one", 256, 1, 512, 784, "f32", True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the operator, then its sizes over the listed ranges, drawn
    again until they cost no more than the operator's largest listed case."""
    op = rng.choice(["route", "gate", "experts", "experts_gradient", "mx4_quantize", "mx4_matmul", "mx4_matmul"])
    while True:
        if op == "route":
            groups = rng.choice([1, 1, 4, 8])
            E = groups * _log(rng, 2, 1024 // groups)
            top_groups = rng.randint(1, groups)
            k = rng.randint(1, min(16, E // groups * top_groups))
            T = _log(rng, 1, 65536)
            if T * E > 65536 * 256:
                continue
            c = _route("", T, E, k, rng.choice(["f32", "bf16"]), rng.choice(["softmax", "sigmoid"]),
                       rng.random() < 0.5, groups, top_groups, 2 if groups > 1 and E // groups > 1 and
                       rng.random() < 0.5 else 1, rng.random() < 0.6, rng.choice([1.0, 2.5]))
        elif op == "gate":
            E = _log(rng, 2, 512)
            c = _gate("", _log(rng, 1, 8192), E, rng.randint(1, min(8, E)), _log(rng, 8, 4096),
                      rng.choice(["f32", "bf16"]), rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5)
            if c["T"] * c["k"] * c["N"] * (2 if c["dtype"] == "f32" else 1) > 8192 * 4 * 1024:
                continue
        elif op in ("experts", "experts_gradient"):
            E = _log(rng, 1, 64)
            c = (_experts if op == "experts" else _experts_gradient)(
                "", _log(rng, 1, 8192), E, rng.randint(1, min(8, E)), _log(rng, 16, 4096), _log(rng, 10, 4096),
                rng.choice(["f32", "bf16", "bf16"]), rng.random() < 0.5)
            most = 8192 * 4 * 2048 * 2048 if op == "experts" else 8192 * 2 * 1024 * 2048
            if (c["T"] * c["k"] * c["K"] * c["N"] * (8 if c["dtype"] == "f32" else 1) > most or
                    E * c["K"] * c["N"] > 64 * 2048 * 1024):
                continue
        elif op == "mx4_quantize":
            c = _quantize("", _log(rng, 1, 65536), _log(rng, 1, 8192), rng.choice(["f32", "bf16"]))
            if c["rows"] * c["K"] > 64 * 512 * 784:
                continue
        else:
            P = _log(rng, 1, 256)
            c = _matmul("", P, _log(rng, 1, 10000), _log(rng, 10, 4096), _log(rng, 32, 8192),
                        rng.choice(["f32", "bf16"]), rng.random() < 0.5,
                        rng.randint(1, min(4, P)) if rng.random() < 0.4 else 0)
            rows = c["M"] * (c["routed"] or P)
            if (rows * c["N"] * (2 if c["out"] == "f32" else 1) > 64 * 10000 * 512 or
                    rows * c["N"] * c["K"] > 64 * 10000 * 512 * 784 or P * c["N"] * c["K"] > 256 * 512 * 784 or
                    rows * c["K"] > 1 << 28):
                continue
        del c["name"]
        return c


# ------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.float32, by=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * by).to(dtype)


def _routing(g, T, E, k):
    """Routing of T rows to k of E experts, some chosen more often: ids, weights
    and the plan, the rows' slots sorted by expert."""
    popularity = torch.randn(E, generator=g, device="cuda") * 0.5
    noise = torch.rand(T, E, generator=g, device="cuda").clamp(min=1e-6)
    ids = (popularity - (-noise.log()).log()).topk(k, dim=1).indices.to(torch.int32)
    w = torch.rand(T, k, generator=g, device="cuda") + 0.1
    return ids, w / w.sum(1, keepdim=True), _plan(ids, E)


def _plan(ids, E):
    flat = ids.reshape(-1)
    by_expert, order = torch.sort(flat, stable=True)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(order.numel(), device=ids.device)
    offsets = torch.searchsorted(by_expert, torch.arange(E + 1, device=ids.device, dtype=flat.dtype))
    return order.to(torch.int32), pos.reshape(ids.shape).to(torch.int32), offsets.to(torch.int32)


def _codes(x):
    """Rows in the 4-bit layout: codes [rows][Kp/2] (two values a byte, the even
    one low) and scales [rows][Kp/32] (power of two + 127), Kp a multiple of
    128, zeros past the row's end."""
    rows, K = x.shape
    Kp = (K + 127) // 128 * 128
    x = torch.nn.functional.pad(x.float(), (0, Kp - K)).reshape(rows, Kp // 32, 32)
    scale = (torch.frexp(x.abs().amax(2))[1] - 3).clamp(min=-127)
    a = torch.ldexp(x.abs(), -scale[..., None])
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    index = (torch.where(q < 2, q * 2, torch.where(q < 4, q + 2, q / 2 + 4))).to(torch.uint8)
    index = index | (torch.signbit(x).to(torch.uint8) << 3)
    index = index.reshape(rows, Kp // 2, 2)
    return (index[..., 0] | (index[..., 1] << 4)).contiguous(), (scale + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    c = case
    st = {"case": dict(c)}
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        st["logits"] = _randn(g, T, E, dtype=DTYPES[c["dtype"]], by=1.5)
        if c.get("gradient"):
            st["ids"], st["weights"], (st["order"], st["pos"], st["offsets"]) = _routing(g, T, E, k)
            st["rows"] = _randn(g, T * k, c["N"], dtype=DTYPES[c["dtype"]])
            st["dy"] = _randn(g, T, c["N"], dtype=DTYPES[c["dtype"]], by=0.1)
            return st
        st["bias"] = _randn(g, E, by=0.1) if c["bias"] else None
        if c["masked"]:
            gone = torch.rand(T, E, generator=g, device="cuda") < c["masked"]
            gone[:, :k] = False                              # k of them always stay
            st["logits"] = st["logits"].masked_fill(gone, float("-inf"))
    elif c["op"] == "experts":
        T, E, k, K, N, d = c["T"], c["E"], c["k"], c["K"], c["N"], DTYPES[c["dtype"]]
        st["ids"], st["weights"], (st["order"], st["pos"], st["offsets"]) = _routing(g, T, E, k)
        st["most"] = int((st["offsets"][1:] - st["offsets"][:-1]).max())    # rows of the busiest expert
        st["x"] = _randn(g, T, K, dtype=d)
        st["w"] = _randn(g, E, N, K, dtype=d, by=K ** -0.5)
        if c.get("gradient"):
            st["dy"] = _randn(g, T * k, N, dtype=d)
            if c["relu"]:
                st["x"] = st["x"].clamp(min=0)               # a hidden layer's outputs
        else:
            st["bias"] = _randn(g, E, N, by=0.1)
    elif c["op"] == "mx4_quantize":
        spread = torch.exp2(torch.randint(-6, 4, (c["rows"], 1), generator=g, device="cuda").float())
        st["x"] = (_randn(g, c["rows"], c["K"]) * spread).to(DTYPES[c["dtype"]])
    else:
        P, M, N, K = c["P"], c["M"], c["N"], c["K"]
        st["a"] = _codes(_randn(g, M, K))
        st["b"] = _codes(_randn(g, P * N, K, by=K ** -0.5))
        st["bias"] = _randn(g, P, N, by=0.1)
        if c["routed"]:
            st["ids"], _, (st["order"], st["pos"], st["offsets"]) = _routing(g, M, P, c["routed"])
            st["most"] = int((st["offsets"][1:] - st["offsets"][:-1]).max())
    return st


# -------------------------------------------------------------- plain forms
def _plain_route(st):
    c, bias = st["case"], st["bias"]
    k, G = c["k"], c["groups"]
    l = st["logits"].double()                                # keys lie close together: in 64 bits
    s = torch.exp(l - l.amax(1, keepdim=True)) if c["score"] == "softmax" else 1 / (1 + torch.exp(-l))
    if c["score"] == "softmax":
        s = s / s.sum(1, keepdim=True)
    key = l if bias is None and c["group_top"] == 1 else s if bias is None else s + bias.double()
    if G > 1:
        per = key.reshape(key.shape[0], G, -1)
        value = per.sort(dim=2, descending=True)[0][..., :c["group_top"]].sum(2)
        best = value.sort(dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        stays = torch.zeros(value.shape, dtype=torch.bool, device=key.device).scatter_(1, best, True)
        key = per.masked_fill(~stays[..., None], float("-inf")).reshape(key.shape)
    ids = key.sort(dim=1, descending=True, stable=True)[1][:, :k]
    w = s.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    ids = ids.to(torch.int32)
    order, pos, offsets = _plan(ids, c["E"])
    return {"weights": (w * c["scale"]).float(), "ids": ids, "order": order, "pos": pos, "offsets": offsets}


def _plain_gate(st):
    c = st["case"]
    T, k, dt = c["T"], c["k"], DTYPES[c["dtype"]]
    rows = st["rows"].float()[st["pos"].long()]              # [T][k][N]
    dy = st["dy"].float()
    dw = (rows * dy[:, None, :]).sum(2)
    slot = st["order"].long()
    drows = (dy[slot // k] * st["weights"].reshape(-1)[slot, None]).to(dt)
    l, ids = st["logits"].float(), st["ids"].long()
    if c["score"] == "softmax":
        s = torch.exp(l - l.amax(1, keepdim=True))
        s = s / s.sum(1, keepdim=True)
    else:
        s = 1 / (1 + torch.exp(-l))
    chosen = s.gather(1, ids)
    ds = dw * c["scale"]
    if c["renorm"]:
        total = chosen.sum(1, keepdim=True)
        ds = (ds - (ds * chosen).sum(1, keepdim=True) / total) / total
    full = torch.zeros_like(s).scatter_(1, ids, ds)
    if c["score"] == "softmax":
        dl = s * (full - (chosen * ds).sum(1, keepdim=True))
    else:
        dl = s * (1 - s) * full
    return {"dlogits": dl.to(dt), "drows": drows, "dweights": dw}


def _places(st, k):
    """Token, expert and place among the expert's rows of every sorted slot."""
    slot = st["order"].long()
    e = st["ids"].reshape(-1).long()[slot]
    return slot // k, e, torch.arange(slot.numel(), device=slot.device) - st["offsets"].long()[e]


def _spread(x, E, most, e, at):
    """Rows x of the sorted slots as [E][most][width], zeros where an expert has fewer."""
    out = torch.zeros(E, most, x.shape[1], device=x.device)
    out[e, at] = x
    return out


def _plain_experts(st):
    c = st["case"]
    k, E, dt = c["k"], c["E"], DTYPES[c["dtype"]]
    token, e, at = _places(st, k)
    xs = _spread(st["x"].float()[token], E, st["most"], e, at)
    w = st["w"].float()
    if c.get("gradient"):
        dys = _spread(st["dy"].float(), E, st["most"], e, at)
        dx = torch.bmm(dys, w)[e, at]
        if c["relu"]:
            dx = dx * (st["x"][token] > 0)
        return {"dx": dx.to(dt), "dw": torch.bmm(dys.transpose(1, 2).contiguous(), xs), "db": dys.sum(1)}
    y = torch.bmm(xs, w.transpose(1, 2).contiguous()) + st["bias"][:, None, :]
    if c["relu"]:
        y = y.clamp(min=0)
    y = y[e, at][st["pos"].long()]                           # [T][k][N]
    return {"y": (y * st["weights"][..., None]).sum(1).to(dt)}


def _plain_quantize(st):
    x = st["x"].float()
    rows, K = x.shape
    b = torch.nn.functional.pad(x, (0, -K % 32)).reshape(rows, -1, 32)
    scale = (torch.frexp(b.abs().amax(2, keepdim=True))[1] - 3).clamp(min=-127)
    a = torch.ldexp(b, -scale)
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(-6.0, 6.0)
    return {"values": torch.ldexp(q, scale).reshape(rows, -1)[:, :K].to(torch.bfloat16).contiguous()}


def _decoded(codes, scales, dtype):
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device, dtype=dtype)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).reshape(codes.shape[0], -1, 32)
    return (v * torch.exp2(scales.to(dtype) - 127)[..., None]).reshape(codes.shape[0], -1)


def _plain_matmul(st):
    c = st["case"]
    a = _decoded(*st["a"], torch.float32)
    b = _decoded(*st["b"], torch.float32).reshape(c["P"], c["N"], -1)
    if c["routed"]:
        token, e, at = _places(st, c["routed"])
        y = torch.bmm(_spread(a[token], c["P"], st["most"], e, at), b.transpose(1, 2)) + st["bias"][:, None, :]
        y = y[e, at]
    else:
        y = torch.matmul(a, b.transpose(1, 2)) + st["bias"][:, None, :]
    if c["relu"]:
        y = y.clamp(min=0)
    return {"y": y.to(DTYPES[c["out"]])}


# -------------------------------------------------------- the library's calls
def _own(st):
    import paper_2310_10211_amd as g
    c = st["case"]
    if c["op"] == "route" and c.get("gradient"):
        plan = g.RoutePlan(st["order"], st["pos"], st["offsets"])
        drows, dw = g.expert_combine_backward(st["dy"], st["rows"], plan, st["weights"])
        dl = g.route_backward(st["logits"], st["ids"], dw, score=c["score"], renorm=c["renorm"], scale=c["scale"])
        return {"dlogits": dl, "drows": drows, "dweights": dw}
    if c["op"] == "route":
        w, ids = g.route(st["logits"], c["k"], score=c["score"], bias=st["bias"], groups=c["groups"],
                         top_groups=c["top_groups"], group_top=c["group_top"], renorm=c["renorm"], scale=c["scale"])
        plan = g.route_plan(ids, c["E"])
        return {"weights": w, "ids": ids, "order": plan.order, "pos": plan.pos, "offsets": plan.offsets}
    if c["op"] == "experts":
        plan = g.RoutePlan(st["order"], st["pos"], st["offsets"])
        if c.get("gradient"):
            dx, dw, db = g.expert_backward(st["dy"], st["x"], st["w"], plan, relu_input=c["relu"])
            return {"dx": dx, "dw": dw, "db": db}
        rows = g.expert_forward(st["x"], st["w"], plan, bias=st["bias"], relu=c["relu"], out_dtype=torch.float32)
        return {"y": g.expert_combine(rows, plan, st["weights"], out_dtype=DTYPES[c["dtype"]])}
    if c["op"] == "mx4_quantize":
        return {"values": g.mx4_quantize(st["x"]).dequantize(torch.bfloat16)}
    a = g.Mx4(*st["a"], c["K"])
    b = g.Mx4(st["b"][0].view(c["P"], c["N"], -1), st["b"][1].view(c["P"], c["N"], -1), c["K"])
    plan = g.RoutePlan(st["order"], st["pos"], st["offsets"]) if c["routed"] else None
    return {"y": g.mx4_matmul(a, b, bias=st["bias"], relu=c["relu"], plan=plan, out_dtype=DTYPES[c["out"]])}


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "route":
        return _plain_gate(state) if c.get("gradient") else _plain_route(state)
    return {"experts": _plain_experts, "mx4_quantize": _plain_quantize, "mx4_matmul": _plain_matmul}[c["op"]](state)


# ------------------------------------------------------------------- counts
def work(case):
    c = case
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        e = 4 if c["dtype"] == "f32" else 2
        if c.get("gradient"):
            S, N = T * k, c["N"]
            return {"bytes": 2 * S * N * e + T * N * e + 2 * T * E * e + 20 * S, "flops": 3 * S * N + 6 * T * E}
        return {"bytes": T * E * e + (4 * E if c["bias"] else 0) + 16 * T * k + 4 * (E + 1), "flops": 6 * T * E}
    if c["op"] == "experts":
        T, E, k, K, N = c["T"], c["E"], c["k"], c["K"], c["N"]
        e = 4 if c["dtype"] == "f32" else 2
        S = T * k
        if c.get("gradient"):
            return {"bytes": S * N * e + T * K * e + min(E, S) * N * K * e + S * K * e + E * N * K * 4 + E * N * 4,
                    "flops": 4 * S * N * K}
        return {"bytes": T * K * e + min(E, S) * (N * K * e + N * 4) + T * N * e + 8 * S, "flops": 2 * S * N * K}
    if c["op"] == "mx4_quantize":
        n = c["rows"] * c["K"]
        return {"bytes": n * ((4 if c["dtype"] == "f32" else 2) + 2), "flops": 4 * n}
    P, M, N, K = c["P"], c["M"], c["N"], c["K"]
    rows = M * (c["routed"] or P)
    blocks = (K + 31) // 32
    read = min(P, rows) if c["routed"] else P
    return {"bytes": 17 * blocks * (M + read * N) + read * N * 4 + rows * N * (4 if c["out"] == "f32" else 2),
            "flops": 2 * rows * N * K}


# ------------------------------------------------------------ in 64 bits
def _exact_route(st):
    c = st["case"]
    l = st["logits"].double()
    s = torch.softmax(l, 1) if c["score"] == "softmax" else torch.sigmoid(l)
    key = s + (0 if st["bias"] is None else st["bias"].double())
    if st["bias"] is None and c["group_top"] == 1:
        key = l.clone()
    T, E = key.shape
    low = torch.full((), -math.inf, dtype=torch.float64, device=key.device)
    index = torch.arange(E, device=key.device)

    def take(v, n):                                          # n largest by repeated maximum, lowest index first
        v, out = v.clone(), []
        for _ in range(n):
            i = torch.where(v == v.amax(1, keepdim=True), index[:v.shape[1]], E).amin(1, keepdim=True)
            out.append(i)
            v.scatter_(1, i, -math.inf)
        return torch.cat(out, 1)

    if c["groups"] > 1:
        per = key.reshape(T, c["groups"], -1)
        value = per.topk(c["group_top"], dim=2)[0].sum(2)
        stays = torch.zeros_like(value).scatter_(1, take(value, c["top_groups"]), 1.0)
        key = torch.where(stays.repeat_interleave(E // c["groups"], 1) > 0, key, low)
    ids = take(key, c["k"])
    w = s.gather(1, ids)
    w = c["scale"] * (w / w.sum(1, keepdim=True) if c["renorm"] else w)
    flat = ids.reshape(-1).cpu().numpy()
    order = np.argsort(flat, kind="stable")
    pos = np.empty_like(order)
    pos[order] = np.arange(len(order))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))])
    return {"weights": w, "ids": ids.to(torch.int32), "order": order.astype(np.int32),
            "pos": pos.reshape(T, -1).astype(np.int32), "offsets": offsets.astype(np.int32)}


def _exact_gate(st):
    c = st["case"]
    T, k = c["T"], c["k"]
    l = st["logits"].double().requires_grad_(True)
    rows = st["rows"].double()
    dy = st["dy"].double()
    pos, ids = st["pos"].long(), st["ids"].long()
    dw = torch.stack([(rows[pos[:, j]] * dy).sum(1) for j in range(k)], 1)
    drows = torch.empty_like(rows)
    for j in range(k):
        drows[pos[:, j]] = dy * st["weights"][:, j, None].double()
    s = torch.softmax(l, 1) if c["score"] == "softmax" else torch.sigmoid(l)
    w = s.gather(1, ids)
    w = c["scale"] * (w / w.sum(1, keepdim=True) if c["renorm"] else w)
    (dl,) = torch.autograd.grad(w, l, dw)
    return {"dlogits": dl, "drows": drows, "dweights": dw}


def _exact_experts(st):
    c = st["case"]
    T, E, k, K, N = c["T"], c["E"], c["k"], c["K"], c["N"]
    x = st["x"].double()
    flat = st["ids"].reshape(-1)
    y = torch.zeros(T * k, N, dtype=torch.float64, device=x.device)
    dx = torch.zeros(T * k, K, dtype=torch.float64, device=x.device)
    dw = torch.zeros(E, N, K, dtype=torch.float64, device=x.device) if c.get("gradient") else None
    db = torch.zeros(E, N, dtype=torch.float64, device=x.device)
    at = 0
    for e in range(E):
        slots = (flat == e).nonzero()[:, 0]
        n = slots.numel()
        xe, we = x[slots // k], st["w"][e].double()
        if c.get("gradient"):
            d = st["dy"][at:at + n].double()
            dx[at:at + n] = (d @ we) * ((xe > 0) if c["relu"] else 1)
            dw[e], db[e] = d.T @ xe, d.sum(0)
        else:
            ye = xe @ we.T + st["bias"][e].double()
            y[slots] = ye.relu() if c["relu"] else ye
        at += n
    if c.get("gradient"):
        return {"dx": dx, "dw": dw, "db": db}
    return {"y": (y.view(T, k, N) * st["weights"].double()[..., None]).sum(1)}


def _exact_quantize(st):
    x = st["x"].double()
    rows, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % 32)).reshape(rows, -1, 32)
    scale = torch.exp2(torch.floor(torch.log2(x.abs().amax(2, keepdim=True).clamp(min=2.0 ** -125))) - 2)
    v = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    middle = (v[1:] + v[:-1]) / 2                            # between two neighbours, a tie goes to the even one
    up = torch.tensor([i % 2 == 0 for i in range(7)], device=x.device)
    a = x.abs() / scale
    index = torch.zeros(a.shape, dtype=torch.int64, device=x.device)
    for i in range(7):
        index += (a > middle[i]) | ((a == middle[i]) & ~up[i])
    return {"values": (v[index] * scale * torch.sign(x)).reshape(rows, -1)[:, :K]}


def _exact_matmul(st):
    c = st["case"]
    a, b = _decoded(*st["a"], torch.float64), _decoded(*st["b"], torch.float64).reshape(c["P"], c["N"], -1)
    if c["routed"]:
        flat = st["ids"].reshape(-1)
        out = []
        for p in range(c["P"]):
            slots = (flat == p).nonzero()[:, 0]
            out.append(a[slots // c["routed"]] @ b[p].T + st["bias"][p].double())
        y = torch.cat(out)
    else:
        y = torch.stack([a @ b[p].T + st["bias"][p].double() for p in range(c["P"])])
    return {"y": y.relu() if c["relu"] else y}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "route":
        return _exact_gate(st) if case.get("gradient") else _exact_route(st)
    return {"experts": _exact_experts, "mx4_quantize": _exact_quantize, "mx4_matmul": _exact_matmul}[case["op"]](st)
