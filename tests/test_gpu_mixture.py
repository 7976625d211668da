"""A population's variants as one model: copies of their layers, predictions of
all of them in each numerics, and of the few that a router chooses."""
import numpy as np
import pytest

import synthetic
from oracle import operators as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2310_10211_amd as g                     # noqa: E402
from paper_2310_10211_amd.mixture import Mixture, scores   # noqa: E402
from paper_2310_10211_amd.search import Search       # noqa: E402


def _population(dims, P, dtype, n_train=200, n_test=150, epochs=1, stream=None, **over):
    rng = np.random.default_rng(sum(dims) + P)
    cfg = synthetic.config(3, P=P, dims=dims, batch=32, dtype=dtype, dens=(0.4, 1.0), **over)
    x = lambda n: rng.normal(size=(n, dims[0])).astype(np.float32)     # noqa: E731
    y = lambda n: rng.integers(0, dims[-1], n).astype(np.int32)        # noqa: E731
    pop = g.Population(cfg, x(n_train), y(n_train), x(n_test), y(n_test), stream=stream)
    for e in range(epochs):
        pop.train_epoch(e)
    return pop


SHAPES = [([40, 10], 3), ([784, 128, 10], 5), ([784, 128, 10], 40), ([100, 70, 33, 7], 6), ([256, 512, 256, 10], 4)]


@pytest.mark.parametrize("dims,P", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_weights_are_the_exported_parameters(dims, P, dtype):
    print(f"[gpu] layer_weights {dims} {P} {dtype}", flush=True)
    pop = _population(dims, P, dtype)
    full = [pop.layer_weights(l, torch.float32) for l in range(1, len(dims))]
    half = [pop.layer_weights(l, torch.bfloat16) for l in range(1, len(dims))]
    own = pop.layer_weights(1)[0]
    assert own.dtype == (torch.bfloat16 if dtype == "bf16" else torch.float32)
    for v in sorted({0, 1, P - 1}):
        p, off = pop.export(v)["params"], 0
        for (w, b), (wh, bh), K, N in zip(full, half, dims[:-1], dims[1:]):
            want = torch.from_numpy(p[off:off + K * N].reshape(K, N).T.copy()).cuda()
            assert torch.equal(w[v], want) and torch.equal(wh[v], want.bfloat16())
            off += K * N
            assert torch.equal(b[v].cpu(), torch.from_numpy(p[off:off + N])) and torch.equal(bh, b)
            off += N
    for bad in (0, len(dims)):
        with pytest.raises(g.GevoError):
            pop.layer_weights(bad)
    with pytest.raises(g.GevoError):
        pop.layer_weights(1, torch.float16)
    pop.close()


@pytest.mark.parametrize("dims,P", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_predict_all_agrees_with_the_populations_prediction(dims, P, dtype):
    pop = _population(dims, P, dtype)
    pop.predict()
    s = pop.scores()
    logits = Mixture(pop).predict_all(pop.x_test)
    loss, acc = scores(logits, pop.y_test)
    assert logits.shape == (P, pop.n_test, dims[-1])
    # the losses' tolerances of the population's own parity tests
    np.testing.assert_allclose(loss.cpu().numpy(), s["test_loss"], rtol=1e-4 if dtype == "f32" else 2e-2)
    assert np.abs(acc.cpu().numpy() - s["test_acc"]).max() <= 1.5 / pop.n_test
    sub = Mixture(pop, variants=[P - 1, 0, 0]).predict_all(pop.x_test)
    assert sub.shape[0] == 3 and torch.equal(sub[1], sub[2])
    np.testing.assert_allclose(sub[0].cpu(), logits[P - 1].cpu(), rtol=2e-2, atol=2e-2)
    pop.close()


def test_mx4_single_layer_against_the_definition():
    pop = _population([130, 10], 4, "f32")
    x = pop.x_test[:37]
    got = Mixture(pop, numerics="mx4").predict_all(x).double().cpu().numpy()
    xv = ref.mx4_quantize(x.cpu().numpy())[0]
    w, b = pop.layer_weights(1)
    for v in range(4):
        wv, bv = ref.mx4_quantize(w[v].cpu().numpy())[0], b[v].double().cpu().numpy()
        want, mag = xv @ wv.T + bv, np.abs(xv) @ np.abs(wv).T + np.abs(bv)
        assert (np.abs(got[v] - want) <= 132 * 2.0 ** -23 * mag).all()       # a sum of 131 terms in binary32
    pop.close()


@pytest.mark.parametrize("dims,P", SHAPES)
def test_mx4_layers_and_scores(dims, P):
    pop = _population(dims, P, "bf16")
    m = Mixture(pop, numerics="mx4")
    logits = m.predict_all(pop.x_test)
    h = g.mx4_quantize(pop.x_test)                   # the same layer by layer, one variant at a time
    for v in (0, P - 1):
        hv = h
        for l, (w, b) in enumerate(m.layers):
            one = g.Mx4(w.codes[v:v + 1], w.scales[v:v + 1], w.k)
            hv = g.mx4_matmul(hv, one, bias=b[v:v + 1], relu=l + 1 < len(m.layers))
            hv = hv if l + 1 == len(m.layers) else g.mx4_quantize(hv[0])
        assert torch.equal(hv[0], logits[v])
    s = pop.predict_mx4()
    loss, acc = scores(logits, pop.y_test)
    np.testing.assert_allclose(s["test_loss"], loss.cpu().numpy(), rtol=1e-5)
    np.testing.assert_allclose(s["test_acc"], acc.cpu().numpy(), atol=1e-6)
    pop.close()


def test_scores_rules():
    nan = float("nan")
    logits = torch.tensor([[[1.0, 1.0, 0.0], [0.0, 2.0, 2.0], [nan, 0.0, 1.0]]], device="cuda")
    loss, acc = scores(logits, torch.tensor([0, 2, 2], device="cuda"))
    assert loss.isnan().all() and abs(float(acc[0]) - 1 / 3) < 1e-6          # a tie is the lower index, NaN a miss
    loss, acc = scores(logits[:, :2], torch.tensor([0, 2], device="cuda"))
    assert abs(float(loss[0]) - (np.log(2 + np.exp(-1)) + np.log(2 + np.exp(-2))) / 2) < 1e-6


@pytest.mark.parametrize("numerics", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("how", [{}, dict(score="sigmoid", renorm=False, scale=1.5)])
def test_predict_is_the_weighted_sum_of_the_chosen_variants(numerics, how):
    dims, P, k = [100, 70, 33, 7], 9, 3
    pop = _population(dims, P, "f32")
    m = Mixture(pop, numerics=numerics)
    x = pop.x_test
    gate = torch.randn(len(x), P, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    y, state = m.predict(x, gate, k, **how)
    every = m.predict_all(x)
    w, ids = ref.route(gate.double().cpu().numpy(), k, **how)
    assert np.array_equal(state[2].cpu().numpy(), ids)
    e = every.double().cpu().numpy()
    want = sum(w[:, j, None] * e[ids[:, j], np.arange(len(x))] for j in range(k))
    mag = sum(np.abs(w[:, j, None] * e[ids[:, j], np.arange(len(x))]) for j in range(k))
    # the same rows through the same layers; their sums' order can differ between few rows and many, which
    # bf16 and 4-bit hidden values carry on by up to a step of themselves
    tol = {"f32": 1e-5, "bf16": 2e-2, "mx4": 2e-1}[numerics]
    assert (np.abs(y.double().cpu().numpy() - want) <= tol * (mag + np.abs(e).max())).all()
    dl = torch.randn(y.shape, generator=torch.Generator("cuda").manual_seed(4), device="cuda")
    got = Mixture.gate_gradient(state, dl).double().cpu().numpy()
    rows, pos = state[4].double().cpu().numpy(), state[3].pos.cpu().numpy()
    dw = (rows[pos] * dl.double().cpu().numpy()[:, None]).sum(2)
    grad = ref.route_backward(gate.double().cpu().numpy(), ids, dw, **how)
    # dweights: sums of 7 terms; the gradient: of 9 and 3 (see the routing tests)
    assert np.abs(got - grad).max() <= 1e-5 * np.abs(dw).max()
    pop.close()


def test_a_gate_learns_by_its_gradient():
    """The gradient through rows, weights and scores is that of the loss: against differences."""
    pop = _population([40, 32, 10], 6, "f32", epochs=2)
    m = Mixture(pop)
    x, y = pop.x_test, pop.y_test.long()
    gate = torch.randn(len(x), 6, generator=torch.Generator("cuda").manual_seed(1), device="cuda")

    def loss(gl):                                    # in 64 bits from the float32 logits
        z = m.predict(x, gl, 2, score="sigmoid", renorm=False)[0].double()
        return float((torch.logsumexp(z, 1) - z.gather(1, y[:, None])[:, 0]).sum())

    z, state = m.predict(x, gate, 2, score="sigmoid", renorm=False)
    p = torch.softmax(z, 1)
    p[torch.arange(len(x)), y] -= 1
    grad = Mixture.gate_gradient(state, p)
    d = torch.sign(grad) * 1e-3
    up, dn = loss(gate + d), loss(gate - d)          # the choice's borders are farther away for nearly every row
    want = float((grad.double() * d.double()).sum()) * 2
    assert abs((up - dn) - want) <= 0.02 * abs(want) + 1e-3, (up - dn, want)
    pop.close()


def test_a_population_on_its_own_stream():
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        pop = _population([100, 70, 10], 5, "bf16", stream=stream)
    m = Mixture(pop)                                 # on the current stream, after what the population has enqueued
    a = m.predict_all(pop.x_test)
    stream.synchronize()
    assert torch.equal(a, Mixture(pop).predict_all(pop.x_test))
    s = pop.predict_mx4()
    assert np.isfinite(s["test_loss"]).all()
    pop.close()


def test_search_with_test_errors_in_4_bits():
    pop = _population([40, 32, 10], 8, "bf16", epochs=0)
    s = Search(pop, 0.05, seed=5, n_elite=2, test_numerics="mx4")
    first = s.start()
    want = 1.0 - pop.predict_mx4()["test_acc"].astype(np.float64)
    assert np.array_equal(first.test_error, want)
    s.step()
    with pytest.raises(ValueError):
        Search(pop, 0.05, seed=5, n_elite=2, test_numerics="int4")
    pop.close()


def test_mixture_refusals():
    pop = _population([40, 10], 3, "f32")
    m = Mixture(pop)
    x = pop.x_test
    for call in (lambda: Mixture(pop, numerics="int8"), lambda: Mixture(pop, variants=[3]), lambda: Mixture(pop, variants=[]),
                 lambda: m.predict_all(x[:, :39]), lambda: m.predict_all(x.cpu()), lambda: m.predict(x, x[:, :3], 4),
                 lambda: m.predict(x, x[:, :4], 1), lambda: m.predict(x, x[:5, :3], 1)):
        with pytest.raises(g.GevoError):
            call()
    pop.close()


def test_the_gates_gradient_takes_the_predictions_scale():
    """A scale changed after predict is not the one that its state's gradient is of."""
    pop = _population([40, 10], 5, "f32")
    m, x = Mixture(pop), pop.x_test
    gate = torch.randn(len(x), 5, generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    dl = torch.randn(len(x), 10, generator=torch.Generator("cuda").manual_seed(8), device="cuda")
    scale = torch.tensor(1.5)
    _, state = m.predict(x, gate, 2, scale=scale)
    scale.fill_(4.0)
    want = Mixture.gate_gradient(m.predict(x, gate, 2, scale=1.5)[1], dl)
    assert torch.equal(Mixture.gate_gradient(state, dl), want)
    pop.close()


def test_layer_weights_are_there_for_the_current_stream():
    """Read at once on another stream than the population's, behind work that it still has to do."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        pop = _population([784, 128, 10], 16, "bf16", n_train=4000, epochs=3, stream=stream)
    got = [[t.clone() for t in pop.layer_weights(l, torch.float32)] for l in (1, 2)]
    torch.cuda.synchronize()
    for l in (1, 2):
        assert all(torch.equal(a, b) for a, b in zip(got[l - 1], pop.layer_weights(l, torch.float32)))
    before = pop.layer_weights(1, torch.float32)[0]
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):                   # memory given back while another stream reads it is not handed out
        w = pop.layer_weights(1, torch.float32)[0]
        copy = w.clone()
        del w
    with torch.cuda.stream(stream):
        torch.full_like(before, 7.0)
    torch.cuda.synchronize()
    assert torch.equal(copy, before)
    pop.close()


def test_variants_are_whole_indices():
    pop = _population([40, 10], 3, "f32")
    want = Mixture(pop, variants=[2, 0])
    for same in ((2, 0), np.array([2, 0]), torch.tensor([2, 0]), torch.tensor([2, 0], device="cuda", dtype=torch.int32)):
        assert torch.equal(Mixture(pop, variants=same).layers[0][0], want.layers[0][0])
    for bad in ([True, False, True], torch.tensor([True, False, True]), [0.0, 1.9], np.array([0.5]), ["0"], 1):
        with pytest.raises(g.GevoError):
            Mixture(pop, variants=bad)
    pop.close()


def test_outputs_ask_for_no_gradient_and_a_gate_of_modules_trains():
    """autograd records none of the calls; the gate's gradient is handed on to torch."""
    pop = _population([40, 10], 5, "f32")
    m, x = Mixture(pop), pop.x_test
    gate = torch.nn.Linear(40, 5, device="cuda")
    logits = gate(x)
    z, state = m.predict(x, logits, 2)
    assert not z.requires_grad
    dl = torch.randn(z.shape, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    grad = Mixture.gate_gradient(state, dl)
    logits.backward(grad)
    # products of at most 150 terms
    want, mag = grad.double().T @ x.double(), grad.double().abs().T @ x.double().abs()
    assert ((gate.weight.grad.double() - want).abs() <= 152 * 2.0 ** -23 * mag).all()
    pop.close()
