"""A population's variants as one model: predictions of all of them, or of the
few that a router chooses for each row.

The search (paper section 4) ends with a population of trained variants of one
net, of which the fittest are usually reported one by one.  A Mixture takes a
copy of every variant's layers and runs them on rows of the user's:

  * predict_all: every variant on every row, as Population.predict does over
    the test split, in the population's type or in microscaled 4 bits (a
    prediction's two objectives, time and error, section 4.3);
  * predict: each row through the k variants that gate logits choose for it,
    their logits joined with the gate's weights; gate_gradient is the gradient
    of that with respect to the gate logits, so that a gate over frozen
    variants can be trained.

Hidden layers end in a ReLU and their outputs have the operand type (bf16
populations: rounded to bf16, 4 bits: quantized in blocks of 32); the output
layer's logits are float32, as in the population's own prediction.
"""
from __future__ import annotations

import torch

from . import BF16, GevoError, Population
from .operators import (_number, expert_combine, expert_combine_backward, expert_forward, mx4_matmul, mx4_quantize,
                        route, route_backward, route_plan)


def _indices(variants, n, device):
    """variants as a tensor of indices below n; neither masks nor fractions are any."""
    try:
        index = torch.as_tensor(variants)
    except (TypeError, ValueError, RuntimeError):
        index = torch.empty(0)
    if (index.dim() != 1 or index.numel() == 0 or index.dtype == torch.bool or index.is_floating_point() or
            index.is_complex() or int(index.min()) < 0 or int(index.max()) >= n):
        raise GevoError(f"variants: indices in [0, {n})")
    return index.to(device, torch.long)


class Mixture:
    """Copies of the layers of a population's variants (all, or `variants`), in
    numerics "f32", "bf16" or "mx4" (None: the population's own type)."""

    def __init__(self, pop: Population, variants=None, numerics=None):
        if numerics not in (None, "f32", "bf16", "mx4"):
            raise GevoError(f"numerics: 'f32', 'bf16' or 'mx4', not {numerics!r}")
        self.numerics = numerics or ("bf16" if pop._cfg.dtype == BF16 else "f32")
        self.dtype = torch.bfloat16 if self.numerics == "bf16" else torch.float32
        self.dims = list(pop.dims)
        self.layers = []
        index = None if variants is None else _indices(variants, pop.P, pop.workspace.device)
        for l in range(1, len(self.dims)):
            w, b = pop.layer_weights(l, self.dtype)
            if index is not None:
                w, b = w[index], b[index]
            self.layers.append((mx4_quantize(w) if self.numerics == "mx4" else w, b))
        self.n_variants = self.layers[0][1].shape[0]

    def _rows(self, x):
        if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2 and x.shape[1] == self.dims[0]):
            raise GevoError(f"x: a tensor [rows][{self.dims[0]}] on the GPU")
        if self.numerics == "mx4":
            return mx4_quantize(x if x.dtype == torch.bfloat16 else x.float())
        return x.to(self.dtype)

    def predict_all(self, x):
        """Logits [variants][rows][classes] float32 of every variant on every row of
        x (in "f32" and "bf16" up to 2,048 variants)."""
        h = self._rows(x)
        last = len(self.layers) - 1
        plan = None
        if self.numerics != "mx4":                   # every row to every variant, in order
            n, P = x.shape[0], self.n_variants
            plan = route_plan(torch.arange(P, device=x.device, dtype=torch.int32).expand(n, P), P)
        for l, (w, b) in enumerate(self.layers):
            if plan is not None:
                h = expert_forward(h, w, plan, b, relu=l < last, sorted_rows=l > 0,
                                   out_dtype=torch.float32 if l == last else self.dtype)
            else:
                h = mx4_matmul(h, w, bias=b, relu=l < last, out_dtype=torch.float32)
                h = h if l == last else mx4_quantize(h)
        return h.view(self.n_variants, x.shape[0], self.dims[-1])

    def rows_of(self, x, plan):
        """Logits [rows k][classes] float32, sorted by variant, of the variants that the plan chose."""
        h = self._rows(x)
        last = len(self.layers) - 1
        for l, (w, b) in enumerate(self.layers):
            if self.numerics == "mx4":
                h = mx4_matmul(h, w, bias=b, relu=l < last, plan=plan, sorted_rows=l > 0, out_dtype=torch.float32)
                h = h if l == last else mx4_quantize(h)
            else:
                h = expert_forward(h, w, plan, b, relu=l < last, sorted_rows=l > 0,
                                   out_dtype=torch.float32 if l == last else self.dtype)
        return h

    def predict(self, x, gate_logits, top_k, **how):
        """(logits [rows][classes] float32, state) of each row's top_k variants by
        gate_logits [rows][variants], joined with route's weights; `how` are
        route's options.  state is what gate_gradient asks for; it holds
        gate_logits themselves, whose values have to stay until then."""
        if gate_logits.shape != (x.shape[0], self.n_variants):
            raise GevoError(f"gate_logits: shape {(x.shape[0], self.n_variants)}, not {tuple(gate_logits.shape)}")
        if "scale" in how:                           # its value now, which the gradient takes too
            how["scale"] = _number("scale", how["scale"])
        weights, ids = route(gate_logits, top_k, **how)
        plan = route_plan(ids, self.n_variants)
        rows = self.rows_of(x, plan)
        state = (gate_logits, weights, ids, plan, rows, {k: how[k] for k in ("score", "renorm", "scale") if k in how})
        return expert_combine(rows, plan, weights), state

    @staticmethod
    def gate_gradient(state, dlogits):
        """Gradient with respect to predict's gate_logits, in their type, from the
        gradient dlogits [rows][classes] float32 of its logits.  autograd sees
        none of this: gate_logits.backward(gate_gradient(state, dlogits)) carries
        it on to a gate made of torch modules."""
        gate_logits, weights, ids, plan, rows, how = state
        _, dweights = expert_combine_backward(dlogits, rows, plan, weights)
        return route_backward(gate_logits, ids, dweights, **how)


def scores(logits, labels):
    """(mean cross-entropy, accuracy) of logits [..., rows][classes] against labels
    [rows]: argmax with the lowest index on ties, a NaN logit a miss and its
    loss NaN, as Population.scores counts them; so is a label that is no class."""
    labels = labels.long().expand(logits.shape[:-1])
    known = (labels >= 0) & (labels < logits.shape[-1])
    own = logits.gather(-1, torch.where(known, labels, 0)[..., None])[..., 0]
    loss = torch.where(known, torch.logsumexp(logits, -1) - own, torch.nan)
    top = logits.amax(-1, keepdim=True)
    index = torch.arange(logits.shape[-1], device=logits.device)
    first = torch.where(logits == top, index, logits.shape[-1]).amin(-1)
    return loss.mean(-1), (known & (first == labels)).float().mean(-1)
