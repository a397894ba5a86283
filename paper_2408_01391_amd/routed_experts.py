"""Experts by clusters: a layer whose tokens go through the matrix of their nearest centroid, forward and backward.

The centroids come from a Lloyd fit over sample rows.  A token has two slots: the matrix of its cluster, weighted by
how near the centroid is, and one that all tokens share.  The matrices are held in 4 bits.

    python -m paper_2408_01391_amd.routed_experts [--tokens N] [--features D] [--outputs F] [--clusters K] [--classes V] [--steps S]

runs a fit, a forward and a backward pass and prints times and the distance from the same layer in 32 bits; then S
training steps of LearnedExperts, experts with a gate that learns, which are to name the clusters of a finer fit.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as ftk


class Experts:
    """out[t] = sum over the slots (t, j) of g[t, j] * W[label[t, j]] x[t] with W [E, F, D] packed to 4 bits, once for either direction."""

    def __init__(self, weights, transposed=True):
        self.E, self.F, self.D = weights.shape
        self.W = self.WT = None
        self.pack(weights, transposed)

    def pack(self, weights, transposed=True):
        """Packs the matrices anew, where they were packed before: a captured graph finds them there.  transposed: those that the rows'
        gradient is formed with, too."""
        E, F, D = weights.shape
        self.W = ftk.mx4_quantize(weights.reshape(E * F, D), out=self.W)
        if transposed:
            self.WT = ftk.mx4_quantize(weights.transpose(1, 2).reshape(E * D, F), out=self.WT)

    def _transposed(self):
        return self.WT

    def products(self, x, labels, gates, training=False):
        """Returns (out [N, F], what gradients() needs, or None)."""
        # (the weights' gradient sums over whole steps of the matrix instruction)
        route = ftk.route_plan(labels, self.E, align=128 if training else 1)
        y = ftk.mx4_linear(x, self.W, route=route, gather=True)
        return ftk.route_combine(y, route, gates), (x, y, route, gates) if training else None

    def gradients(self, dout, saved, out_dtype=torch.float32, rows=True):
        """Gradients (dx [N, D], dgates [N, k], dweights [E, F, D] of out_dtype) of sum(dout * out) with labels and gates held fixed;
        rounding to 4 bits counts as the identity.  Without `rows` dx is not formed, and None."""
        x, y, route, gates = saved
        dy, dgates = ftk.route_combine_grad(dout, y, route, gates)
        dx = ftk.route_combine(ftk.mx4_linear(dy, self._transposed(), route=route), route) if rows else None
        gathered = ftk.route_gather(x, route)
        dweights = ftk.mx4_outer(ftk.mx4_quantize(dy, transpose=True), ftk.mx4_quantize(gathered, transpose=True), route, out_dtype=out_dtype)
        return dx, dgates, dweights


class RoutedExperts(Experts):
    """Experts whose tokens go to the matrix of their nearest centroid and to one that all share.

    weights: [K + 1, F, D]: one matrix a cluster, the last one shared.
    width: squared distance at which a cluster's weight has fallen to 1 / e; without one the mean squared distance of the centroids
    from their own mean.  It belongs to the layer: what a token gets does not depend on its batch."""

    def __init__(self, weights, centroids, width=None):
        E, F, D = weights.shape
        if centroids.shape != (E - 1, D):
            raise ValueError("need a matrix for each of the %d centroids and a shared one, got %d" % (centroids.shape[0], E))
        self.centroids = centroids.float().contiguous()
        if width is None:
            width = self._width((self.centroids - self.centroids.mean(0)).square().sum(1), self.centroids)
        if not width > 0:
            raise ValueError("width must be above 0, got %s" % width)
        self.width = float(width)
        super().__init__(weights)

    @classmethod
    def fitted(cls, weights, samples, iters=10, seed=0):
        """The centroids from a Lloyd fit over sample rows, the width their mean squared distance from them."""
        samples = samples.float().contiguous()
        C = ftk.kmeans_fit(samples, weights.shape[0] - 1, iters, seed=seed, want_inertia=False)["C"]
        return cls(weights, C, cls._width(ftk.kmeans_assign(samples, C)[1], C))

    @staticmethod
    def _width(dist, centroids):
        """Mean of squared distances, at least about what 32 bits resolve beside rows as long as the centroids."""
        return max(float(dist.mean()), float(centroids.square().sum(1).mean()) * 2.0 ** -20, torch.finfo(torch.float32).tiny)

    def gate(self, x):
        """labels int32 [N, 2] and weights float [N, 2]."""
        nearest, dist = ftk.kmeans_assign(x.float().contiguous(), self.centroids)
        near = torch.exp(-dist / self.width)
        labels = torch.stack([nearest, torch.full_like(nearest, self.E - 1)], 1)
        return labels, torch.stack([near, 1 - near], 1)

    def forward(self, x, labels=None, gates=None, training=False):
        """Returns (out [N, F], what backward needs, or None)."""
        if labels is None:
            labels, gates = self.gate(x)
        return self.products(x, labels, gates, training)

    def backward(self, dout, saved):
        """Gradients (dx [N, D], dgates [N, 2], dweights [E, F, D] in 32 bits) of sum(dout * out) with labels and gates held fixed;
        rounding to 4 bits counts as the identity.  Where the gates depend on x, as those of gate() do, what reaches x through
        them is not in dx: it is dgates through whatever made them."""
        return self.gradients(dout, saved)


class LearnedExperts(Experts):
    """Experts with a gate that learns, and a loss over many classes: a token goes to the k experts whose logits x Wg^T are largest,
    weighted by the softmax over them, and their sum is held against the classes' vectors.

    gate [E, D], experts [E, F, D], classes [V, F]: weights of one type, float32 or bfloat16, which the layer updates in place
    (AdamW; 16-bit weights beside 32-bit masters, states of `bits` bits).  bias [V] float: of the classes' logits.
    balance: weight of the balance loss.
    The gate's logits come in the rows' type, which near ties of 16-bit rows do not outlast: the lower index is chosen."""

    def __init__(self, gate, experts, classes, k=2, balance=0.01, bits=8, bias=None, **options):
        E, F, D = experts.shape
        if gate.shape != (E, D) or classes.shape[1] != F:
            raise ValueError("need gate [%d, %d] and classes [V, %d], got %s and %s" % (E, D, F, list(gate.shape), list(classes.shape)))
        if not 1 <= k <= E:
            raise ValueError("need 1 <= k <= %d experts, got %d" % (E, k))
        self.gate, self.experts, self.classes, self.k, self.bias, self.options = gate, experts, classes, k, bias, options
        self.state = ftk.AdamW([gate, experts, classes], bits, master=gate.dtype != torch.float32)
        self.count = torch.zeros(1, dtype=torch.int64, device=gate.device)
        self.balance = torch.full((1,), float(balance), device=gate.device)
        super().__init__(experts, transposed=False)

    def _transposed(self):
        """Packed when the rows' gradient is asked for: no step of the layer's own weights needs them."""
        E, F, D = self.experts.shape
        self.WT = ftk.mx4_quantize(self.experts.transpose(1, 2).reshape(E * D, F), out=self.WT)
        return self.WT

    def forward(self, x, training=False):
        """Returns (out [N, F], what gradients of the weights need)."""
        logits = x @ self.gate.t()
        gate, out, saved = self._routed(x, logits, training)
        return out, (logits, gate, saved)

    def _routed(self, x, logits, training):
        gate = ftk.route_gate(logits, self.k)
        return gate, *self.products(x, gate.labels, gate.weights, training)

    def loss(self, x, labels, weights=None, padding=None, rows=False):
        """Returns (sum of the rows' losses by their weights float [N], by default 1 / N; gradients of it and the balance loss by
        gate, experts and classes; the Gate).  Rows with a label outside [0, V) have no loss; they go to their experts and count in
        the balance loss as the others do.  Rows marked in `padding` (bool [N]) and those without a loss that hold NaN or infinities are no tokens:
        nothing of them is looked at, and they do not count.
        rows: a fourth result, the gradient by x [N, D] through experts and gate, for what made the rows."""
        N = x.shape[0]
        logits = x @ self.gate.t()
        # (such an element makes all logits of its row likewise)
        closed = ((labels < 0) | (labels >= self.classes.shape[0])) & ~logits[:, 0].isfinite()
        if padding is not None:
            closed = closed | padding
            labels = labels.masked_fill(padding, -1)
        logits.masked_fill_(closed.unsqueeze(1), float("-inf"))
        x = x.masked_fill(closed.unsqueeze(1), 0)  # (0 * NaN would reach the gate's gradient)
        gate, out, saved = self._routed(x, logits, training=True)
        loss, lse = ftk.xent(out, self.classes, labels, bias=self.bias)
        if weights is None:
            weights = torch.full((N,), 1.0 / max(N, 1), device=x.device)
        dout, dclasses, _ = ftk.xent_grad(out, self.classes, labels, lse, weights, bias=self.bias, need=(True, True, False))
        dx, dgates, dexperts = self.gradients(dout, saved, x.dtype, rows)
        dlogits = ftk.route_gate_grad(logits, gate, dgates, self.balance)
        results = torch.dot(loss, weights), [dlogits.t() @ x, dexperts, dclasses], gate
        return (*results, torch.addmm(dx, dlogits, self.gate)) if rows else results

    def step(self, x, labels, weights=None, padding=None):
        """One update of all weights; returns (loss, Gate)."""
        loss, grads, gate = self.loss(x, labels, weights, padding)
        self.count.add_(1)
        ftk.adamw_step(self.state, grads, self.count, **self.options)
        self.pack(self.experts, transposed=False)
        return loss, gate


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=16384)
    ap.add_argument("--features", type=int, default=1024)
    ap.add_argument("--outputs", type=int, default=2048)
    ap.add_argument("--clusters", type=int, default=15)
    ap.add_argument("--classes", type=int, default=512, help="as many as there are tokens at most")
    ap.add_argument("--steps", type=int, default=20, help="0: no training")
    a = ap.parse_args()
    g = torch.Generator(device="cuda:0").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda:0")  # noqa: E731
    E, D, F, N = a.clusters + 1, a.features, a.outputs, a.tokens
    x = (rand(a.clusters, D)[torch.randint(a.clusters, (N,), generator=g, device="cuda:0")] + 0.5 * rand(N, D)).bfloat16()
    weights = rand(E, F, D) * D ** -0.5
    layer = RoutedExperts.fitted(weights, x[: 64 * E], iters=5)
    labels, gates = layer.gate(x)
    out, saved = layer.forward(x, labels, gates, training=True)
    grads = layer.backward(out, saved)

    def timed(f):
        f()
        b, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        b.record()
        for _ in range(10):
            f()
        e.record()
        torch.cuda.synchronize()
        return b.elapsed_time(e) * 100

    print("%d tokens, %d experts of %d x %d" % (N, E, F, D))
    print("gate %.0f us, forward %.0f us, backward %.0f us" % (
        timed(lambda: layer.gate(x)), timed(lambda: layer.forward(x, labels, gates, training=True)),
        timed(lambda: layer.backward(out, saved))))
    plain = torch.zeros(N, F, device="cuda:0")
    for e in range(E):
        for j in range(2):
            t = torch.nonzero(labels[:, j] == e).flatten()
            plain[t] += gates[t, j].unsqueeze(1) * (x[t].float() @ weights[e].t().contiguous())
    print("from 32-bit matrices and rows: %.3f of the output" % float((out.float() - plain).norm() / plain.norm()))
    print("gradients: " + ", ".join("%s %s" % (list(t.shape), str(t.dtype)[6:]) for t in grads))

    if a.steps < 1:
        return
    # the clusters of a finer fit are the classes that experts with a gate of their own learn to name
    V = min(a.classes, N)
    fine = ftk.kmeans_fit(x.float(), V, 5, seed=1, want_inertia=False)["C"]
    names = ftk.kmeans_assign(x.float(), fine)[0]
    learner = LearnedExperts((rand(E, D) * D ** -0.5).bfloat16(), weights.bfloat16(), (rand(V, F) * F ** -0.5).bfloat16(), lr=1e-3)
    first, gate = learner.step(x, names)
    for _ in range(a.steps - 1):
        last, gate = learner.step(x, names)
    if a.steps > 1:
        print("%d steps towards %d classes: loss %.3f, then %.3f; balance loss %.3f" % (a.steps, V, float(first), float(last), float(gate.loss)))
    print("a training step %.0f us" % timed(lambda: learner.step(x, names)))


if __name__ == "__main__":
    main()
