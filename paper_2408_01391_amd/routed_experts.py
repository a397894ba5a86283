"""Experts by clusters: a layer whose tokens go through the matrix of their nearest centroid, forward and backward.

The centroids come from a Lloyd fit over sample rows.  A token has two slots: the matrix of its cluster, weighted by
how near the centroid is, and one that all tokens share.  The matrices are held in 4 bits.

    python -m paper_2408_01391_amd.routed_experts [--tokens N] [--features D] [--outputs F] [--clusters K]

runs a fit, a forward and a backward pass and prints times and the distance from the same layer in 32 bits.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as ftk


class RoutedExperts:
    """out[t] = sum over the slots (t, j) of g[t, j] * W[label[t, j]] x[t] with W packed to 4 bits.

    weights: [K + 1, F, D]: one matrix a cluster, the last one shared.  Packed once for either direction.
    width: squared distance at which a cluster's weight has fallen to 1 / e; without one the mean squared distance of the centroids
    from their own mean.  It belongs to the layer: what a token gets does not depend on its batch."""

    def __init__(self, weights, centroids, width=None):
        E, F, D = weights.shape
        if centroids.shape != (E - 1, D):
            raise ValueError("need a matrix for each of the %d centroids and a shared one, got %d" % (centroids.shape[0], E))
        self.E, self.F, self.D = E, F, D
        self.centroids = centroids.float().contiguous()
        if width is None:
            width = self._width((self.centroids - self.centroids.mean(0)).square().sum(1), self.centroids)
        if not width > 0:
            raise ValueError("width must be above 0, got %s" % width)
        self.width = float(width)
        self.W = ftk.mx4_quantize(weights.reshape(E * F, D))
        self.WT = ftk.mx4_quantize(weights.transpose(1, 2).reshape(E * D, F))

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
        # (the weights' gradient sums over whole steps of the matrix instruction)
        route = ftk.route_plan(labels, self.E, align=128 if training else 1)
        y = ftk.mx4_linear(x, self.W, route=route, gather=True)
        return ftk.route_combine(y, route, gates), (x, y, route, gates) if training else None

    def backward(self, dout, saved):
        """Gradients (dx [N, D], dgates [N, 2], dweights [E, F, D] in 32 bits) of sum(dout * out) with labels and gates held fixed;
        rounding to 4 bits counts as the identity.  Where the gates depend on x, as those of gate() do, what reaches x through
        them is not in dx: it is dgates through whatever made them."""
        x, y, route, gates = saved
        dy, dgates = ftk.route_combine_grad(dout, y, route, gates)
        dx = ftk.route_combine(ftk.mx4_linear(dy, self.WT, route=route), route)
        rows = ftk.route_gather(x, route)
        dweights = ftk.mx4_outer(ftk.mx4_quantize(dy, transpose=True), ftk.mx4_quantize(rows, transpose=True), route)
        return dx, dgates, dweights


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=16384)
    ap.add_argument("--features", type=int, default=1024)
    ap.add_argument("--outputs", type=int, default=2048)
    ap.add_argument("--clusters", type=int, default=15)
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


if __name__ == "__main__":
    main()
