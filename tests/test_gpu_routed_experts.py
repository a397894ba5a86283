"""The layer that puts routing and 4-bit products together, against its formula in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from paper_2408_01391_amd.routed_experts import RoutedExperts
from tests.gpu_util import DEV
from tests.test_gpu_mx4 import pack_of, values, values_of
from tests.test_gpu_route import dev, f64

pytestmark = pytest.mark.gpu


def rounded(x):
    return values_of(*pack_of(x), x.shape[1])


@pytest.mark.parametrize("N,D,F,K", [(300, 96, 40, 5), (37, 130, 260, 3), (1, 64, 64, 2)])
def test_layer(N, D, F, K):
    """In 32 bits, with every rounding to 4 bits done by the definition on what the layer itself rounded: what is left are the 32-bit
    roundings of its products and sums, some hundred of 2^-24 of the magnitudes."""
    rng = np.random.default_rng(N)
    centres = rng.standard_normal((K, D)) * 3
    x = dev(centres[rng.integers(0, K, N)] + 0.3 * rng.standard_normal((N, D))).float()
    weights = dev(rng.standard_normal((K + 1, F, D)) * D ** -0.5).float()
    layer = RoutedExperts(weights, dev(centres).float())
    labels, gates = layer.gate(x)
    assert np.array_equal(labels[:, 0].cpu().numpy(), ((f64(x)[:, None] - centres.astype(np.float32)) ** 2).sum(2).argmin(1))
    out, saved = layer.forward(x, labels, gates, training=True)
    dout = dev(rng.standard_normal((N, F))).float()
    dx, dgates, dweights = layer.backward(dout, saved)
    _, y, route, _ = saved
    W, WT = values(layer.W).reshape(K + 1, F, D), values(layer.WT).reshape(K + 1, D, F)
    lab, g, order, off = labels.cpu().numpy(), f64(gates), route.order.cpu().numpy(), route.offsets.cpu().numpy()
    slot = np.maximum(order, 0)
    held = (order >= 0)[:, None]
    prod = np.stack([np.stack([W[lab[t, j]] @ rounded(f64(x))[t] for j in range(2)]) for t in range(N)])
    near = lambda got, want, scale: np.abs(got - want).max() <= 1e-5 * scale  # noqa: E731
    assert near(f64(out), (g[:, :, None] * prod).sum(1), np.abs(prod).max())
    assert near(f64(dgates), (f64(dout)[:, None, :] * prod).sum(2), np.abs(prod).max() * F)
    dy = np.where(held, g.reshape(-1)[slot][:, None] * f64(dout)[slot // 2], 0).astype(np.float32).astype(np.float64)
    rows = np.where(held, f64(x)[slot // 2], 0)
    dy4 = rounded(dy)
    want = np.zeros((N, D))
    for e in range(K + 1):
        for p in range(off[e], off[e + 1]):
            if order[p] >= 0:
                want[order[p] // 2] += WT[e] @ dy4[p]
    assert near(f64(dx), want, np.abs(want).max() + np.abs(WT).max() * np.abs(dy4).max())
    a, b = rounded(dy.T), rounded(rows.T)
    for e in range(K + 1):
        part = slice(off[e], off[e + 1])
        assert near(f64(dweights)[e], a[:, part] @ b[:, part].T, np.abs(a).max() * np.abs(b).max() * max(1, off[e + 1] - off[e]))
    # without a gradient to come, rows are not filled up: the same results
    again, _ = layer.forward(x, labels, gates)
    assert torch.equal(again, out)


def test_fitted_router_and_refusals():
    rng = np.random.default_rng(2)
    x = dev(rng.standard_normal((500, 32))).float()
    weights = dev(rng.standard_normal((5, 16, 32))).float()
    layer = RoutedExperts.fitted(weights, x, iters=3)
    out, saved = layer.forward(x)
    assert out.shape == (500, 16) and saved is None and torch.isfinite(out).all()
    with pytest.raises(ValueError):
        RoutedExperts(weights, x[:7])
    assert ftk.mx4_dequantize(layer.W).shape == (80, 32)
    assert DEV.type == "cuda"


def test_gate_on_the_centroids():
    """Tokens that all lie on their centroids: their weight is 1, not 0 / 0."""
    centres = dev(np.arange(24).reshape(3, 8) % 7 * 3.0).float()
    weights = dev(np.random.default_rng(3).standard_normal((4, 16, 8))).float()
    x = centres[torch.tensor([0, 2, 2, 1], device=DEV)]
    for layer in (RoutedExperts(weights, centres), RoutedExperts(weights, centres, width=4.0), RoutedExperts.fitted(weights, centres, iters=2),
                  RoutedExperts(weights[:2], torch.zeros(1, 8, device=DEV))):
        y = x if layer.E == 4 else torch.zeros(4, 8, device=DEV)
        labels, gates = layer.gate(y)
        assert torch.equal(gates, torch.tensor([[1.0, 0.0]] * 4, device=DEV))
        assert torch.isfinite(layer.forward(y)[0]).all()


def test_gate_of_a_token_does_not_depend_on_its_batch():
    """Small whole numbers, whose distances are exact in 32 bits: exp(-distance / width), in a batch and alone."""
    rng = np.random.default_rng(8)
    K, N, D = 5, 60, 64
    centres = rng.integers(-4, 5, (K, D)).astype(np.float32)
    x = centres[rng.integers(0, K, N)] + rng.integers(-1, 2, (N, D)).astype(np.float32) * (np.arange(N)[:, None] % 3)
    weights = dev(rng.standard_normal((K + 1, 24, D))).float()
    nearest = ((x[:, None].astype(np.float64) - centres) ** 2).sum(2).min(1)
    for layer in (RoutedExperts(weights, dev(centres)), RoutedExperts(weights, dev(centres), width=50.0)):
        labels, gates = layer.gate(dev(x))
        want = np.exp(-nearest / layer.width)
        # one rounding of the quotient (2^-24 of at most 104, beyond which the weight is 0) and of the exponential
        assert np.abs(f64(gates) - np.stack([want, 1 - want], 1)).max() <= 104 * 2.0 ** -23
        for t in range(0, N, 7):
            one = layer.gate(dev(x[t:t + 1]))
            assert torch.equal(one[0], labels[t:t + 1]) and torch.equal(one[1], gates[t:t + 1])
    fitted = RoutedExperts.fitted(weights, dev(x), iters=4)
    spread = ((x[:, None].astype(np.float64) - f64(fitted.centroids)) ** 2).sum(2).min(1).mean()
    assert abs(fitted.width - spread) <= 1e-4 * spread
    for width in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            RoutedExperts(weights, dev(centres), width=width)


def test_backward_holds_the_gates_fixed():
    """The layer's own gates give the same gradients as the same gates given, and dgates is what the gates' own gradient starts from:
    moving them moves sum(dout * out) by that much, the sum being linear in them."""
    rng = np.random.default_rng(12)
    N, D, F, K = 90, 64, 48, 4
    centres = dev(rng.standard_normal((K, D)) * 2).float()
    layer = RoutedExperts(dev(rng.standard_normal((K + 1, F, D)) * 0.1).float(), centres)
    x = centres[dev(rng.integers(0, K, N))] + dev(rng.standard_normal((N, D)) * 0.3).float()
    dout = dev(rng.standard_normal((N, F))).float()
    labels, gates = layer.gate(x)
    out, saved = layer.forward(x, training=True)
    own, given = layer.backward(dout, saved), layer.backward(dout, layer.forward(x, labels, gates, training=True)[1])
    for a, b in zip(own, given):
        assert torch.equal(a, b) and not a.requires_grad
    step = dev(rng.standard_normal((N, 2)) * 0.5).float()
    moved = layer.forward(x, labels, gates + step)[0]
    by = (f64(dout) * (f64(moved) - f64(out))).sum()
    want, size = (f64(own[1]) * f64(step)).sum(), (np.abs(f64(dout)) @ np.abs(f64(moved)).T).max() * N
    assert abs(by - want) <= 1e-5 * size
