"""Gate, experts, cross entropy and update put together as a training step uses them, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk, routed_experts
from paper_2408_01391_amd.routed_experts import LearnedExperts
from tests.gpu_util import DEV
from tests.test_gpu_adamw import one_step
from tests.test_gpu_gate import choice, gradient, outputs
from tests.test_gpu_mx4 import pack_of, values, values_of
from tests.test_gpu_route import dev, f64

pytestmark = pytest.mark.gpu


def rounded(x):
    return values_of(*pack_of(x), x.shape[1])


def layer_of(rng, N, D, F, E, V, dtype, **options):
    weights = [dev(rng.standard_normal(s) * s[-1] ** -0.5).to(dtype) for s in ((E, D), (E, F, D), (V, F))]
    x = dev(rng.standard_normal((N, D))).to(dtype)
    labels = dev(rng.integers(0, V, N)).int()
    if N > 4:
        labels[::5] = -1
    return LearnedExperts(*weights, **options), x, labels


@pytest.mark.parametrize("N,D,F,E,V,k", [(300, 96, 40, 6, 50, 2), (37, 130, 260, 9, 333, 3), (1, 64, 64, 4, 7, 1)])
def test_gradients(N, D, F, E, V, k):
    """In 32 bits; every rounding to 4 bits is done by the definition on what the layer itself rounded, and the gate's choice is taken
    from its own logits, so that what is left are the 32-bit roundings of products and sums."""
    rng = np.random.default_rng(N)
    layer, x, labels = layer_of(rng, N, D, F, E, V, torch.float32, k=k, balance=0.5)
    weights = dev(rng.random(N)).float()
    got, (dgate, dexperts, dclasses), gate = layer.loss(x, labels, weights)
    out, (logits, _, (_, y, route, _)) = layer.forward(x, training=True)
    z = f64(logits)
    lab = choice(z, k)
    assert np.array_equal(gate.labels.cpu().numpy(), lab)
    g, _ = outputs(z, lab, gate.counts.cpu().numpy(), True)
    W, order, off = values(layer.W).reshape(E, F, D), route.order.cpu().numpy(), route.offsets.cpu().numpy()
    x4 = rounded(f64(x))
    prod = np.stack([np.stack([W[lab[t, j]] @ x4[t] for j in range(k)]) for t in range(N)])
    want = (g[:, :, None] * prod).sum(1)
    near = lambda a, b, scale: np.abs(a - b).max() <= 2e-5 * scale  # noqa: E731
    assert near(f64(out), want, np.abs(prod).max())
    # the loss from the layer's own outputs on
    C, l, w, live = f64(layer.classes), labels.cpu().numpy(), f64(weights), labels.cpu().numpy() >= 0
    s = f64(out) @ C.T
    lse = np.log(np.exp(s - s.max(1, keepdims=True)).sum(1)) + s.max(1)
    rows = np.where(live, lse - s[np.arange(N), np.maximum(l, 0)], 0)
    assert near(float(got), (w * rows).sum(), (w * np.abs(rows)).sum() + 1)
    d = np.exp(s - lse[:, None])
    d[np.arange(N), np.maximum(l, 0)] -= 1
    d *= np.where(live, w, 0)[:, None]
    dout = d @ C
    assert near(f64(dclasses), d.T @ f64(out), np.abs(f64(out)).max() * np.abs(d).sum(0).max() + 1e-30)
    # through the experts
    slot, held = np.maximum(order, 0), (order >= 0)[:, None]
    dy = np.where(held, g.reshape(-1)[slot][:, None] * dout[slot // k], 0).astype(np.float32).astype(np.float64)
    dg = (dout[:, None, :] * prod).sum(2)
    dz, size = gradient(z, lab, gate.counts.cpu().numpy(), True, dg, 0.5)
    assert near(f64(dgate), dz.T @ f64(x), np.abs(f64(x)).max() * (size.sum(0).max() + np.abs(dout).max() * np.abs(prod).max() * F * N))
    # (4-bit codes of the layer's own dy, which its 32-bit roundings may bring over a border)
    mine, _ = ftk.route_combine_grad(dev(dout).float(), y, route, gate.weights)
    assert near(f64(mine), dy, np.abs(dy).max() + 1e-30)
    a, b = rounded(dy.T), rounded(np.where(held, f64(x)[slot // k], 0).T)
    for e in range(E):
        part = slice(off[e], off[e + 1])
        wide = np.abs(f64(dexperts)[e] - a[:, part] @ b[:, part].T)
        step = np.abs(dy).max() * np.abs(b).max()  # one element of dy that falls into the next code
        assert (wide > 2e-5 * step * max(1, off[e + 1] - off[e])).mean() < 0.02 and wide.max(initial=0) <= step


def test_step_moves_the_weights():
    rng = np.random.default_rng(8)
    for dtype in (torch.float32, torch.bfloat16):
        layer, x, labels = layer_of(rng, 200, 64, 128, 8, 100, dtype, k=2, bits=32, lr=1e-3, weight_decay=0.1)
        _, grads, _ = layer.loss(x, labels)
        before = [f64(p) for p in (layer.state.master or layer.state.params)]
        layer.step(x, labels)
        for p, old, g in zip(layer.state.master or layer.state.params, before, grads):
            m, v, w, change = one_step(old, f64(g), 0 * old, 0 * old, 1, weight_decay=0.1)
            assert (np.abs(f64(p) - w) <= 40 * 2.0 ** -24 * change + 2 * 2.0 ** -24 * np.abs(w)).all()
        assert torch.equal(ftk.mx4_dequantize(layer.W), ftk.mx4_dequantize(ftk.mx4_quantize(layer.experts.reshape(8 * 128, 64))))


def test_captured_step():
    """A whole training step in a graph, replayed: what eager steps give, bit for bit."""
    make = lambda: layer_of(np.random.default_rng(4), 256, 64, 128, 8, 300, torch.bfloat16, k=2, lr=3e-3, seed=5)  # noqa: E731
    (layer, x, labels), (other, _, _) = make(), make()
    layer.step(x, labels), other.step(x, labels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, gate = layer.step(x, labels)
    for turn in range(3):
        if turn:  # (other operands)
            x.copy_(x.flip(0))
            labels.copy_(labels.roll(3))
        graph.replay()
        want, other_gate = other.step(x, labels)
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(gate.counts, other_gate.counts)
        for a, b in zip(layer.state.params + layer.state.master + layer.state.m + layer.state.v,
                        other.state.params + other.state.master + other.state.m + other.state.v):
            assert torch.equal(a, b)


def test_refusals():
    z = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    for call in (lambda: LearnedExperts(z(4, 8), z(4, 6, 9), z(5, 6)), lambda: LearnedExperts(z(4, 8), z(4, 6, 8), z(5, 7)),
                 lambda: LearnedExperts(z(4, 8), z(4, 6, 8), z(5, 6), k=5)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("marked", [True, False])
def test_padding_takes_no_part(marked, dtype):
    """Rows that are no tokens, marked or filled with what nobody wrote: gradients, loss and the gate's counts are those of whatever else
    they hold, and those of the batch without them."""
    N, E, V, keep = 128, 6, 50, 90
    weights = torch.full((N,), 0.01, device=DEV)
    layer, x, labels = layer_of(np.random.default_rng(5), N, 96, 64, E, V, dtype, balance=0.5)
    labels[keep:] = -1
    padding = torch.arange(N, device=DEV) >= keep if marked else None
    if marked:
        labels[keep + 3] = 7  # (a label does not make it a token)
    results = []
    for fill in (float("nan"), float("inf"), -float("inf")) + ((0.0, 3.0) if marked else ()):
        x[keep:] = fill
        results.append(layer.loss(x, labels, weights, padding))
    results.append(layer.loss(x[:keep].contiguous(), labels[:keep].contiguous(), weights[:keep].contiguous()))
    loss, grads, gate = results[0]
    assert loss.isfinite() and all(g.isfinite().all() for g in grads) and int(gate.counts[-1]) == keep
    assert (gate.labels[keep:] == -1).all() and (gate.weights[keep:] == 0).all()
    for other, others, that in results[1:-1]:
        assert torch.equal(loss, other) and torch.equal(gate.counts, that.counts) and all(torch.equal(a, b) for a, b in zip(grads, others))
    # fewer rows may be added up in another order: 32-bit sums, and in 16 bits a step of the result
    other, others, that = results[-1]
    assert torch.equal(gate.counts, that.counts) and abs(float(loss - other)) <= 1e-5 * abs(float(other))
    for a, b in zip(grads, others):
        assert (f64(a) - f64(b)).__abs__().max() <= (2e-5 if dtype == torch.float32 else 2.0 ** -7) * np.abs(f64(b)).max()


def test_rows_without_a_loss_count_in_the_balance():
    """Tokens without a class are routed like others; one with a class that holds NaN shows in the balance loss and in the gate."""
    layer, x, labels = layer_of(np.random.default_rng(6), 64, 96, 64, 6, 50, torch.float32)
    labels[:] = torch.arange(64, device=DEV, dtype=torch.int32) % 50
    labels[::2] = -1
    _, _, gate = layer.loss(x, labels)
    assert int(gate.counts[-1]) == 64 and (gate.labels >= 0).all()
    x[1] = float("nan")
    loss, grads, gate = layer.loss(x, labels)
    assert gate.loss.isnan().all() and grads[0].isnan().any() and int(gate.counts[-1]) == 64
    padding = torch.zeros(64, dtype=torch.bool, device=DEV)
    padding[1] = True
    loss, _ = layer.step(x, labels, padding=padding)
    assert loss.isfinite() and all(p.isfinite().all() for p in layer.state.params)


@pytest.mark.parametrize("N,D,F,E,V,k", [(300, 96, 40, 6, 50, 2), (37, 130, 260, 9, 333, 3), (1, 64, 64, 4, 7, 1)])
def test_gradient_of_the_rows(N, D, F, E, V, k):
    """What a net in front of the layer gets: through the experts' matrices and through the gate, after a step, in 32 bits."""
    rng = np.random.default_rng(N + 1)
    layer, x, labels = layer_of(rng, N, D, F, E, V, torch.float32, k=k, balance=0.5, lr=1e-2)
    assert layer.WT is None  # (no step asks for it)
    layer.step(x, labels)
    plain = layer.loss(x, labels)
    loss, grads, gate, dx = layer.loss(x, labels, rows=True)
    assert torch.equal(loss, plain[0]) and all(torch.equal(a, b) for a, b in zip(grads, plain[1]))
    out, (logits, _, (_, y, route, _)) = layer.forward(x, training=True)
    _, lse = ftk.xent(out, layer.classes, labels)
    dout, _, _ = ftk.xent_grad(out, layer.classes, labels, lse, torch.full((N,), 1.0 / N, device=DEV))
    dy, dg = ftk.route_combine_grad(dout, y, route, gate.weights)
    WT = values_of(*pack_of(f64(layer.experts).transpose(0, 2, 1).reshape(E * D, F)), F).reshape(E, D, F)
    slots, off, order = rounded(f64(dy)), route.offsets.cpu().numpy(), route.order.cpu().numpy()
    want, size = np.zeros((N, D)), np.zeros((N, D))
    for e in range(E):
        for row in range(off[e], off[e + 1]):
            if order[row] >= 0:
                want[order[row] // k] += WT[e] @ slots[row]
                size[order[row] // k] += abs(WT[e]) @ abs(slots[row])
    dz, dsize = gradient(f64(logits), gate.labels.cpu().numpy(), gate.counts.cpu().numpy(), True, f64(dg), 0.5)
    want, size = want + dz @ f64(layer.gate), size + dsize @ abs(f64(layer.gate))
    # sums of F and of E products and of the slots; p within (80 + 12 + E) steps, four times
    assert (abs(f64(dx) - want) <= (F + E + k + 16 + 4 * (92 + E)) * 2.0 ** -24 * size + 1e-30).all()
    assert (f64(dx)[labels.cpu().numpy() < 0] != 0).any() or N == 1  # (by the balance)
    # the inherited call has it, too
    assert torch.equal(layer.gradients(dout, (x, y, route, gate.weights))[0], ftk.route_combine(ftk.mx4_linear(dy, layer.WT, route=route), route))


def test_gradient_of_the_rows_in_16_bits():
    """In the rows' type; rows that are no tokens get zeros."""
    layer, x, labels = layer_of(np.random.default_rng(9), 70, 96, 40, 6, 50, torch.bfloat16)
    x[60:] = float("nan")
    labels[60:] = -1
    dx = layer.loss(x, labels, rows=True)[3]
    assert dx.dtype == x.dtype and dx.shape == x.shape and dx.isfinite().all() and (dx[60:] == 0).all() and (dx[:60] != 0).any(1).all()


@pytest.mark.parametrize("options,trained", [("--tokens 300 --features 64 --outputs 64 --clusters 3 --steps 2", 300),
                                             ("--tokens 20 --features 64 --outputs 64 --clusters 3 --steps 1", 20),
                                             ("--tokens 300 --features 64 --outputs 64 --clusters 3 --classes 7 --steps 3", 7),
                                             ("--tokens 300 --features 64 --outputs 64 --clusters 3 --steps 0", None)])
def test_command(options, trained, monkeypatch, capsys):
    """Fewer tokens than there are classes by default, and no steps: what ran without the training runs."""
    monkeypatch.setattr("sys.argv", ["routed_experts", *options.split()])
    routed_experts.main()
    said = capsys.readouterr().out
    assert "gradients: " in said
    assert ("a training step" in said) == (trained is not None)
    if trained and "--steps 1" not in options:
        assert "towards %d classes" % trained in said
