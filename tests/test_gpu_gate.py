"""The gate over experts and its gradient against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
INF = np.inf


def f64(t):
    return t.detach().double().cpu().numpy()


def probabilities(z):
    top = z.max(1, initial=-INF, keepdims=True)
    with np.errstate(invalid="ignore"):
        e = np.where(z == -INF, 0, np.exp(z - np.where(top == -INF, 0, top)))
        s = e.sum(1, keepdims=True)
        return e / np.where(s == 0, 1, s), np.where(s[:, 0] > 0, top[:, 0] + np.log(np.where(s[:, 0] > 0, s[:, 0], 1)), -INF)


def choice(z, k):
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(z, order, 1) == -INF, -1, order)


def outputs(z, labels, counts, normalise):
    """weights and loss with labels and counts held fixed (counts [E + 1])."""
    E, k, T = z.shape[1], labels.shape[1], max(1, counts[-1])
    p, _ = probabilities(z)
    w = np.where(labels >= 0, np.take_along_axis(p, np.maximum(labels, 0), 1), 0)
    if normalise:
        s = w.sum(1, keepdims=True)
        w = w / np.where(s == 0, 1, s)
    return w, E * float((counts[:-1] / (k * T) * (p.sum(0) / T)).sum())


def gradient(z, labels, counts, normalise, dw, dloss):
    """The formula, and the sum of its terms' magnitudes."""
    N, E = z.shape
    k, T = labels.shape[1], max(1, counts[-1])
    p, _ = probabilities(z)
    w, _ = outputs(z, labels, counts, normalise)
    c = dloss * E * counts[:-1] / (k * T) / T
    dz = p * (c - (p * c).sum(1, keepdims=True))
    size = p * (abs(c) + (p * abs(c)).sum(1, keepdims=True))
    inner = (w * dw).sum(1, keepdims=True)
    held = labels >= 0
    at = np.maximum(labels, 0)
    for j in range(k):
        part = w[:, j] * (dw[:, j] - (inner[:, 0] if normalise else 0))
        np.add.at(dz, (np.arange(N), at[:, j]), np.where(held[:, j], part, 0))
        np.add.at(size, (np.arange(N), at[:, j]), np.where(held[:, j], w[:, j] * (abs(dw[:, j]) + (w * abs(dw)).sum(1)), 0))
    if not normalise:
        dz -= p * inner
        size += p * (w * abs(dw)).sum(1, keepdims=True)
    return dz, size


def logits_of(rng, N, E, dtype, masked):
    z = 2 * rng.standard_normal((N, E)) + rng.standard_normal(E)
    z[rng.random((N, E)) < 0.2] = 0.5  # ties
    z[rng.random((N, E)) < 0.05] = -0.0
    if masked:
        z[rng.random((N, E)) < 0.3] = -INF
        z[N // 2] = -INF
        z[N // 3, :-1] = -INF
    return torch.from_numpy(z).to(DEV).to(dtype)


def relative(E):
    """A probability is off by: its exponent, of at most 40 (these logits), which takes two roundings, 2 * 40 * 2^-24; the
    exponential, logarithm, sum (an element goes through E / 4 / 4 + 8 additions at most) and division."""
    return (80 + min(E, 136) + 12) * 2.0 ** -24


CASES = [(1, 1, 1), (1, 64, 2), (2, 8192, 64), (3, 5, 5), (17, 16, 4), (63, 31, 16), (64, 32, 2), (65, 33, 3), (130, 64, 8), (77, 65, 17),
         (200, 129, 8), (150, 513, 64), (70, 1030, 7), (40, 2100, 2), (7, 4097, 5), (5, 8191, 2), (3000, 77, 3), (1500, 256, 8)]


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k", CASES)
def test_gate_and_gradient(N, E, k, dtype, normalise):
    rng = np.random.default_rng(N * 10 + E)
    t = TYPES[dtype]
    logits = logits_of(rng, N, E, t, masked=N % 2 == 0 or N > 1000)
    z = f64(logits)
    gate = ftk.route_gate(logits, k, normalise=normalise)
    labels = choice(z, k)
    assert np.array_equal(gate.labels.cpu().numpy(), labels)
    p, lse = probabilities(z)
    held = labels[labels >= 0]
    counts = np.concatenate([np.bincount(held, minlength=E), [(lse > -INF).sum()]])
    assert np.array_equal(gate.counts.cpu().numpy(), counts)
    w, loss = outputs(z, labels, counts, normalise)
    tol = relative(E)
    assert (abs(f64(gate.weights) - w) <= 3 * tol * w).all()
    assert np.array_equal(f64(gate.lse) == -INF, lse == -INF)
    some = lse > -INF
    assert (abs(f64(gate.lse)[some] - lse[some]) <= tol + 2.0 ** -23 * abs(lse[some])).all()
    mean = p.sum(0) / max(1, counts[-1])
    # sums over rows: a lane's own N / 64 at the least often, then lines of sums; all terms are positive
    rows = (N + 40) * 2.0 ** -24
    assert (abs(f64(gate.probs) - mean) <= (tol + rows) * mean + 1e-38).all()
    assert abs(float(gate.loss) - loss) <= (tol + rows + 2.0 ** -23) * loss
    dw, dloss = rng.standard_normal((N, k)).astype(np.float32), np.float32(0.3 * N)
    args = torch.from_numpy(dw).to(DEV), torch.full((1,), float(dloss), device=DEV)
    for use in ((0, 1), (0,), (1,)):
        got = ftk.route_gate_grad(logits, gate, args[0] if 0 in use else None, args[1] if 1 in use else None)
        want, size = gradient(z, labels, counts, normalise, dw if 0 in use else 0 * dw, float(dloss) if 1 in use else 0.0)
        assert got.dtype == t
        # the smallest normal fp16 numbers' half step beside the relative one
        tiny = 2.0 ** -25 if t == torch.float16 else 1e-38
        assert (abs(f64(got) - want) <= 4 * tol * size + HALF[t] * abs(want) * 1.01 + tiny).all()


@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(normalise):
    """The formula that the kernels are held to, by central differences of weights and loss in 64 bits."""
    rng = np.random.default_rng(5)
    N, E, k, h = 6, 9, 3, 1e-6
    z = rng.standard_normal((N, E))
    z[1, 4] = z[2, 0] = -INF
    labels = choice(z, k)
    counts = np.concatenate([np.bincount(labels.reshape(-1), minlength=E), [N]])
    dw, dloss = rng.standard_normal((N, k)), 1.7
    want, _ = gradient(z, labels, counts, normalise, dw, dloss)
    value = lambda z: (lambda w, loss: (w * dw).sum() + dloss * loss)(*outputs(z, labels, counts, normalise))  # noqa: E731
    for n in range(N):
        for e in range(E):
            if z[n, e] == -INF:
                assert want[n, e] == 0
                continue
            up, down = z.copy(), z.copy()
            up[n, e] += h
            down[n, e] -= h
            assert abs((value(up) - value(down)) / (2 * h) - want[n, e]) < 1e-8


def test_bad_rows_show():
    z = torch.randn(70, 40, device=DEV)
    z[3, 7] = float("nan")
    z[9, 0] = float("inf")
    z[20] = float("nan")
    for dtype in TYPES.values():
        gate = ftk.route_gate(z.to(dtype), 3)
        bad = torch.zeros(70, dtype=torch.bool, device=DEV)
        bad[[3, 9, 20]] = True
        assert (gate.labels[bad] == -1).all() and gate.weights[bad].isnan().all() and gate.lse[bad].isnan().all()
        assert (gate.labels[~bad] >= 0).all() and gate.weights[~bad].isfinite().all()
        assert gate.probs.isnan().all() and gate.loss.isnan().all()
        assert int(gate.counts[-1]) == 70 and int(gate.counts[:-1].sum()) == 67 * 3


@pytest.mark.parametrize("N", [0, 5, 100])
def test_rows_closed_to_all(N):
    z = torch.full((N, 12), -INF, device=DEV)
    gate = ftk.route_gate(z, 2)
    assert (gate.labels == -1).all() and (gate.weights == 0).all() and (gate.lse == -INF).all()
    assert (gate.counts == 0).all() and (gate.probs == 0).all() and float(gate.loss) == 0
    if N:
        assert (ftk.route_gate_grad(z, gate, torch.ones(N, 2, device=DEV), torch.ones(1, device=DEV)) == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_offsets_places(dtype):
    """Rows of a wider array at an odd address, results in arrays of the caller, the gradient in the logits' place."""
    N, E, k, t = 321, 70, 4, TYPES[dtype]
    g = torch.Generator(device=DEV).manual_seed(3)
    wide = torch.randn(N, 97, generator=g, device=DEV).to(t)
    z = wide[:, 3:3 + E]
    dw, dl = torch.randn(N, k, generator=g, device=DEV), torch.ones(1, device=DEV)
    plain = ftk.route_gate(z.contiguous(), k)
    dz = ftk.route_gate_grad(z.contiguous(), plain, dw, dl)
    own = ftk.Gate(*[torch.full_like(getattr(plain, n), 7) for n in ("labels", "weights", "lse", "counts", "probs", "loss")], True)
    need = ftk.route_gate_workspace_bytes(N, E)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    got = ftk.route_gate(z, k, gate=own, workspace=ws)
    for n in ("labels", "weights", "lse", "counts", "probs", "loss"):
        assert torch.equal(getattr(got, n), getattr(plain, n)), n
    before = wide.clone()
    assert ftk.route_gate_grad(z, got, dw, dl, out=z) is z
    assert torch.equal(z, dz)
    wide[:, 3:3 + E] = before[:, 3:3 + E]
    assert torch.equal(wide, before)  # nothing beside the rows


def test_graph_and_streams():
    """Captured once, replayed on other logits with eager calls between: the eager results every time."""
    N, E, k = 700, 48, 4
    g = torch.Generator(device=DEV).manual_seed(9)
    z = torch.randn(N, E, generator=g, device=DEV).bfloat16()
    dw, dl = torch.randn(N, k, generator=g, device=DEV), torch.ones(1, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ftk.route_gate(z, k)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gate = ftk.route_gate(z, k)
        plan = ftk.route_plan(gate.labels, E)
        dz = ftk.route_gate_grad(z, gate, dw, dl)
    for turn in range(4):
        z.copy_(torch.randn(N, E, generator=g, device=DEV))
        graph.replay()
        eager = ftk.route_gate(z, k)
        assert torch.equal(gate.labels, eager.labels) and torch.equal(gate.weights, eager.weights)
        assert torch.equal(gate.loss, eager.loss) and torch.equal(gate.counts, eager.counts)
        assert torch.equal(plan.counts, eager.counts[:E])
        assert torch.equal(dz, ftk.route_gate_grad(z, eager, dw, dl))
        torch.cuda.synchronize()


def test_rows_far_apart():
    """Row strides of 2^31 elements, and a million rows."""
    for dtype in TYPES.values():
        far = torch.empty((1 << 32) + 64, dtype=dtype, device=DEV)
        z = far.as_strided((3, 20), (1 << 31, 1))
        z.copy_(torch.randn(3, 20, device=DEV))
        a, b = ftk.route_gate(z, 3), ftk.route_gate(z.contiguous(), 3)
        assert torch.equal(a.labels, b.labels) and torch.equal(a.loss, b.loss)
        dw, dl = torch.randn(3, 3, device=DEV), torch.ones(1, device=DEV)
        want = ftk.route_gate_grad(z.contiguous(), b, dw, dl)
        assert torch.equal(ftk.route_gate_grad(z, a, dw, dl, out=z), want)
        del far, z
    z = torch.randn(1 << 20, 8, device=DEV)
    gate = ftk.route_gate(z, 2)
    top = z.double().topk(2, dim=1)
    assert torch.equal(gate.labels.long(), top.indices) and int(gate.counts[-1]) == 1 << 20
    p = torch.softmax(z.double(), 1).mean(0)
    assert ((gate.probs.double() - p).abs() <= 1e-5 * p).all()
    assert torch.equal(gate.counts[:-1].long(), torch.bincount(gate.labels.flatten(), minlength=8))


def test_calls_at_once():
    """Two streams, each with its own workspace."""
    g = torch.Generator(device=DEV).manual_seed(11)
    zs = [torch.randn(3000, 100, generator=g, device=DEV) for _ in range(2)]
    want = [ftk.route_gate(z, 4) for z in zs]
    streams = [torch.cuda.Stream() for _ in zs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for z, st in zip(zs, streams):
            with torch.cuda.stream(st):
                got.append(ftk.route_gate(z, 4))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("labels", "weights", "lse", "counts", "probs", "loss"))


def test_counts_of_several_parts():
    """Counts summed over parts of a batch give every part the whole batch's gradient."""
    g = torch.Generator(device=DEV).manual_seed(4)
    z = torch.randn(500, 20, generator=g, device=DEV)
    dl = torch.ones(1, device=DEV)
    whole = ftk.route_gate(z, 2)
    want = ftk.route_gate_grad(z, whole, None, dl)
    parts = [ftk.route_gate(z[:200], 2), ftk.route_gate(z[200:], 2)]
    counts = parts[0].counts + parts[1].counts
    assert torch.equal(counts, whole.counts)
    for part, at in zip(parts, (slice(0, 200), slice(200, 500))):
        part.counts.copy_(counts)
        assert torch.equal(ftk.route_gate_grad(z[at], part, None, dl), want[at])


def test_refusals():
    z = torch.zeros(4, 8, device=DEV)
    gate = ftk.route_gate(z, 2)
    for call in (lambda: ftk.route_gate(z, 0), lambda: ftk.route_gate(z, 9), lambda: ftk.route_gate(z.t(), 2),
                 lambda: ftk.route_gate(z, 3, gate=gate), lambda: ftk.route_gate_grad(z, gate, torch.zeros(4, 3, device=DEV)),
                 lambda: ftk.route_gate_grad(z, gate, None, torch.zeros(2, device=DEV)),
                 lambda: ftk.route_gate_grad(z[:3], gate, torch.zeros(3, 2, device=DEV))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ftk.route_gate(z.double(), 2)
    with pytest.raises(ftk.FtkError):
        ftk.route_gate_grad(z, gate)


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k", [(9, 5, 2), (70, 64, 4), (300, 65, 8), (33, 600, 9), (6, 2100, 2), (5, 8192, 64)])
def test_masks_of_the_lowest_value(N, E, k, dtype, normalise):
    """Experts masked by the type's lowest value: long runs of them, all but one, and whole rows, whose experts are all alike."""
    rng = np.random.default_rng(N + E)
    t = TYPES[dtype]
    logits = logits_of(rng, N, E, t, masked=False)
    low = torch.finfo(t).min
    logits[::2, E // 4:] = low
    logits[1, :-1] = low
    logits[2] = low
    logits[N - 1, : E // 2 + 1] = low
    logits[4] = 1e4  # (equal ones as large as fp16 holds)
    z = f64(logits)
    gate = ftk.route_gate(logits, k, normalise=normalise)
    labels = choice(z, k)
    assert np.array_equal(gate.labels.cpu().numpy(), labels)
    p, lse = probabilities(z)
    counts = np.concatenate([np.bincount(labels.ravel(), minlength=E), [N]])
    assert np.array_equal(gate.counts.cpu().numpy(), counts)
    w, loss = outputs(z, labels, counts, normalise)
    tol = relative(E)
    assert (abs(f64(gate.weights) - w) <= 3 * tol * w).all()
    assert (abs(f64(gate.lse) - lse) <= tol + 2.0 ** -23 * abs(lse)).all()
    assert abs(float(gate.loss) - loss) <= (4 * tol + (N + 40) * 2.0 ** -24) * loss
    dw = torch.from_numpy(rng.standard_normal((N, k))).to(DEV).float()
    dloss = torch.tensor([0.7], device=DEV)
    dz = ftk.route_gate_grad(logits, gate, dw, dloss)
    want, size = gradient(z, labels, counts, normalise, f64(dw), 0.7)
    # as elsewhere; a probability divided by the sum of them (E / 16 additions in a lane at most) is off by its rounding besides
    assert (abs(f64(dz) - want) <= (6 * tol + (E / 16 + 16) * 2.0 ** -24) * size + HALF[t] * abs(want) * 1.01 + 2.0 ** -25).all()


@pytest.mark.parametrize("N,E,k,lanes", [(300, 8, 2, 4), (200, 16, 4, 4), (70, 64, 8, 16)])
def test_gradient_of_32_bit_logits_far_from_zero(N, E, k, lanes):
    """Logits between 33 and 62, where lse is off by up to 2^-19: the balance loss' gradient of a row adds up to 0 within the roundings of
    its own sums, which are less."""
    rng = np.random.default_rng(E)
    z = (rng.uniform(33, 58, (N, 1)) + rng.uniform(0, 2, (N, E))).astype(np.float32)
    logits = torch.from_numpy(z).to(DEV)
    gate = ftk.route_gate(logits, k)
    p, lse = probabilities(z.astype(np.float64))
    assert (lse > 33).all() and (lse < 64).all()
    dloss, counts = float(np.float32(0.3 * N)), gate.counts.cpu().numpy()
    got = f64(ftk.route_gate_grad(logits, gate, None, torch.full((1,), dloss, device=DEV)))
    mean = (p * (dloss * E * counts[:-1] / (k * N) / N)).sum(1)
    # p: four terms of a lane and the lanes' are added, divided and multiplied; <p, c>: as many additions; the difference and the last
    # product: a half step (2^-24) each of p |c - <p, c>|, whose sum is at most twice <p, c>
    steps = 2 * (4 + np.log2(lanes)) + 2 + 4 + 1
    assert steps < 32
    assert (abs(got.sum(1)) <= steps * 2.0 ** -24 * mean).all()


class Elsewhere(torch.Tensor):
    """A tensor that says it lives on another device."""

    def get_device(self):
        return torch.cuda.current_device() + 1


def test_arrays_on_another_device():
    z = torch.randn(300, 70, device=DEV)
    names = ("labels", "weights", "lse", "counts", "probs", "loss")
    for name in names:
        gate = ftk.route_gate(z, 2)
        setattr(gate, name, getattr(gate, name).as_subclass(Elsewhere))
        before = getattr(gate, name).clone()
        with pytest.raises(ValueError, match="device"):
            ftk.route_gate(-z, 2, normalise=False, gate=gate)
        assert gate.normalise and torch.equal(getattr(gate, name), before)
        if name not in ("probs", "loss"):
            with pytest.raises(ValueError, match="device"):
                ftk.route_gate_grad(z, gate, torch.ones(300, 2, device=DEV))
    gate = ftk.route_gate(z, 2)
    with pytest.raises(ValueError, match="device"):
        ftk.route_gate(z.as_subclass(Elsewhere), 2)
    with pytest.raises(ValueError, match="device"):
        ftk.route_gate_grad(z, gate, torch.ones(300, 2, device=DEV).as_subclass(Elsewhere))
