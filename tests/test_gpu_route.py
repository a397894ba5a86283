"""Rows sorted by label and back (ftk_route_*) against plain numpy in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, and the smallest step, of a type
UNIT = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
STEP = {"f32": 2.0 ** -149, "f64": 0.0, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def plan_of(labels, E, align, rows):
    """offsets, counts, order, pos by the definition."""
    N, k = labels.shape
    flat = labels.reshape(-1).astype(np.int64)
    slots = [np.flatnonzero(flat == e) for e in range(E)] if E < 200 else None
    counts = np.bincount(flat[(flat >= 0) & (flat < E)], minlength=E)
    offsets = np.concatenate([[0], np.cumsum((counts + align - 1) // align * align)])
    order, pos = np.full(rows, -1), np.full(N * k, -1)
    if slots is None:
        inside = np.flatnonzero((flat >= 0) & (flat < E))
        by = inside[np.argsort(flat[inside], kind="stable")]
        at = offsets[flat[by]] + np.arange(by.size) - (np.cumsum(counts) - counts)[flat[by]]
        order[at], pos[by] = by, at
    else:
        for e, s in enumerate(slots):
            order[offsets[e]:offsets[e] + s.size] = s
            pos[s] = offsets[e] + np.arange(s.size)
    return offsets, counts, order, pos.reshape(N, k)


def labels_of(rng, N, k, E, kind):
    if kind == "even":
        l = rng.integers(0, E, (N, k))
    elif kind == "one":
        l = np.full((N, k), E - 1)
    elif kind == "none":
        l = np.full((N, k), -1)
    elif kind == "wild":
        l = rng.choice([-2 ** 31, -1, 0, E - 1, E, E + 1, 2 ** 31 - 1], (N, k))
    else:  # skewed, some dropped
        l = np.minimum((rng.random((N, k)) ** 4 * E).astype(np.int64), E - 1)
        l[rng.random((N, k)) < 0.1] = -1
    return l.astype(np.int32)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def check_plan(r, want):
    for name, w in zip(("offsets", "counts", "order", "pos"), want):
        got = getattr(r, name).cpu().numpy()
        assert np.array_equal(got, w), name


@pytest.mark.parametrize("N,k,E,align,kind", [
    (0, 2, 4, 8, "even"), (1, 1, 1, 1, "even"), (1, 1, 3, 128, "none"), (1, 4, 64, 1, "even"), (32, 2, 16, 1, "skew"),
    (63, 1, 7, 4, "skew"), (64, 1, 2, 1, "one"), (65, 3, 300, 16, "even"), (300, 64, 5, 1, "skew"), (1023, 1, 256, 1, "even"),
    (1024, 1, 257, 3, "skew"), (1025, 1, 1, 1, "even"), (2049, 2, 1000, 1, "wild"), (4096, 1, 13, 7, "none"),
    (30007, 3, 77, 1, "skew"), (60000, 1, 1024, 1, "even"), (20000, 2, 8192, 2, "skew"), (5, 1, 8192, 65536, "even"),
    (700001, 1, 64, 128, "skew"), (262144, 2, 3, 1, "one")])
def test_plan(N, k, E, align, kind):
    print("plan", N, k, E, align, kind, flush=True)
    rng = np.random.default_rng(N + 7 * k + E)
    labels = labels_of(rng, N, k, E, kind)
    rows = ftk.route_rows(N, k, E, align)
    assert rows >= ((np.bincount(labels[(labels >= 0) & (labels < E)], minlength=E) + align - 1) // align).sum() * align
    want = plan_of(labels, E, align, rows)
    check_plan(ftk.route_plan(dev(labels), E, align), want)
    X = torch.arange(N, dtype=torch.float32, device=DEV).unsqueeze(1).repeat(1, 5)
    out, r = ftk.route_dispatch(X, dev(labels), E, align)
    check_plan(r, want)
    token = np.where(want[2] >= 0, want[2] // k, 0)
    assert np.array_equal(out.cpu().numpy(), np.where(want[2] >= 0, token, 0)[:, None].repeat(5, 1))


def test_plan_into_larger_arrays_and_given_workspace():
    rng = np.random.default_rng(3)
    labels = labels_of(rng, 5000, 2, 40, "skew")
    rows = ftk.route_rows(5000, 2, 40, 16) + 777
    i32 = lambda *s: torch.full(s, 12345, dtype=torch.int32, device=DEV)  # noqa: E731
    r = ftk.Route(i32(41), i32(40), i32(rows), i32(5000, 2), 16)
    ws = torch.empty(ftk.route_workspace_bytes(5000, 2, 40) + 256, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        ftk.route_plan(dev(labels), 40, 16, route=r, workspace=ws)
        check_plan(r, plan_of(labels, 40, 16, rows))


def make(rng, N, k, E, D, dtype, align, kind="skew"):
    labels = labels_of(rng, N, k, E, kind)
    r = ftk.route_plan(dev(labels), E, align)
    order, pos = r.order.cpu().numpy().astype(np.int64), r.pos.cpu().numpy().astype(np.int64)
    x = lambda n: dev(rng.standard_normal((n, D))).to(DTYPES[dtype])  # noqa: E731
    w = rng.random((N, k)) * 2 - 0.5
    w = dev(w if dtype == "f64" else w.astype(np.float32))
    return r, order, pos, x(N), x(order.size), w


def f64(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 1, 1, 1, "f32", 1), (1, 2, 4, 1024, "bf16", 1), (3, 2, 2, 3, "bf16", 4), (17, 4, 5, 7, "f16", 1),
          (64, 3, 6, 8, "f16", 1), (50, 2, 9, 9, "bf16", 16), (33, 1, 3, 2, "f64", 1), (40, 5, 8, 131, "f64", 2),
          (777, 3, 13, 333, "f16", 1), (1500, 2, 30, 45, "f32", 128), (500, 8, 64, 65, "bf16", 1), (9, 64, 100, 257, "f32", 1),
          (300, 2, 8, 4096, "bf16", 128), (2, 1, 2, 16384, "f32", 1), (5000, 1, 100, 16, "bf16", 1), (4, 2, 3, 33000, "f16", 1)]


@pytest.mark.parametrize("N,k,E,D,dtype,align", SHAPES)
def test_rows(N, k, E, D, dtype, align):
    """Copies are exact; products and sums are off by their roundings: one of the type for the result, 2^-24 (2^-53) of the
    magnitudes for each step of a sum."""
    print("rows", N, k, E, D, dtype, align, flush=True)
    rng = np.random.default_rng(N + D)
    r, order, pos, X, Y, w = make(rng, N, k, E, D, dtype, align)
    u, acc, step = UNIT[dtype], 2.0 ** -53 if dtype == "f64" else 2.0 ** -24, STEP[dtype]
    held, token = order >= 0, np.maximum(order, 0) // k
    x, y, wf = f64(X), f64(Y), f64(w)
    got = ftk.route_gather(X, r)
    assert np.array_equal(f64(got), np.where(held[:, None], x[token], 0))
    want = np.where(held[:, None], x[token] * wf.reshape(-1)[np.maximum(order, 0)][:, None], 0)
    assert np.all(np.abs(f64(ftk.route_gather(X, r, w)) - want) <= (u + 2 * acc) * np.abs(want) + step)
    for weights in (w, None):
        terms = np.where((pos >= 0)[:, :, None], y[np.maximum(pos, 0)] * (wf if weights is not None else np.ones_like(wf))[:, :, None], 0)
        want, size = terms.sum(1), np.abs(terms).sum(1)
        got = f64(ftk.route_combine(Y, r, weights))
        assert np.all(np.abs(got - want) <= u * np.abs(want) + 2 * (k + 1) * acc * size + step)
        assert np.all(got[(pos < 0).all(1)] == 0)
    dY, dw = ftk.route_combine_grad(X, Y, r, w)
    want = np.where(held[:, None], x[token] * wf.reshape(-1)[np.maximum(order, 0)][:, None], 0)
    assert np.all(np.abs(f64(dY) - want) <= (u + 2 * acc) * np.abs(want) + step)
    terms = np.where((pos >= 0)[:, :, None], y[np.maximum(pos, 0)] * x[:, None, :], 0)
    assert np.all(np.abs(f64(dw) - terms.sum(2)) <= 2 * (D + 1) * acc * np.abs(terms).sum(2))
    assert np.all(f64(dw)[pos < 0] == 0)


def test_gradients_against_differences():
    """L = sum(G * combine(Y, w)) and L = sum(G * gather(X)) are linear in each of Y, w and X, so a difference of
    step 1 is the gradient but for the roundings of two sums of some hundred terms in 64 bits."""
    rng = np.random.default_rng(5)
    N, k, E, D = 11, 3, 4, 6
    r, order, pos, X, Y, w = make(rng, N, k, E, D, "f64", 4)
    G = dev(rng.standard_normal((N, D)))
    Gr = dev(rng.standard_normal((order.size, D)))
    loss = lambda Y, w: float((G * ftk.route_combine(Y, r, w)).sum())  # noqa: E731
    dY, dw = ftk.route_combine_grad(G, Y, r, w)
    base = loss(Y, w)
    for p in range(0, order.size, 3):
        Z = Y.clone()
        Z[p, p % D] += 1
        assert abs(loss(Z, w) - base - float(dY[p, p % D])) < 1e-12
    for t in range(N):
        v = w.clone()
        v[t, t % k] += 1
        assert abs(loss(Y, v) - base - float(dw[t, t % k])) < 1e-12
    dX = ftk.route_combine(Gr, r)
    gathered = lambda X: float((Gr * ftk.route_gather(X, r)).sum())  # noqa: E731
    base = gathered(X)
    for t in range(N):
        Z = X.clone()
        Z[t, t % D] += 1
        assert abs(gathered(Z) - base - float(dX[t, t % D])) < 1e-12


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f64"])
def test_what_is_dropped_or_unused_counts_nowhere(dtype):
    """NaN weights of dropped slots, NaN and infinities in sorted rows that no slot has, a token nobody takes."""
    rng = np.random.default_rng(8)
    N, k, E, D = 50, 2, 6, 37
    labels = labels_of(rng, N, k, E, "skew")
    labels[7] = -1
    r = ftk.route_plan(dev(labels), E, 16)
    X = dev(rng.standard_normal((N, D))).to(DTYPES[dtype])
    Y = dev(rng.standard_normal((r.rows, D))).to(DTYPES[dtype])
    w = dev(rng.random((N, k))).to(torch.float64 if dtype == "f64" else torch.float32)
    clean = ftk.route_combine(Y, r, w), *ftk.route_combine_grad(X, Y, r, w), ftk.route_gather(X, r, w)
    w2, Y2, X2 = w.clone(), Y.clone(), X.clone()
    w2[r.pos < 0] = float("nan")
    Y2[r.order < 0] = float("nan")
    Y2[torch.nonzero(r.order < 0)[0]] = float("inf")
    X2[(r.pos < 0).all(1)] = float("nan")
    again = ftk.route_combine(Y2, r, w2), *ftk.route_combine_grad(X2, Y2, r, w2), ftk.route_gather(X2, r, w2)
    for a, b in zip(clean, again):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    assert (clean[0][7] == 0).all()
    # what does count keeps its NaN and infinities to itself
    Y[r.pos[3, 0] if r.pos[3, 0] >= 0 else r.pos[3, 1], 5] = float("nan")
    got = ftk.route_combine(Y, r, w)
    bad = torch.isnan(got)
    assert bad.sum() == 1 and bad[3, 5]


@pytest.mark.parametrize("dtype,D,pad", [("bf16", 40, 3), ("f32", 45, 1), ("f16", 333, 8), ("f64", 5, 2)])
def test_strided_rows_and_untouched_surroundings(dtype, D, pad):
    rng = np.random.default_rng(D)
    N, k, E = 70, 2, 5
    labels = labels_of(rng, N, k, E, "skew")
    dt = DTYPES[dtype]
    r = ftk.route_plan(dev(labels), E, 8)
    wide = lambda n: dev(rng.standard_normal((n, D + 2 * pad))).to(dt)  # noqa: E731
    Xw, Yw = wide(N), wide(r.rows)
    X, Y = Xw[:, pad:pad + D], Yw[:, pad:pad + D]
    w = dev(rng.random((N, k))).to(torch.float64 if dtype == "f64" else torch.float32)
    for run, rows in ((lambda X, Y, o: ftk.route_gather(X, r, w, out=o), r.rows),
                      (lambda X, Y, o: ftk.route_combine(Y, r, w, out=o), N),
                      (lambda X, Y, o: ftk.route_combine_grad(X, Y, r, w, dY=o)[0], r.rows),
                      (lambda X, Y, o: ftk.route_dispatch(X, dev(labels), E, 8, out=o)[0], r.rows)):
        plain = run(X.contiguous(), Y.contiguous(), torch.empty(rows, D, dtype=dt, device=DEV))
        o = torch.full((rows, D + 2 * pad), 7.0, dtype=dt, device=DEV)
        run(X, Y, o[:, pad:pad + D])
        assert torch.equal(o[:, pad:pad + D], plain)
        assert (o[:, :pad] == 7).all() and (o[:, pad + D:] == 7).all()


def test_nothing_to_do():
    labels = torch.empty(0, 3, dtype=torch.int32, device=DEV)
    X = torch.empty(0, 8, device=DEV)
    out, r = ftk.route_dispatch(X, labels, 5, 16)
    assert out.shape == (0, 8) and r.offsets.tolist() == [0] * 6 and r.counts.tolist() == [0] * 5
    assert ftk.route_combine(out, r).shape == (0, 8)
    dY, dw = ftk.route_combine_grad(X, out, r, torch.empty(0, 3, device=DEV))
    assert dY.shape == (0, 8) and dw.shape == (0, 3)
    # arrays for more slots than there are: all of them hold nothing
    i32 = lambda *s: torch.full(s, 12345, dtype=torch.int32, device=DEV)  # noqa: E731
    for align in (1, 16):
        big = ftk.Route(i32(6), i32(5), i32(48), torch.empty(0, 3, dtype=torch.int32, device=DEV), align)
        out = torch.full((48, 8), 3.0, device=DEV)
        ftk.route_dispatch(X, labels, 5, align, out=out, route=big)
        assert (out == 0).all() and (big.order == -1).all() and big.offsets.tolist() == [0] * 6
        dY = torch.full((48, 8), 3.0, device=DEV)
        ftk.route_combine_grad(X, out, big, torch.empty(0, 3, device=DEV), dY=dY)
        assert (dY == 0).all()


def test_index_arrays_that_lie():
    """A call cannot look at device data first: entries out of range take no row and harm nothing."""
    rng = np.random.default_rng(2)
    N, k, D = 40, 2, 24
    r, order, pos, X, Y, w = make(rng, N, k, 4, D, "f32", 1, "even")
    bad = ftk.Route(r.offsets, r.counts, r.order.clone(), r.pos.clone(), 1)
    bad.pos[3, 1], bad.pos[5, 0], bad.pos[6] = r.rows, 2 ** 31 - 1, -2 ** 31
    got = ftk.route_combine(Y, bad, w)
    off = r.pos.clone()
    off[3, 1], off[5, 0], off[6] = -1, -1, -1
    assert torch.equal(got, ftk.route_combine(Y, ftk.Route(r.offsets, r.counts, r.order, off, 1), w))
    bad.order[0] = N * k
    assert (ftk.route_combine_grad(X, Y, bad, w)[1][6] == 0).all()
    torch.cuda.synchronize()


def test_elements_beyond_32_bits():
    """More than 2^32 elements in the sorted rows."""
    N, D = 2_100_001, 2064
    rng = np.random.default_rng(1)
    labels = rng.integers(0, 3, (N, 1)).astype(np.int32)
    r = ftk.route_plan(dev(labels), 3)
    assert r.rows * D > 2 ** 32
    X = torch.zeros(N, D, dtype=torch.bfloat16, device=DEV)
    X[:, 0] = torch.arange(N, device=DEV) % 251
    X[:, -1] = torch.arange(N, device=DEV) % 241
    out = ftk.route_gather(X, r)
    t = r.order.long()
    assert torch.equal(out[:, 0], X[t, 0]) and torch.equal(out[:, -1], X[t, -1])
    assert not out[:, 1000].any()
    back = ftk.route_combine(out, r)
    assert torch.equal(back[:, 0], X[:, 0]) and torch.equal(back[:, -1], X[:, -1])


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(4)
    labels = dev(labels_of(rng, 6000, 2, 30, "skew"))
    X = dev(rng.standard_normal((6000, 64)).astype(np.float32))
    w = dev(rng.random((6000, 2)).astype(np.float32))
    rows, r = ftk.route_dispatch(X, labels, 30, 16)
    want = ftk.route_combine(rows, r, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rows2, r2 = ftk.route_dispatch(X, labels, 30, 16)
        got = ftk.route_combine(rows2, r2, w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    ws = torch.empty(ftk.route_workspace_bytes(6000, 2, 30) + 256, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ftk.route_dispatch(X, labels, 30, 16, out=rows2, route=r2, workspace=ws)
        ftk.route_combine(rows2, r2, w, out=out)
    for seed in range(3):
        labels.copy_(dev(labels_of(np.random.default_rng(seed), 6000, 2, 30, "skew")))
        rows, r = ftk.route_dispatch(X, labels, 30, 16)
        want = ftk.route_combine(rows, r, w)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(r2.pos, r.pos)


def test_plans_of_many_experts_from_two_threads():
    """Calls that need different amounts of more than 64 KB of LDS, under way in two threads at once."""
    import threading
    rng = np.random.default_rng(31)
    N, wrong = 3000, []

    def work(E):
        labels = labels_of(rng, N, 1, E, "even")
        want = plan_of(labels, E, 1, N)
        labels = dev(labels)
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(40):
                try:
                    check_plan(ftk.route_plan(labels, E), want)
                except Exception as e:  # (an assertion in a thread would be lost)
                    wrong.append((E, repr(e)))

    dev(np.zeros(1))
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(E,)) for E in (8192, 4200)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]


def test_plan_of_many_experts_in_a_graph():
    rng = np.random.default_rng(32)
    N, E = 5000, 8000
    labels = dev(labels_of(rng, N, 2, E, "skew"))
    r = ftk.route_plan(labels, E)
    ws = torch.empty(ftk.route_workspace_bytes(N, 2, E) + 256, dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ftk.route_plan(labels, E, route=r, workspace=ws)
    for seed in range(3):
        labels.copy_(dev(labels_of(np.random.default_rng(seed), N, 2, E, "skew")))
        want = ftk.route_plan(labels, E)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for name in ("offsets", "counts", "order", "pos"):
            assert torch.equal(getattr(r, name), getattr(want, name)), name
