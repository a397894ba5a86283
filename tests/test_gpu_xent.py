"""Softmax cross entropy over many classes and its gradients against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
INF = float("inf")


def problem(N, V, D, dtype, bias=False, seed=0, spread=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed + N + V + D)
    X = torch.randn(N, D, generator=g, device=DEV).to(TYPES[dtype])
    W = (torch.randn(V, D, generator=g, device=DEV) * spread * D ** -0.5).to(TYPES[dtype])
    labels = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    if N > 3:
        labels[::7] = torch.tensor([-1, V, -5, 2 ** 31 - 1], dtype=torch.int32, device=DEV).repeat(N)[:labels[::7].numel()]
    b = torch.randn(V, generator=g, device=DEV) if bias else None
    dloss = torch.randn(N, generator=g, device=DEV) * (64.0 if dtype == "f16" else 1.0) / max(N, 1)
    return X, W, labels, b, dloss


def formulas(X, W, labels, b, dloss, scale):
    """loss, lse, dX, dW, dbias in 64 bits, and of each the sum of its terms' magnitudes (of loss and lse: the largest logit's)."""
    V = W.shape[0]
    live = (labels >= 0) & (labels < V)
    x, w = torch.where(live.unsqueeze(1), X, 0).double(), W.double()
    bias = torch.zeros(V, dtype=torch.float64, device=DEV) if b is None else b.double()
    z = scale * (x @ w.t()) + bias
    size = (abs(scale) * (x.abs() @ w.abs().t()) + torch.where(bias.isfinite(), bias.abs(), 0)).amax(1)
    lse = torch.logsumexp(z, 1)
    at = torch.where(live, labels, 0).long().unsqueeze(1)
    loss = torch.where(live, lse - z.gather(1, at).squeeze(1), 0)
    p = torch.exp(z - lse.unsqueeze(1))
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    g = torch.where(live, dloss.double(), 0).unsqueeze(1)
    d, dsize = g * (p - one), g.abs() * (p + one)
    return ((loss, torch.where(live, lse, 0), scale * (d @ w), scale * (d.t() @ x), d.sum(0)),
            (size, abs(scale) * (dsize @ w.abs()), abs(scale) * (dsize.t() @ x.abs()), dsize.sum(0)))


def check(X, W, labels, b, dloss, scale=1.0, **outs):
    (loss, lse, dX, dW, db), (size, sX, sW, sb) = formulas(X, W, labels, b, dloss, scale)
    N, D = X.shape
    V, t = W.shape[0], X.dtype
    half, one = HALF[t], 2.0 ** -24
    # logits: D products added in 32 bits (six times as many where 32-bit rows go by pieces, which leave out 2^-23 of them besides),
    # a product and a sum; the exponent's two roundings are of their size too
    terms = D * (6 if t == torch.float32 else 1) + 8
    off = (terms * one * size + 2.0 ** -20) * 1.0
    got = ftk.xent(X, W, labels, bias=b, scale=scale)
    for mine, want in zip(got, (loss, lse)):
        # and V terms' sum: by lanes and tiles, each term through less than 300 additions
        assert ((mine.double() - want).abs() <= 2 * off + 300 * one + 4 * one * want.abs()).all()
    live = (labels >= 0) & (labels < V)
    assert (got[0][~live] == 0).all() and (got[1][~live] == 0).all()
    grads = ftk.xent_grad(X, W, labels, got[1], dloss, bias=b, scale=scale, need=(True, True, True), **outs)
    worst = float(off.max()) * 3 + 300 * one
    # d is off by the logits' error and by its rounding (to 24 bits by pieces; fp16: a half step of 2^-24 of the largest dloss, 2^14
    # times as large, at the least), then come sums over V classes or N rows, and the rounding of the result
    rounding = 2.0 ** -22 if t == torch.float32 else half
    top = float(torch.where(live, dloss.abs(), 0).max()) if N else 0.0
    for mine, want, s, n, scaled in ((grads[0], dX, sX, V, W), (grads[1], dW, sW, N, X)):
        n = n * (6 if t == torch.float32 else 1) + 8
        tiny = 0.0
        if t == torch.float16:
            tiny = 2.0 ** -25 + top * 2.0 ** -38 * n * float(torch.where(scaled.isfinite(), scaled.abs(), 0).max()) * abs(scale)
        assert ((mine.double() - want).abs() <= (worst + rounding + n * one) * s + 1.01 * half * want.abs() + tiny + 1e-37).all()
    assert ((grads[2].double() - db).abs() <= (worst + (N + 8) * one) * sb + one * db.abs() + 1e-37).all()
    return got, grads


SIZES = [(1, 1, 1), (1, 2, 8), (1, 1000, 64), (3, 65, 72), (5, 700, 129), (16, 513, 40), (63, 64, 64), (65, 127, 200), (130, 300, 96),
         (257, 259, 136), (700, 1100, 64), (40, 5000, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", SIZES)
def test_loss_and_gradients(N, V, D, dtype):
    check(*problem(N, V, D, dtype, bias=V % 2 == 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D,rows,cols", [(2500, 4000, 256, 256, 256), (1200, 2100, 320, 128, 128)])
def test_large_tiles(N, V, D, rows, cols, dtype):
    check(*problem(N, V, D, dtype, bias=True))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,V,D", [(1, 17, 1024), (1, 9001, 1032), (2, 4097, 2048), (16, 8200, 2040), (15, 20000, 520), (16, 3000, 4096),
                                   (9, 5003, 4088), (17, 9000, 1000), (32, 8191, 2048), (31, 12345, 64), (1, 70000, 32)])
def test_few_rows(N, V, D, dtype):
    """Rows that stay in registers while the classes pass: one, sixteen, up to thirty-two, and lengths that end within a step."""
    check(*problem(N, V, D, dtype, bias=V % 2 == 1))


@pytest.mark.parametrize("N,V,D,dtype", [(12000, 9000, 72, "f32"), (12000, 14000, 72, "bf16"), (12000, 14000, 64, "f16"),
                                         (150000, 1700, 16, "bf16"), (150000, 4000, 16, "f32")])
def test_pieces_of_the_classes(N, V, D, dtype):
    """So many rows that the classes go in several pieces: sums and gradients of the rows are added up over them."""
    check(*problem(N, V, D, dtype, bias=True))


@pytest.mark.parametrize("N,V,D,dtype", [(777, 10007, 333, "f32"), (777, 10007, 333, "bf16"), (9001, 1000, 250, "f16"), (9001, 1000, 250, "f32"),
                                         (65, 40001, 130, "f32"), (33, 30000, 136, "f16"), (20000, 3, 129, "f32"), (20000, 3, 129, "bf16")])
def test_products_in_shares(N, V, D, dtype):
    """Few tiles and long sums, which several workgroups share: shares of unequal length, tiles that are no multiple of the XCDs."""
    check(*problem(N, V, D, dtype, bias=True))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [90, 10])
@pytest.mark.parametrize("D,ldx,ldw,shift", [(64, 80, 72, 8), (64, 64, 67, 0), (33, 40, 50, 1), (40, 41, 40, 3), (1, 3, 5, 1),
                                             (128, 131, 136, 8)])
def test_strides_and_addresses(D, ldx, ldw, shift, N, dtype):
    """Rows of wider arrays, NaN between and around them, at addresses of every alignment; results likewise."""
    V, t = 140, TYPES[dtype]
    X, W, labels, b, dloss = problem(N, V, D, dtype, bias=True)

    def inside(a, ld):
        wide = torch.full((a.shape[0] * ld + shift + ld,), float("nan"), dtype=t, device=DEV)
        view = wide[shift:shift + a.shape[0] * ld].view(-1, ld)[:, :D]
        view.copy_(a)
        return wide, view

    (_, x), (_, w), (around, dX), (beside, dW) = inside(X, ldx), inside(W, ldw), inside(0 * X, ldx), inside(0 * W, ldw)
    got, grads = check(x, w, labels, b, dloss, scale=0.7, dX=dX, dW=dW)
    assert grads[0] is dX and grads[1] is dW
    assert int(around.isnan().sum()) == around.numel() - N * D and int(beside.isnan().sum()) == beside.numel() - V * D
    plain, _ = check(X, W, labels, b, dloss, scale=0.7)
    if N > 32:  # (few rows are added up in another order where their classes lie aligned)
        assert torch.equal(plain[0], got[0]) and torch.equal(plain[1], got[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_ignored_rows_are_not_looked_at(dtype):
    X, W, labels, b, dloss = problem(200, 333, 64, dtype)
    live = (labels >= 0) & (labels < 333)
    clean = ftk.xent(X, W, labels), ftk.xent_grad(X, W, labels, ftk.xent(X, W, labels)[1], dloss)
    X[~live] = float("nan")
    dloss = torch.where(live, dloss, INF)
    loss, lse = ftk.xent(X, W, labels)
    assert torch.equal(loss, clean[0][0]) and torch.equal(lse, clean[0][1])
    dX, dW, db = ftk.xent_grad(X, W, labels, lse, dloss)
    assert torch.equal(dX, clean[1][0]) and torch.equal(dW, clean[1][1]) and db is None
    assert (dX[~live] == 0).all()
    none = torch.full_like(labels, -1)
    loss, lse = ftk.xent(X, W, none)
    assert (loss == 0).all()
    assert all((t == 0).all() for t in ftk.xent_grad(X, W, none, lse, dloss, need=(True, True, True)))


@pytest.mark.parametrize("dtype", TYPES)
def test_closed_classes_and_bad_values(dtype):
    X, W, labels, b, dloss = problem(60, 200, 64, dtype, bias=True)
    b[::3] = -INF
    labels = torch.where(labels % 3 == 0, labels + 1, labels)  # (all in range: 199 % 3 == 1)
    check(X, W, labels, b, dloss)
    labels[4] = 3  # a closed class
    loss, lse = ftk.xent(X, W, labels, bias=b)
    assert loss[4] == INF and lse[4].isfinite()
    dX, dW, db = ftk.xent_grad(X, W, labels, lse, dloss, bias=b)
    assert dX.isfinite().all() and dW.isfinite().all() and db.isfinite().all()
    loss, lse = ftk.xent(X, W, labels, bias=torch.full_like(b, -INF))
    live = (labels >= 0) & (labels < 200)
    assert (lse[live] == -INF).all() and loss[live].isnan().all()
    X[9] = float("nan")
    labels[9] = 1
    loss, lse = ftk.xent(X, W, labels, bias=b)
    assert loss[9].isnan() and int(loss.isnan().sum()) == 1
    dX, dW, db = ftk.xent_grad(X, W, labels, lse, dloss, bias=b)
    assert dX[9].isnan().all() and int(dX.isnan().any(1).sum()) == 1 and db.isnan().any()


def test_large_logits():
    """Logits of some thousands: nothing overflows, the loss is their difference."""
    X, W, labels, b, dloss = problem(50, 300, 64, "bf16", spread=800.0)
    check(X, W, labels, b, dloss)


def test_offsets_beyond_32_bits():
    """Classes' rows of more than 2^32 elements, and few rows at strides as long: what lies at the end is read and written."""
    V, D = (1 << 21) + 777, 2048
    W = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
    W[:V - 1000] = 0  # (equal logits but for the last classes)
    W[V - 1000:] = torch.randn(1000, D, device=DEV)
    for N in (8, 70):
        X = (torch.randn(N, D, device=DEV) * D ** -0.5).bfloat16()
        labels = torch.arange(V - N, V, dtype=torch.int32, device=DEV)
        loss, lse = ftk.xent(X, W, labels)
        z = X.double() @ W[V - 1000:].double().t()
        want = (z.exp().sum(1) + (V - 1000)).log()
        assert ((lse.double() - want).abs() < 1e-5).all()
        assert ((loss.double() - (want - z[torch.arange(N), torch.arange(1000 - N, 1000)])).abs() < 2e-5).all()
    dloss = torch.ones(N, device=DEV)
    dX, dW, _ = ftk.xent_grad(X, W, labels, lse, dloss)
    d = (z - want.unsqueeze(1)).exp()
    d[torch.arange(N), torch.arange(1000 - N, 1000)] -= 1
    x = X.double()
    size = d.abs() @ W[V - 1000:].double().abs()
    assert ((dX.double() - d @ W[V - 1000:].double()).abs() <= 2 * 2.0 ** -8 * size + 1e-30).all()
    assert ((dW[V - 1000:].double() - d.t() @ x).abs() <= 2 * 2.0 ** -8 * (d.t().abs() @ x.abs()) + 1e-30).all()
    del W, dW
    for dtype in TYPES.values():
        far = torch.empty((1 << 32) // dtype.itemsize * 2 + 64, dtype=dtype, device=DEV)
        ld = (1 << 32) // dtype.itemsize
        x, w = far.as_strided((3, 32), (ld, 1)), far.as_strided((3, 32), (ld, 1), 32)
        x.copy_(torch.randn(3, 32, device=DEV)), w.copy_(torch.randn(3, 32, device=DEV))
        labels = torch.tensor([0, 2, 1], dtype=torch.int32, device=DEV)
        a, b = ftk.xent(x, w, labels), ftk.xent(x.contiguous(), w.contiguous(), labels)
        assert torch.equal(a[0], b[0])
        for p, q in zip(ftk.xent_grad(x, w, labels, a[1], torch.ones(3, device=DEV)),
                        ftk.xent_grad(x.contiguous(), w.contiguous(), labels, a[1], torch.ones(3, device=DEV))):
            assert p is None or torch.equal(p, q)
        del far, x, w


def test_assignment_scores():
    """With minus half the squared norms as bias the likeliest class is the assignment's label."""
    g = torch.Generator(device=DEV).manual_seed(2)
    C = torch.randn(50, 24, generator=g, device=DEV)
    X = C[torch.randint(50, (400,), generator=g, device=DEV)] + 0.2 * torch.randn(400, 24, generator=g, device=DEV)
    labels, dist = ftk.kmeans_assign(X, C)
    bias = -0.5 * C.square().sum(1)
    loss, lse = ftk.xent(X, C, labels, bias=bias)
    score = (X.double() @ C.double().t() + bias).gather(1, labels.long().unsqueeze(1)).squeeze(1)
    assert ((lse - loss).double() - score).abs().max() < 1e-4
    # raising the rows along the gradient lowers the loss: a step of the descent reaches what its slope says
    dX, _, _ = ftk.xent_grad(X, C, labels, lse, torch.ones(400, device=DEV), bias=bias, need=(True, False, False))
    again, _ = ftk.xent((X - 1e-3 * dX).contiguous(), C, labels, bias=bias)
    slope = dX.double().square().sum(1) * 1e-3
    assert ((loss - again).double() - slope).abs().max() < 0.05 * float(slope.max()) + 1e-5


def test_parts_and_no_rows():
    X, W, labels, b, dloss = problem(70, 90, 40, "bf16", bias=True)
    loss, lse = ftk.xent(X, W, labels, bias=b)
    whole = ftk.xent_grad(X, W, labels, lse, dloss, bias=b)
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        part = ftk.xent_grad(X, W, labels, lse, dloss, bias=b, need=need)
        for n, a, c in zip(need, part, whole):
            assert torch.equal(a, c) if n else a is None
    empty = ftk.xent(X[:0], W, labels[:0])
    assert empty[0].shape == (0,)
    dX, dW, db = ftk.xent_grad(X[:0], W, labels[:0], lse[:0], dloss[:0], bias=b)
    assert dX.shape == (0, 40) and (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_graph(dtype):
    """Both directions captured once, replayed on other operands with eager calls between; the workspace holds NaN before."""
    N, V, D = 300, 700, 72
    X, W, labels, b, dloss = problem(N, V, D, dtype, bias=True)
    code = ftk._MX_DTYPES[X.dtype]
    ws = [torch.full((ftk.xent_workspace_bytes(code, N, V, D, grad) // 4 + 64,), float("nan"), device=DEV) for grad in (False, True)]

    def step():
        loss, lse = ftk.xent(X, W, labels, bias=b, workspace=ws[0])
        return (loss, lse, *ftk.xent_grad(X, W, labels, lse, dloss, bias=b, workspace=ws[1]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        x, w, l, bb, dl = problem(N, V, D, dtype, bias=True, seed=10 + turn)
        for to, new in zip((X, W, labels, b, dloss), (x, w, l, bb, dl)):
            to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in held]
        loss, lse = ftk.xent(x, w, l, bias=bb)
        for a, c in zip(kept, (loss, lse, *ftk.xent_grad(x, w, l, lse, dl, bias=bb))):
            assert torch.equal(a, c)


def test_refusals():
    X, W, labels, b, dloss = problem(10, 12, 16, "f32", bias=True)
    _, lse = ftk.xent(X, W, labels)
    for call in (lambda: ftk.xent(X, W[:, :8], labels), lambda: ftk.xent(X, W.bfloat16(), labels), lambda: ftk.xent(X, W, labels.long()),
                 lambda: ftk.xent(X, W, labels[:5]), lambda: ftk.xent(X, W, labels, bias=b[:5]), lambda: ftk.xent(X.t(), W.t(), labels),
                 lambda: ftk.xent_grad(X, W, labels, lse[:4], dloss), lambda: ftk.xent_grad(X, W, labels, lse, dloss.double()),
                 lambda: ftk.xent_grad(X, W, labels, lse, dloss, dX=W)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ftk.xent(X.double(), W.double(), labels)
    with pytest.raises(ftk.FtkError):
        ftk.xent(X, W, labels, scale=INF)
    with pytest.raises(ftk.FtkError):
        ftk.xent(X, W, labels, workspace=torch.empty(300, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", [(7, 900, 128), (30, 3000, 256), (300, 900, 72), (2500, 4000, 256)])
def test_masks_of_the_lowest_value(N, V, D, dtype):
    """A bias of the 32-bit type's lowest value, on whole tiles and single classes, closes them as -infinity does."""
    X, W, labels, b, dloss = problem(N, V, D, dtype, bias=True)
    shut = torch.zeros(V, dtype=torch.bool, device=DEV)
    shut[V // 3:V // 3 + 600] = True
    shut[::5] = True
    labels = torch.where(shut[labels.clamp(0, V - 1).long()], 1 + 0 * labels, labels)  # (an open class)
    low, closed = b.masked_fill(shut, torch.finfo(torch.float32).min), b.masked_fill(shut, -INF)
    got, want = ftk.xent(X, W, labels, bias=low), ftk.xent(X, W, labels, bias=closed)
    assert got[0].isfinite().all() and all(torch.equal(a, c) for a, c in zip(got, want))
    grads = [ftk.xent_grad(X, W, labels, got[1], dloss, bias=bias, need=(True, True, True)) for bias in (low, closed)]
    assert all(a.isfinite().all() and torch.equal(a, c) for a, c in zip(*grads))
    # a label there: its loss is as large; and all classes: their logits are that value, the logarithm of their number vanishes
    labels[N // 2] = V // 3 + 7
    loss, lse = ftk.xent(X, W, labels, bias=low)
    assert loss[N // 2] > 3e38 and lse[N // 2].isfinite()
    loss, lse = ftk.xent(X, W, labels, bias=torch.full_like(b, torch.finfo(torch.float32).min))
    live = (labels >= 0) & (labels < V)
    assert (lse[live] == torch.finfo(torch.float32).min).all() and (loss == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", [(1, 9, 8), (60, 200, 64), (300, 900, 72), (12000, 14000, 16)])
def test_rows_without_open_classes_have_no_gradient(N, V, D, dtype):
    """All logits -infinity: lse says so, and gradients are zeros, at the labels too; over one and several pieces of the classes."""
    X, W, labels, _, dloss = problem(N, V, D, dtype)
    bias = torch.full((V,), -INF, device=DEV)
    _, lse = ftk.xent(X, W, labels, bias=bias)
    live = (labels >= 0) & (labels < V)
    assert (lse[live] == -INF).all()
    for grad in ftk.xent_grad(X, W, labels, lse, dloss, bias=bias, need=(True, True, True)):
        assert (grad == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, -1e9])
@pytest.mark.parametrize("N,V,D", [(1, 9, 8), (16, 513, 41), (70, 333, 64), (300, 900, 72), (130, 5000, 256), (2500, 4000, 256), (12000, 14000, 16)])
def test_gradient_of_classes_that_are_all_masked(N, V, D, low, dtype):
    """A bias so low that 32-bit logits are all alike, the logarithm of their number lost in lse: each class has probability 1 / V."""
    X, W, labels, _, dloss = problem(N, V, D, dtype)
    bias = torch.full((V,), low, device=DEV)
    _, lse = ftk.xent(X, W, labels, bias=bias)
    grads = ftk.xent_grad(X, W, labels, lse, dloss, bias=bias, need=(True, True, True))
    live = (labels >= 0) & (labels < V)
    g = torch.where(live, dloss.double(), 0).unsqueeze(1)
    d = (g / V).expand(N, V).clone()
    d.scatter_add_(1, torch.where(live, labels, 0).long().unsqueeze(1), -g)
    x, w, half, one = X.double(), W.double(), HALF[X.dtype], 2.0 ** -24
    # the sum of V equal terms and the division by it; d's rounding (fp16: a half step of 2^-38 of the largest dloss at least); the sums
    for mine, want, size, n, scaled in ((grads[0], d @ w, d.abs() @ w.abs(), V, w), (grads[1], d.t() @ x, d.abs().t() @ x.abs(), N, x),
                                        (grads[2], d.sum(0), d.abs().sum(0), N, None)):
        rounding = 0 if scaled is None else 2.0 ** -22 if X.dtype == torch.float32 else half
        n = n * (6 if X.dtype == torch.float32 else 1) + 8
        tiny = 2.0 ** -25 + float(g.abs().max()) * 2.0 ** -38 * n * float(scaled.abs().max()) if X.dtype == torch.float16 and scaled is not None else 0
        last = one if scaled is None else half
        assert ((mine.double() - want).abs() <= (rounding + (V + n + 8) * one) * size + 1.01 * last * want.abs() + tiny + 1e-37).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 41])
def test_gradient_of_rows_with_far_logits(D, dtype):
    """Rows whose logits all lie at 3 * 10^5, steps of 2^-5 apart, among others: their probabilities add up to 1, which exp(z - lse)
    do not; the other rows' gradients are what they are without them, bit for bit."""
    N, V = 200, 333
    X, W, labels, _, dloss = problem(N, V, D, dtype)
    far = [3, 64, 70, 199]
    labels = torch.where(labels < 0, 5, labels.clamp(max=V - 1))
    W[:, 0], X[:, 0], X[far, 0] = 8, 0, 4e4
    dloss[far] = 1e-4
    _, lse = ftk.xent(X, W, labels)
    assert ((lse.abs() > 3e5).nonzero().flatten().cpu() == torch.tensor(far)).all()
    for n in far:
        alone = torch.zeros_like(dloss)
        alone[n] = 1.0
        db = ftk.xent_grad(X, W, labels, lse, alone, need=(False, False, True))[2]
        # V terms' sum there and here
        assert abs(float(db.double().sum())) <= 2 * (V + 20) * 2.0 ** -24
        assert (db[torch.arange(V, device=DEV) != labels[n]] >= 0).all() and -1 < float(db[labels[n]]) < 0
    dX = ftk.xent_grad(X, W, labels, lse, dloss)[0]
    closed = labels.clone()
    closed[far] = -1
    others = ftk.xent_grad(X, W, closed, lse, dloss)[0]
    rest = torch.ones(N, dtype=torch.bool, device=DEV)
    rest[far] = False
    assert torch.equal(dX[rest], others[rest]) and (others[far] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_graph_of_far_logits(dtype):
    """Shares of the classes that count each other's ends, captured and replayed with eager calls between, in a workspace of any content."""
    N, V, D = 130, 5000, 72
    X, W, labels, _, dloss = problem(N, V, D, dtype)
    bias = torch.full((V,), -1e9, device=DEV)
    _, lse = ftk.xent(X, W, labels, bias=bias)
    ws = torch.full((ftk.xent_workspace_bytes(ftk._MX_DTYPES[X.dtype], N, V, D, True) + 512,), 255, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ftk.xent_grad(X, W, labels, lse, dloss, bias=bias, workspace=ws)
    for turn in range(4):
        if turn == 2:
            ws.fill_(127)
        dloss.mul_(-0.5)
        graph.replay()
        want = ftk.xent_grad(X, W, labels, lse, dloss, bias=bias)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_no_rows_and_their_gradient_alone():
    X, W, labels, b, dloss = problem(70, 90, 40, "bf16", bias=True)
    lse = torch.zeros(0, device=DEV)
    for bias, need in ((None, (True, False, None)), (b, (True, False, False))):
        dX, dW, db = ftk.xent_grad(X[:0], W, labels[:0], lse, lse, bias=bias, need=need)
        assert dX.shape == (0, 40) and dX.dtype == X.dtype and dW is None and db is None
    out = torch.empty(0, 40, dtype=X.dtype, device=DEV)
    assert ftk.xent_grad(X[:0], W, labels[:0], lse, lse, dX=out, need=(False, False, False))[0] is out
    with pytest.raises(ftk.FtkError):  # (refused as with rows)
        ftk.xent_grad(X[:0], W, labels[:0], lse, lse, scale=INF, need=(True, False, False))


@pytest.mark.parametrize("N,V,D,dtypes", [
    # tiles of 256 x 256 for the logits and both gradients, two pieces of the classes; the rows' gradient in four shares of the classes
    (5001, 33001, 520, ("bf16", "f16")),
    # the same without shares, where the rows' sums go on from piece to piece, 160 and 157 stages of classes and 128 of rows, rows read
    # where they lie and packed
    (8150, 20003, 1096, ("bf16", "f16")), (8150, 20003, 1101, ("bf16",)),
    # tiles of 128 x 128 for the gradients, of 256 and of 128 for the logits, the classes' gradient in sixteen shares
    (30001, 1003, 255, ("f16",)), (20001, 1000, 248, ("bf16",)),
    # three pieces of 16 bits: tiles of 128 x 128, in shares and without, two pieces of the classes
    (5001, 9001, 333, ("f32",)), (777, 10007, 333, ("f32",))])
def test_every_stage_of_large_products(N, V, D, dtypes):
    """Within bounds that a stage of k too many or too few would break, of 64 or 32 terms among thousands: errors of d and of the logits
    are independent of each other, so that the sum of n terms of size t and relative error e is off by 8 e sqrt(sum t^2), but in one
    of 10^13 cases (Hoeffding)."""
    for dtype in dtypes:
        X, W, labels, b, dloss = problem(N, V, D, dtype, bias=True)
        live = (labels >= 0) & (labels < V)
        x, w = torch.where(live.unsqueeze(1), X, 0).double(), W.double()
        z = (x @ w.t()).add_(b.double())
        # a logit's D products (times six) are added to partial sums that stay below 4 sqrt(D) times the largest of them or so: 8 is more
        # than any logit here has
        logit = 8 * (D * (6 if dtype == "f32" else 1)) ** 0.5 * 2.0 ** -24 * max(8.0, float(z.abs().max())) + 2.0 ** -22
        lse = torch.logsumexp(z, 1)
        loss, mine = ftk.xent(X, W, labels, bias=b)
        at = torch.where(live, labels, 0).long().unsqueeze(1)
        want = torch.where(live, lse - z.gather(1, at).squeeze(1), 0)
        for a, c in ((mine, torch.where(live, lse, 0)), (loss, want)):
            assert ((a.double() - c).abs() <= 2 * logit + 64 * 2.0 ** -24).all()
        d = z.sub_(lse.unsqueeze(1)).exp_()
        d.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float64))
        d *= torch.where(live, dloss.double(), 0).unsqueeze(1)
        dX, dW, db = ftk.xent_grad(X, W, labels, mine, dloss, bias=b)
        each = logit + (2.0 ** -22 if dtype == "f32" else HALF[X.dtype])
        least = 2.0 ** -38 * float(dloss.abs().max()) if dtype == "f16" else 0.0  # (half a step of the smallest d)
        half, common = HALF[X.dtype], 400 * 2.0 ** -24  # lse and its sums err alike for all classes of a row
        squares = d.square()
        for got, right, q, u, n in ((dX, d @ w, squares @ w.square(), w, V), (dW, d.t() @ x, squares.t() @ x.square(), x, N)):
            size = (d.abs() if n == V else d.abs().t()) @ u.abs()
            tiny = 8 * least * n ** 0.5 * float(u.abs().max()) + (2.0 ** -25 if dtype == "f16" else 1e-37)
            bound = 8 * each * q.sqrt() + common * size + 1.01 * half * right.abs() + tiny
            within = bool(((got.double() - right).abs() <= bound).all())
            assert within, dtype
            # (the bounds tell: the terms of a stage of 64, or of 32 in three pieces, have that part of the squares)
            stage = 32 if dtype == "f32" else 64
            tells = float((bound / (stage / n * q).sqrt().clamp(min=1e-37)).median()) < 1
            assert tells, dtype
            del size, bound, q
        assert ((db.double() - d.sum(0)).abs() <= 8 * logit * squares.sum(0).sqrt() + common * d.abs().sum(0) + 1e-37).all()
        del x, w, z, d, squares, X, W, dX, dW
