"""Rows in microscaled 4-bit floating point (ftk_mx4_*) against plain numpy in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from tests.gpu_util import DEV
from tests.test_gpu_route import DTYPES, STEP, UNIT, dev, f64, labels_of

pytestmark = pytest.mark.gpu

TABLE = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def pack_of(x):
    """codes and scales of the rows of x (float64) by the definition."""
    n, d = x.shape
    dp = -(-d // 128) * 128
    p = np.zeros((n, dp))
    p[:, :d] = x
    p = p.reshape(n, dp // 32, 32)
    top = np.abs(p).max(2)
    bad = ~np.isfinite(top)
    _, e = np.frexp(np.where(bad, 1, top))
    b = np.where(top > 0, np.maximum(e - 3, -127), -127)
    y = np.abs(np.where(bad[:, :, None], 0, p)) / np.exp2(b.astype(np.float64))[:, :, None]
    near = np.abs(y[..., None] - TABLE)
    code = near.argmin(3)  # of two equally near ones the lower, unless the upper is even
    up = np.minimum(code + 1, 7)
    tie = (np.take_along_axis(near, up[..., None], 3)[..., 0] == near.min(3)) & (up % 2 == 0) & (up != code)
    code = np.where(tie, up, code) + 8 * np.signbit(p)
    code = code.reshape(n, dp)
    return (code[:, ::2] + 16 * code[:, 1::2]).astype(np.uint8), np.where(bad, 255, b + 127).astype(np.uint8)


def values_of(codes, scales, d):
    codes = codes.astype(np.int64)
    code = np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], 2 * codes.shape[1])
    v = np.where(code & 8, -1.0, 1.0) * TABLE[code & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * s.repeat(32, 1))[:, :d]


def values(q):
    return values_of(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.D)


def check_pack(q, x):
    codes, scales = pack_of(x)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    fine = (scales != 255).repeat(16, 1)
    assert np.array_equal(q.codes.cpu().numpy()[fine], codes[fine])


def same(got, want):
    """Equal, NaN where NaN is."""
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.where(torch.isnan(got), 0, got), torch.where(torch.isnan(want), 0, want))


def edges(dtype):
    """Every magnitude of the type's upper 16 bits (f16: all) in blocks of close neighbours, ties and their neighbours
    among them, each with a few larger values that set the block's scale."""
    if dtype == "f16":
        x = np.arange(0x7c00, dtype=np.uint16).view(np.float16).astype(np.float64)
    else:
        x = (np.arange(0x7f80, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)
    top = torch.finfo(DTYPES[dtype]).max
    rows = [x]
    for f in (2.0, 1.5, 0.25, 1 / 12):
        rows.append(np.minimum(x * f, top))
    x = np.concatenate([r[:len(r) // 31 * 31].reshape(-1, 31) for r in rows])
    lead = np.concatenate([np.minimum(np.abs(x).max(1) * f, top) for f in (1.0, 4.0, 11.0)])
    x = np.tile(x, (3, 1))
    x = np.concatenate([lead[:, None], x], 1)
    x[::2, 1::2] *= -1
    x = x[:len(x) // 4 * 4].reshape(-1, 128)
    return dev(x).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_every_magnitude(dtype):
    X = edges(dtype)
    q = ftk.mx4_quantize(X)
    check_pack(q, f64(X))
    check_pack(ftk.mx4_quantize(X.t().contiguous(), transpose=True), f64(X))
    if dtype == "f32":  # neighbours of every value in the last place
        for d in (-1, 1):
            Z = (X.view(torch.int32) + torch.where(X == 0, 0, d)).view(torch.float32)
            Z = torch.where(torch.isfinite(Z), Z, 0)
            check_pack(ftk.mx4_quantize(Z), f64(Z))


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_every_code_under_every_scale(out):
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(4, 64), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8), 4)[:, None].repeat(4, 1)
    q = ftk.Mx4(dev(codes), dev(scales), 128)
    want = torch.from_numpy(values_of(codes, scales, 128)).to(DTYPES[out])
    got = ftk.mx4_dequantize(q, DTYPES[out]).cpu()
    same(got, want)


@pytest.mark.parametrize("N,D,dtype,pad", [(0, 5, "f32", 0), (1, 1, "f32", 0), (1, 4096, "bf16", 0), (3, 31, "bf16", 1),
                                           (7, 32, "f16", 0), (5, 33, "f16", 3), (33, 127, "f32", 2), (64, 128, "bf16", 8),
                                           (100, 129, "bf16", 0), (129, 1000, "f32", 0), (257, 333, "f16", 5),
                                           (1000, 45, "f32", 0), (31, 2048, "bf16", 0)])
def test_pack_and_back(N, D, dtype, pad):
    print("pack", N, D, dtype, pad, flush=True)
    rng = np.random.default_rng(N + D)
    x = rng.standard_normal((N, D + pad)) * np.exp2(rng.integers(-20, 20, (N, D + pad)) * (rng.random((N, 1)) < 0.5))
    X = dev(x).to(DTYPES[dtype])[:, :D]
    for transpose in (False, True):
        q = ftk.mx4_quantize(X, transpose=transpose)
        x = f64(X).T if transpose else f64(X)
        check_pack(q, x)
        out = torch.full((x.shape[0], x.shape[1] + 2), 3.0, dtype=DTYPES[dtype], device=DEV)
        ftk.mx4_dequantize(q, DTYPES[dtype], out=out[:, 1:-1])
        want = torch.from_numpy(values(q)).to(DTYPES[dtype])
        same(out[:, 1:-1].cpu(), want)
        assert (out[:, 0] == 3).all() and (out[:, -1] == 3).all()


def test_infinities_and_nan_take_their_block():
    X = torch.ones(4, 200, device=DEV)
    X[0, 40], X[1, 199], X[2, 0] = float("inf"), float("nan"), -float("inf")
    q = ftk.mx4_quantize(X)
    v = ftk.mx4_dequantize(q)
    bad = torch.isnan(v)
    want = torch.zeros_like(bad)
    want[0, 32:64] = want[1, 192:] = want[2, :32] = True
    assert torch.equal(bad, want) and (v[~bad] == 1).all()
    W = ftk.mx4_quantize(torch.ones(3, 200, device=DEV))
    for out in (ftk.mx4_matmul(q, W, out_dtype=torch.float32), ftk.mx4_linear(X, W)):
        assert torch.isnan(out[:3]).all() and (out[3] == 200).all()
    out = ftk.mx4_matmul(W, q, out_dtype=torch.float32)
    assert torch.isnan(out[:, :3]).all() and (out[:, 3] == 200).all()


def close(got, want, size, steps, dtype):
    """A step of 128 products is off by at most 2^-23 of the magnitudes (twice what the instruction was seen to be), the sum
    over the steps by as much again for each, the result by one rounding of its type."""
    err = np.abs(f64(got) - want)
    bound = UNIT[dtype] * np.abs(want) + (steps + 8) * 2.0 ** -23 * size + STEP[dtype]
    assert np.all(err <= bound), float((err / np.maximum(bound, 1e-300)).max())


PRODUCTS = [  # N, D, F, E (0: no route), k, dtype, align, labels
    (1, 1, 1, 0, 1, "f32", 1, ""), (1, 4096, 4096, 0, 1, "bf16", 1, ""), (5, 100, 33, 0, 1, "f32", 1, ""),
    (130, 257, 70, 0, 1, "f16", 1, ""), (300, 512, 513, 0, 1, "bf16", 1, ""), (1024, 128, 256, 0, 1, "f32", 1, ""),
    (1, 512, 300, 8, 2, "bf16", 1, "even"), (7, 96, 17, 3, 1, "f32", 1, "none"), (16, 640, 129, 4, 2, "f16", 1, "one"),
    (200, 1000, 333, 13, 2, "f32", 1, "skew"), (333, 384, 256, 5, 3, "bf16", 16, "skew"), (64, 200, 65, 300, 1, "f32", 1, "even"),
    (2000, 256, 512, 4, 1, "bf16", 128, "skew"), (1500, 130, 260, 2, 2, "f32", 1, "skew"), (40, 64, 40, 8192, 1, "bf16", 1, "even"),
    (3000, 1024, 768, 6, 2, "bf16", 1, "skew"), (2500, 333, 300, 9, 3, "f32", 1, "wild"), (260, 4096, 260, 1, 1, "f32", 1, "even")]


@pytest.mark.parametrize("N,D,F,E,k,dtype,align,kind", PRODUCTS)
def test_products(N, D, F, E, k, dtype, align, kind):
    print("product", N, D, F, E, k, dtype, align, kind, flush=True)
    rng = np.random.default_rng(N + D + F)
    X = dev(rng.standard_normal((N, D)) * np.exp2(rng.integers(-3, 4, (N, D)))).to(DTYPES[dtype])
    W = ftk.mx4_quantize(dev(rng.standard_normal((max(E, 1) * F, D))).to(torch.float32))
    x, w = values_of(*pack_of(f64(X)), D), values(W).reshape(-1, F, D)
    q, steps = ftk.mx4_quantize(X), -(-D // 128)
    if E == 0:
        want, size = x @ w[0].T, np.abs(x) @ np.abs(w[0]).T
        close(ftk.mx4_linear(X, W), want, size, steps, dtype)
        close(ftk.mx4_matmul(q, W, out_dtype=DTYPES[dtype]), want, size, steps, dtype)
        return
    r = ftk.route_plan(dev(labels_of(rng, N, k, E, kind)), E, align)
    order, offsets = r.order.cpu().numpy().astype(np.int64), r.offsets.cpu().numpy()
    want, size = np.zeros((r.rows, F)), np.zeros((r.rows, F))
    for e in range(E):
        p = np.arange(offsets[e], offsets[e + 1])
        p = p[order[p] >= 0]
        want[p], size[p] = x[order[p] // k] @ w[e].T, np.abs(x[order[p] // k]) @ np.abs(w[e]).T
    for sorted_rows in (False, True):
        A = ftk.route_gather(X, r) if sorted_rows else X
        close(ftk.mx4_linear(A, W, r, gather=not sorted_rows), want, size, steps, dtype)
        close(ftk.mx4_matmul(ftk.mx4_quantize(A), W, r, gather=not sorted_rows, out_dtype=DTYPES[dtype]), want, size, steps, dtype)
    # into a part of wider rows
    out = torch.full((r.rows, F + 6), 9.0, dtype=DTYPES[dtype], device=DEV)
    ftk.mx4_linear(X, W, r, gather=True, out=out[:, 3:-3])
    close(out[:, 3:-3], want, size, steps, dtype)
    assert (out[:, :3] == 9).all() and (out[:, -3:] == 9).all()


@pytest.mark.parametrize("N,D,F,E,k,dtype,align,kind", [
    (40001, 256, 2050, 5, 1, "bf16", 1, "skew"), (20000, 384, 2100, 3, 2, "f32", 1, "skew"), (30000, 640, 2048, 4, 1, "f16", 16, "even"),
    (12000, 1024, 4096, 2, 1, "bf16", 128, "skew"), (20000, 100, 4000, 16, 2, "bf16", 1, "wild"), (9000, 1408, 4200, 3, 1, "bf16", 1, "one")])
def test_products_in_large_tiles(N, D, F, E, k, dtype, align, kind):
    """Enough rows and columns for tiles of 256 by 256: whole and broken ones, an odd and an even number of steps, rows of fewer and of
    more than 16 scales, the last 16 scales moved back into the row."""
    print("large product", N, D, F, E, k, dtype, align, kind, flush=True)
    g = torch.Generator(device=DEV).manual_seed(N)
    X = (torch.randn(N, D, generator=g, device=DEV) * torch.exp2(torch.randint(-3, 4, (N, 1), generator=g, device=DEV))).to(DTYPES[dtype])
    W = ftk.mx4_quantize(torch.randn(E * F, D, generator=g, device=DEV))
    r = ftk.route_plan(dev(labels_of(np.random.default_rng(N), N, k, E, kind)), E, align)
    x, w = ftk.mx4_dequantize(ftk.mx4_quantize(X)).double(), ftk.mx4_dequantize(W).double().view(E, F, D)
    A = ftk.route_gather(X, r)
    got = [ftk.mx4_linear(X, W, r, gather=True), ftk.mx4_linear(A, W, r),
           ftk.mx4_matmul(ftk.mx4_quantize(X), W, r, gather=True, out_dtype=DTYPES[dtype])]
    off, steps = r.offsets.tolist(), -(-D // 128)
    for e in range(E + 1):
        p = slice(off[e], off[e + 1] if e < E else r.rows)
        slot = r.order[p].long()
        rows = torch.where((slot >= 0).unsqueeze(1), x[slot.clamp(min=0) // k], 0) if e < E else x.new_zeros(slot.numel(), D)
        m = w[e].t().contiguous() if e < E else x.new_zeros(D, F)
        want, size = rows @ m, rows.abs() @ m.abs()
        bound = UNIT[dtype] * want.abs() + (steps + 8) * 2.0 ** -23 * size + STEP[dtype]
        for out in got:
            assert ((out[p].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("N,F,D,E,dtype", [(2400, 2048, 2048, 8, "bf16"), (3000, 2100, 1990, 6, "f32"), (700, 4096, 4096, 2, "f16")])
def test_sums_in_large_tiles(N, F, D, E, dtype):
    print("large outer", N, F, D, E, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(N)
    r = ftk.route_plan(dev(labels_of(np.random.default_rng(N), N, 1, E, "skew")), E, 128)
    A = ftk.route_gather(torch.randn(N, F, generator=g, device=DEV).to(DTYPES[dtype]), r)
    B = ftk.route_gather(torch.randn(N, D, generator=g, device=DEV).to(DTYPES[dtype]), r)
    qa, qb = ftk.mx4_quantize(A, transpose=True), ftk.mx4_quantize(B, transpose=True)
    a, b = ftk.mx4_dequantize(qa).double(), ftk.mx4_dequantize(qb).double()
    got, off = ftk.mx4_outer(qa, qb, r, out_dtype=DTYPES[dtype]), r.offsets.tolist()
    for e in range(E):
        p = slice(off[e], off[e + 1])
        m = b[:, p].t().contiguous()
        want, size = a[:, p] @ m, a[:, p].abs() @ m.abs()
        bound = UNIT[dtype] * want.abs() + ((off[e + 1] - off[e]) // 128 + 8) * 2.0 ** -23 * size + STEP[dtype]
        assert ((got[e].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("N,F,D,E,k,dtype,kind", [
    (1, 1, 1, 1, 1, "f32", "even"), (50, 20, 33, 3, 2, "f32", "skew"), (700, 130, 257, 5, 2, "bf16", "skew"),
    (3, 64, 64, 4, 1, "f16", "none"), (1000, 300, 129, 2, 1, "f32", "one"), (2000, 256, 512, 6, 2, "bf16", "even"),
    (300, 17, 16, 200, 1, "f32", "even"), (5000, 64, 48, 2, 1, "f32", "skew")])
def test_sums_over_an_experts_rows(N, F, D, E, k, dtype, kind):
    print("outer", N, F, D, E, k, dtype, kind, flush=True)
    rng = np.random.default_rng(N + F)
    r = ftk.route_plan(dev(labels_of(rng, N, k, E, kind)), E, 128)
    A = ftk.route_gather(dev(rng.standard_normal((N, F))).to(DTYPES[dtype]), r)
    B = ftk.route_gather(dev(rng.standard_normal((N, D))).to(DTYPES[dtype]), r)
    qa, qb = ftk.mx4_quantize(A, transpose=True), ftk.mx4_quantize(B, transpose=True)
    a, b = values_of(*pack_of(f64(A).T), r.rows), values_of(*pack_of(f64(B).T), r.rows)
    got = ftk.mx4_outer(qa, qb, r, out_dtype=DTYPES[dtype])
    offsets = r.offsets.cpu().numpy()
    for e in range(E):
        p = slice(offsets[e], offsets[e + 1])
        steps = (offsets[e + 1] - offsets[e]) // 128
        close(got[e], a[:, p] @ b[:, p].T, np.abs(a[:, p]) @ np.abs(b[:, p]).T, steps, dtype)
    whole = ftk.mx4_outer(qa, qb, out_dtype=torch.float32)
    close(whole[0], a @ b.T, np.abs(a) @ np.abs(b).T, -(-r.rows // 128), "f32")


def test_gradient_of_the_matrices_against_differences():
    """Rows that 4 bits hold exactly, in either direction: moving one element of a matrix from one value to another moves
    sum(dY * product) by the step times its gradient.  All sums are exact in 32 bits."""
    rng = np.random.default_rng(6)
    N, D, F, E = 200, 96, 40, 3
    r = ftk.route_plan(dev(labels_of(rng, N, 1, E, "skew")), E, 128)
    held = (r.order >= 0).unsqueeze(1)
    pick = lambda n, d: dev(rng.choice(TABLE, (n, d)) * rng.choice([-1, 1], (n, d))).float()  # noqa: E731
    X, dY, W = pick(r.rows, D) * held, pick(r.rows, F) * held, pick(E * F, D)
    X[:, :3], dY[:, :2], W[:, 0] = 6.0 * held, 6.0 * held, 6.0
    X[::32] = 6.0 * held[::32]
    dY[::32] = 6.0 * held[::32]
    loss = lambda W: float((dY.double() * ftk.mx4_linear(X, ftk.mx4_quantize(W), r).double()).sum())  # noqa: E731
    dW = ftk.mx4_outer(ftk.mx4_quantize(dY, transpose=True), ftk.mx4_quantize(X, transpose=True), r).view(E * F, D)
    formula = torch.zeros(E * F, D, dtype=torch.float64)
    o = r.offsets.tolist()
    for e in range(E):
        formula[e * F:(e + 1) * F] = (dY[o[e]:o[e + 1]].double().t() @ X[o[e]:o[e + 1]].double()).cpu()
    assert torch.equal(dW.double().cpu(), formula)
    base = loss(W)
    for i in range(0, E * F, 11):
        Z = W.clone()
        j = 1 + (7 * i) % (D - 1)
        Z[i, j] = 0.0 if W[i, j] != 0 else 4.0
        assert loss(Z) - base == float((Z - W)[i, j]) * float(dW[i, j])
    # rows' gradient: the same product with the transposed matrices
    WT = W.view(E, F, D).transpose(1, 2).reshape(E * D, F).contiguous()
    WT[:, 0::32] = 6.0
    dX = ftk.mx4_linear(dY, ftk.mx4_quantize(WT), r)
    for e in range(E):
        rows = slice(o[e], o[e + 1])
        assert torch.equal(dX[rows].double(), dY[rows].double() @ WT[e * D:(e + 1) * D].double().t().contiguous())


def test_offsets_that_lie():
    """Offsets are device data: whatever they hold, nothing outside the arrays is touched."""
    rng = np.random.default_rng(9)
    N, D, F, E = 100, 128, 64, 3
    X = dev(rng.standard_normal((N, D)).astype(np.float32))
    W = ftk.mx4_quantize(dev(rng.standard_normal((E * F, D)).astype(np.float32)))
    q = ftk.mx4_quantize(X, transpose=True)
    order = torch.arange(N, dtype=torch.int32, device=DEV)
    pos = order.view(N, 1)
    for offsets in ([0, -5, 1000, 2 ** 31 - 1], [7, 3, 90, 10], [-2 ** 31, 2 ** 31 - 1, -1, 5], [0, 0, 0, 0]):
        off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        r = ftk.Route(off, off[:E], order, pos, 128)
        whole = torch.full((N + 2, F), 5.0, device=DEV)
        ftk.mx4_linear(X, W, r, out=whole[1:-1])
        assert (whole[0] == 5).all() and (whole[-1] == 5).all()
        ftk.mx4_outer(q, q, r)
        torch.cuda.synchronize()
    assert (whole[1:-1] == 0).all()
    lying = torch.full((N,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    r = ftk.Route(torch.tensor([0, 10, 50, 100], dtype=torch.int32, device=DEV), off[:E], lying, pos, 1)
    assert (ftk.mx4_linear(X, W, r, gather=True) == 0).all()


def test_packed_rows_beyond_32_bits():
    """More than 2^32 bytes of codes."""
    N, D = 4_200_000, 2048
    X = torch.zeros(N, D, dtype=torch.bfloat16, device=DEV)
    X[:, 5] = torch.arange(N, device=DEV) % 3 + 1
    X[:, -1] = 1
    q = ftk.mx4_quantize(X)
    assert q.codes.numel() > 2 ** 32
    del X
    W = torch.zeros(2, D, device=DEV)
    W[0, 5] = W[1, -1] = 2
    out = ftk.mx4_matmul(q, ftk.mx4_quantize(W), out_dtype=torch.float32)
    want = (torch.arange(N, device=DEV) % 3 + 1) * 2.0
    assert torch.equal(out[:, 0], want) and (out[:, 1] == 2).all()
    # as the experts' side
    out = ftk.mx4_matmul(ftk.mx4_quantize(W), q, out_dtype=torch.float32)
    assert torch.equal(out[0], want) and (out[1] == 2).all()


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(4)
    N, D, F, E = 900, 256, 320, 5
    X = dev(rng.standard_normal((N, D)).astype(np.float32))
    W = ftk.mx4_quantize(dev(rng.standard_normal((E * F, D)).astype(np.float32)))
    r = ftk.route_plan(dev(labels_of(rng, N, 2, E, "skew")), E)
    want = ftk.mx4_linear(X, W, r, gather=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ftk.mx4_linear(X, W, r, gather=True)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    ws = torch.empty(ftk.mx4_workspace_bytes(N, D, r.rows, E) + 256, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ftk.mx4_linear(X, W, r, gather=True, out=out, workspace=ws)
    for i in range(3):
        X.mul_(0.7)
        want = ftk.mx4_linear(X, W, r, gather=True)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("M", [1, 8, 16, 40, 700])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_without_a_slot_are_zero_beside_nan_weights(M, dtype):
    """An output row whose order is -1 becomes zero whatever its expert's matrix holds, for few rows and many."""
    rng = np.random.default_rng(21)
    N, D, F, E = max(1, M // 2), 160, 70, 2
    X = dev(rng.standard_normal((N, D)).astype(np.float32)).to(DTYPES[dtype])
    B = rng.standard_normal((E * F, D)).astype(np.float32)
    B[3, 7] = np.nan  # of the first expert
    B[F + 5, 150] = np.inf  # of the second
    W = ftk.mx4_quantize(dev(B))
    order = torch.arange(M, dtype=torch.int32, device=DEV) % (2 * N)
    order[::2] = -1
    first = (M + 1) // 2
    off = torch.tensor([0, first, M], dtype=torch.int32, device=DEV)
    r = ftk.Route(off, off[:E], order, torch.arange(2 * N, dtype=torch.int32, device=DEV).view(N, 2), 1)
    for out in (ftk.mx4_linear(X, W, r, gather=True), ftk.mx4_matmul(ftk.mx4_quantize(X), W, r, gather=True, out_dtype=X.dtype)):
        assert (out[::2] == 0).all()
        nan = torch.isnan(out)
        want = torch.zeros_like(nan)
        want[1:first:2, 3] = True
        want[first + (first + 1) % 2::2, 5] = True
        assert torch.equal(nan, want)


def test_sums_over_very_many_rows():
    """More than 2^25 rows, beyond which lines of codes are too long for the tiles' 32-bit offsets.  All sums are exact."""
    big, rows = 2 ** 25, 2 ** 25 + 384
    A = torch.zeros(rows, 3, dtype=torch.float16, device=DEV)
    B = torch.zeros(rows, 2, dtype=torch.float16, device=DEV)
    A[:, 0] = 1
    A[big - 1, 1], A[-1, 1] = 3, 2
    A[::1024, 2] = 1
    B[:, 0] = 1
    B[big - 1, 1], B[-1, 1] = 2, -4
    off = torch.tensor([0, big, rows], dtype=torch.int32, device=DEV)
    order = torch.arange(rows, dtype=torch.int32, device=DEV)
    r = ftk.Route(off, off[:2], order, order.view(rows, 1), 128)
    got = ftk.mx4_outer(ftk.mx4_quantize(A, transpose=True), ftk.mx4_quantize(B, transpose=True), r)
    assert got[0].tolist() == [[2.0 ** 25, 2.0], [3.0, 6.0], [2.0 ** 15, 0.0]]
    assert got[1].tolist() == [[384.0, -4.0], [2.0, -8.0], [1.0, 0.0]]


@pytest.mark.parametrize("M,D,F,offsets,dtype", [
    (1, 40, 20, [1, 1], "f32"), (5, 100, 33, [3, 4, 5], "bf16"), (16, 640, 129, [1, 9, 9, 12], "f16"), (16, 64, 40, [16, 16], "f32"),
    (40, 64, 40, list(range(5, 105)), "bf16"), (200, 1000, 333, [70, 130, 131, 190], "f32"), (3000, 512, 768, [129, 2000, 2000, 2900], "bf16"),
    (300, 130, 64, [300, 300, 300], "f32"), (20000, 384, 2100, [1000, 9000, 19999], "bf16"), (12000, 1100, 4096, [255, 12000], "f16")])
def test_rows_before_the_first_expert_are_zero(M, D, F, offsets, dtype):
    """Offsets that begin above 0: the rows in front belong to no expert, as those behind the last, whatever the first one's matrix holds."""
    print("first offset", M, D, F, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(M)
    E = len(offsets) - 1
    X = torch.randn(M, D, generator=g, device=DEV).to(DTYPES[dtype])
    B = torch.randn(E * F, D, generator=g, device=DEV)
    B[3, 7] = float("nan")  # of the first expert
    W = ftk.mx4_quantize(B)
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    order = torch.randint(-1, 2 * M, (M,), generator=g, device=DEV).int()
    r = ftk.Route(off, off[:E], order, torch.zeros(M, 2, dtype=torch.int32, device=DEV), 1)
    x, w = ftk.mx4_dequantize(ftk.mx4_quantize(X)).double(), ftk.mx4_dequantize(W).double().view(E, F, D)
    for gather in (False, True):
        source = torch.where(order < 0, -1, order // 2).long() if gather else torch.arange(M, device=DEV)
        rows = torch.where((source >= 0).unsqueeze(1), x[source.clamp(min=0)], 0)
        want, size = torch.zeros(M, F, dtype=torch.float64, device=DEV), torch.zeros(M, F, dtype=torch.float64, device=DEV)
        for e in range(E):
            p, m = slice(min(offsets[e], M), min(offsets[e + 1], M)), w[e].t().contiguous()
            want[p], size[p] = rows[p] @ m, rows[p].abs() @ m.abs()
        empty = source < 0
        empty[:offsets[0]] = True
        empty[min(offsets[E], M):] = True
        want[empty], size[empty] = 0, 0  # (also where zeros met NaN)
        nan = torch.isnan(want)
        bound = UNIT[dtype] * want.abs() + (-(-D // 128) + 8) * 2.0 ** -23 * size + STEP[dtype]
        for out in (ftk.mx4_linear(X, W, r, gather=gather), ftk.mx4_matmul(ftk.mx4_quantize(X), W, r, gather=gather, out_dtype=DTYPES[dtype])):
            assert (out[empty] == 0).all()
            assert torch.equal(torch.isnan(out), nan)
            assert ((out.double() - want).abs() <= bound)[~nan].all()


@pytest.mark.parametrize("N,F,D", [(20000, 2100, 384), (6000, 768, 512), (1500, 2048, 2048)])
def test_large_tiles_in_a_graph(N, F, D):
    """Products and sums over rows in tiles that take more than 64 KB of LDS, and the packing before them."""
    g = torch.Generator(device=DEV).manual_seed(N)
    E = 3
    X = torch.randn(N, D, generator=g, device=DEV).bfloat16()
    W = ftk.mx4_quantize(torch.randn(E * F, D, generator=g, device=DEV))
    r = ftk.route_plan(dev(labels_of(np.random.default_rng(N), N, 1, E, "skew")), E, 128)
    ws = torch.empty(ftk.mx4_workspace_bytes(N, D, r.rows, E) + 256, dtype=torch.uint8, device=DEV)
    A = ftk.route_gather(X, r)
    qy, qa = ftk.mx4_quantize(ftk.mx4_linear(X, W, r, gather=True), transpose=True), ftk.mx4_quantize(A, transpose=True)
    out = torch.empty(r.rows, F, dtype=X.dtype, device=DEV)
    sums = torch.empty(E, F, D, device=DEV)

    def step():
        ftk.mx4_linear(X, W, r, gather=True, out=out, workspace=ws)
        ftk.route_gather(X, r, out=A)
        ftk.mx4_quantize(out, transpose=True, out=qy)
        ftk.mx4_quantize(A, transpose=True, out=qa)
        ftk.mx4_outer(qy, qa, r, out=sums)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        X.mul_(-0.6)
        step()
        want = out.clone(), sums.clone()
        out.fill_(7), sums.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(sums, want[1])
        assert torch.isfinite(sums).all() and sums.abs().max() > 0
