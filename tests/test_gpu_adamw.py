"""The update of many weights at once against its formulas: states bit for bit, weights in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_01391_amd import binding as ftk
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

F, B, H = torch.float32, torch.bfloat16, torch.float16
HALF = {F: 2.0 ** -24, B: 2.0 ** -8, H: 2.0 ** -11}
SIZES = [1, 7, 8, 31, 32, 33, 64, 255, 2047, 2048, 2049, 8191, 8192, 8193, 70001]
M64 = (1 << 64) - 1


def mix64(z):
    z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ z >> 27) * 0x94D049BB133111EB) & M64
    return z ^ z >> 31


def random32(seed, step, place, n):
    key = mix64((mix64((seed + 0x9E3779B97F4A7C15 * step) & M64) + place) & M64)
    x = np.arange(n, dtype=np.uint64) ^ np.uint64(mix64(key) & 0xFFFFFFFF)
    for shift, factor in ((16, 0xC8E1ED59), (15, 0x876BA2B3), (16, 1)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return x.astype(np.int64)


def units(M):
    """What the codes without a sign stand for, in units of their block."""
    c = np.arange(16 << M)
    return np.where(c < 1 << M, c, ((1 << M) + c % (1 << M)) * 2.0 ** np.maximum((c >> M) - 1, 0)).astype(np.float64)


def decode(codes, scales, M):
    v = units(M)[codes & ((16 << M) - 1)] * 2.0 ** (scales.astype(np.float64).repeat(32)[:codes.size] - 127)
    return np.where((codes > 127) & (M == 3), -v, v)


def encode(x, M, random):
    """Codes and scales of 32-bit numbers: the lower neighbour's code, one more where what is left and the random part of the step
    reach a step."""
    n = x.size
    size = np.abs(np.pad(x, (0, -n % 32))).reshape(-1, 32)
    bits = size.max(1).astype(np.float32).view(np.int32).astype(np.int64)
    scales = np.maximum(((bits + (1 << (23 - M)) - 1) >> 23) - (M + 14), 0)
    y = (size.astype(np.float64) * 2.0 ** (127.0 - scales[:, None])).reshape(-1)[:n]
    table = units(M)
    # (below the first binade the number counts to 32 bits of itself and 2^M)
    y = np.where(y < 1 << M, (y + (1 << M)).astype(np.float32).astype(np.float64) - (1 << M), y)
    low = np.searchsorted(table, y, side="right") - 1
    step = np.append(table, 2 * table[-1] - table[-2])[low + 1] - table[low]
    codes = low + ((y - table[low]) / step + random >= 1)
    if M == 4:
        codes = np.where(x > 0, np.maximum(codes, 1), codes)
        return codes.astype(np.uint8), scales.astype(np.uint8)
    return (codes + 128 * np.signbit(x)).astype(np.uint8), scales.astype(np.uint8)


def one_step(p, g, m, v, t, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, lr_scale=1.0, grad_scale=1.0):
    """m', v' (32-bit numbers) and w' in 64 bits, with the size of w's change."""
    f = np.float32
    g = g.astype(f) * f(grad_scale)
    m = f(beta1) * m.astype(f) + f(1 - beta1) * g
    v = f(beta2) * v.astype(f) + f(1 - beta2) * (g * g)
    rate = lr * float(f(lr_scale))
    update = (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return m, v, p - rate * (weight_decay * p + update), rate * (abs(update) + abs(weight_decay * p))


def setup(sizes, dtype, grads, bits, master, seed, aligned):
    g = torch.Generator(device=DEV).manual_seed(seed)
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // 64) * 64 if aligned else n
    flat = lambda scale: torch.randn(at + 1, generator=g, device=DEV) * scale  # noqa: E731
    views = lambda t: [t[0 if aligned else 1:][a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
    weights = flat(0.05)
    params, masters = views(weights.to(dtype)), views(weights.clone()) if master else None
    gr = flat(1e-2)
    gr[torch.rand(at + 1, generator=g, device=DEV) < 0.02] *= 50
    gr[torch.rand(at + 1, generator=g, device=DEV) < 0.1] = 0
    return params, masters, views(gr.to(grads))


def numpy(t):
    return t.detach().cpu().numpy() if t.dtype == torch.uint8 else t.detach().double().cpu().numpy()


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grads,master", [(F, F, False), (F, B, False), (F, H, False), (B, B, False), (B, B, True), (B, F, True),
                                                (B, F, False), (H, H, True), (H, F, True), (H, H, False), (H, F, False)])
def test_steps(dtype, grads, master, bits, aligned):
    """Three steps from zero states: the states of every step exactly, the weights within their roundings."""
    params, masters, gs = setup(SIZES, dtype, grads, bits, master, 3 + bits, aligned)
    state = ftk.AdamW(params, bits, master=masters)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    for t in range(1, 4):
        old = [numpy(w) for w in (masters if master else params)]
        before = [(numpy(m), numpy(v)) for m, v in zip(state.m, state.v)]
        if bits == 8:
            before = [(decode(m, numpy(a), 3), decode(v, numpy(b), 4))
                      for (m, v), a, b in zip(before, state.m_scales, state.v_scales)]
        step.add_(1)
        options = dict(lr=2e-3, weight_decay=0.1 * t, seed=77 << 40)
        ftk.adamw_step(state, gs, step, **options)
        for i, n in enumerate(SIZES):
            m, v, w, change = one_step(old[i], numpy(gs[i]), *before[i], t, lr=2e-3, weight_decay=0.1 * t)
            if bits == 32:
                assert np.array_equal(numpy(state.m[i]), m) and np.array_equal(numpy(state.v[i]), v)
            else:
                r = random32(77 << 40, t, i, n)
                for codes, scales, x, M, u in ((state.m, state.m_scales, m, 3, r >> 16), (state.v, state.v_scales, v, 4, r & 0xFFFF)):
                    want = encode(x, M, u / 65536.0)
                    assert np.array_equal(numpy(scales[i]), want[1]), (i, M)
                    assert np.array_equal(numpy(codes[i]), want[0]), (i, M)
            # a dozen roundings of the change (1 - beta^t is known to 2^-22), two of the weight
            tol = 40 * 2.0 ** -24 * change + 2 * 2.0 ** -24 * abs(w)
            if master:
                assert (abs(numpy(masters[i]) - w) <= tol).all()
                assert torch.equal(params[i], masters[i].to(dtype))
            else:
                least = 2.0 ** -25 if dtype == H else 0
                assert (abs(numpy(params[i]) - w) <= tol + HALF[dtype] * abs(w) * 1.01 + least).all()
    if bits == 8:
        for dt in (F, B, H):
            ms, vs = ftk.adamw_moments(state, dtype=dt)
            for i in range(len(SIZES)):
                for got, codes, scales, M in ((ms[i], state.m[i], state.m_scales[i], 3), (vs[i], state.v[i], state.v_scales[i], 4)):
                    want = torch.from_numpy(decode(numpy(codes), numpy(scales), M))
                    assert torch.equal(got.cpu(), want.to(dt)), (dt, i, M)


def test_states_of_all_magnitudes():
    """Gradients from 2^-60 to 2^60, block by block and within blocks: codes and scales exactly, twice in a row."""
    rng = np.random.default_rng(1)
    n = 32 * 400
    size = np.repeat(rng.uniform(-60, 60, 400), 32) + rng.uniform(-20, 0, n) * (rng.random(n) < 0.5)
    g = (rng.standard_normal(n) * 2.0 ** size).astype(np.float32)
    p = torch.zeros(n, device=DEV)
    state = ftk.AdamW([p], 8)
    for t in (1, 2):
        before = [decode(numpy(c[0]), numpy(s[0]), M) for c, s, M in ((state.m, state.m_scales, 3), (state.v, state.v_scales, 4))]
        ftk.adamw_step(state, [torch.from_numpy(g).to(DEV)], torch.full((1,), t, dtype=torch.int64, device=DEV), seed=2)
        with np.errstate(over="ignore"):
            m, v, _, _ = one_step(np.zeros(n), g, *before, t)
        r = random32(2, t, 0, n)
        for codes, scales, x, M, u in ((state.m, state.m_scales, m, 3, r >> 16), (state.v, state.v_scales, v, 4, r & 0xFFFF)):
            want = encode(x, M, u / 65536.0)
            assert np.array_equal(numpy(scales[0]), want[1]) and np.array_equal(numpy(codes[0]), want[0]), (t, M)
        g = (g * rng.uniform(-2, 2, n)).astype(np.float32)
        ms, vs = ftk.adamw_moments(state)
        assert np.array_equal(numpy(ms[0]), decode(numpy(state.m[0]), numpy(state.m_scales[0]), 3))
        assert np.array_equal(numpy(vs[0]), decode(numpy(state.v[0]), numpy(state.v_scales[0]), 4))


def test_more_elements_than_32_bits_count():
    """The end of a tensor of 2^32 elements and some: its states exactly, from bits of their own."""
    n, tail = (1 << 32) + 5000, 4500
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(3)
    g[-tail:] = torch.from_numpy(rng.standard_normal(tail)).to(DEV)
    state = ftk.AdamW([p], 8)
    ftk.adamw_step(state, [g], torch.ones(1, dtype=torch.int64, device=DEV), seed=6)
    assert not p[:n - tail].any() and not state.v[0][:n - tail].any()
    lead = (n - tail) % 32  # whole blocks
    grads = np.concatenate([np.zeros(lead), numpy(g[-tail:])])
    m, v, w, _ = one_step(0 * grads, grads, 0 * grads, 0 * grads, 1)
    key = mix64((mix64((mix64((6 + 0x9E3779B97F4A7C15) & M64) + 0) & M64) + 1) & M64)
    x = np.arange(n - tail - lead - (1 << 32), n - (1 << 32), dtype=np.uint64) ^ np.uint64(key & 0xFFFFFFFF)
    for shift, factor in ((16, 0xC8E1ED59), (15, 0x876BA2B3), (16, 1)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    r = x.astype(np.int64)
    for codes, want in ((state.m[0], encode(m, 3, (r >> 16) / 65536.0)[0]), (state.v[0], encode(v, 4, (r & 0xFFFF) / 65536.0)[0])):
        assert np.array_equal(numpy(codes[n - tail - lead:]), want)


def test_empty_tensors_and_shared_gradients():
    """Tensors without elements are passed over; one gradient may serve two weights."""
    a, b, none = torch.ones(50, device=DEV), torch.ones(50, device=DEV), torch.ones(0, device=DEV)
    state = ftk.AdamW([a, none, b], 8)
    g = torch.linspace(-1, 1, 50, device=DEV)
    ftk.adamw_step(state, [g, none.clone(), g], torch.ones(1, dtype=torch.int64, device=DEV))
    assert torch.equal(a, b) and not torch.equal(a, torch.ones_like(a))
    assert [t.numel() for t in ftk.adamw_moments(state)[0]] == [50, 0, 50]
    ftk.adamw_step(state, [None, None, None], torch.ones(1, dtype=torch.int64, device=DEV))
    assert torch.equal(a, b)


def test_more_tensors_than_a_launch_takes():
    """With tensors left out here and there: those stay, the others keep their place in the list."""
    sizes = [1 + (i * 37) % 300 for i in range(170)]
    for bits in (8, 32):
        params, _, gs = setup(sizes, F, F, bits, False, 9, False)
        gs = [None if i % 5 == 2 else g for i, g in enumerate(gs)]
        state = ftk.AdamW(params, bits)
        before = [p.clone() for p in params]
        ftk.adamw_step(state, gs, torch.ones(1, dtype=torch.int64, device=DEV), seed=5)
        for i, (p, q) in enumerate(zip(params, before)):
            if gs[i] is None:
                assert torch.equal(p, q) and not state.m[i].any() and not state.v[i].any()
                continue
            m, v, w, change = one_step(numpy(q), numpy(gs[i]), 0 * numpy(q), 0 * numpy(q), 1)
            assert (abs(numpy(p) - w) <= 40 * 2.0 ** -24 * change + 2 * 2.0 ** -24 * abs(w)).all()
            if bits == 8:
                assert np.array_equal(numpy(state.v[i]), encode(v, 4, (random32(5, 1, i, sizes[i]) & 0xFFFF) / 65536.0)[0])


def test_scales_from_the_device():
    params, _, gs = setup([1000, 77], F, F, 32, False, 4, True)
    twin = [p.clone() for p in params]
    state, other = ftk.AdamW(params), ftk.AdamW(twin)
    step = torch.full((1,), 5, dtype=torch.int64, device=DEV)
    half, quarter = torch.full((1,), 0.5, device=DEV), torch.full((1,), 0.25, device=DEV)
    ftk.adamw_step(state, gs, step, lr=1e-2, lr_scale=half, grad_scale=quarter)
    ftk.adamw_step(other, [g * 0.25 for g in gs], step, lr=5e-3)
    for a, b in zip(params + state.m + state.v, twin + other.m + other.v):
        assert torch.allclose(a, b, rtol=1e-6, atol=0)


def test_rounding_has_no_bias():
    """A million equal states: their mean is the number, within five standard deviations; successive steps and both states
    round independently."""
    n = 1 << 20
    p = torch.zeros(n, device=DEV)
    g = torch.full((n,), 0.0123, device=DEV)
    g[::32] = 1.0  # every block's scale
    state = ftk.AdamW([p], 8)
    drawn = []
    for t in (1, 2):
        state.m[0].zero_(), state.v[0].zero_()
        ftk.adamw_step(state, [g], torch.full((1,), t, dtype=torch.int64, device=DEV), seed=1)
        for values, x in zip(ftk.adamw_moments(state), (np.float32(0.1) * np.float32(0.0123), np.float32(0.001) * np.float32(0.0123) ** 2)):
            small = values[0].view(-1, 32)[:, 1:].double().flatten()
            lo, hi = float(small.min()), float(small.max())
            assert lo < x < hi and int((small == lo).sum() + (small == hi).sum()) == small.numel()
            share = (x - lo) / (hi - lo)
            up = (small == hi).double()
            sigma = (share * (1 - share) / small.numel()) ** 0.5
            assert abs(float(up.mean()) - share) < 5 * sigma + 2.0 ** -16
            drawn.append((up - up.mean()) / up.std())
        assert (values[0] > 0).all()
    for i in range(4):
        assert abs(float((drawn[i][1:] * drawn[i][:-1]).mean())) < 6e-3  # neighbours
        for j in range(i):
            assert abs(float((drawn[i] * drawn[j]).mean())) < 6e-3


def test_states_decay():
    """Without gradients the second moment falls by its factor at every step, though a step is far less than half a code."""
    p = torch.zeros(1 << 16, device=DEV)
    state = ftk.AdamW([p], 8)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    for t in range(400):
        step.add_(1)
        ftk.adamw_step(state, [torch.full_like(p, 1.0 if t == 0 else 0.0)], step, lr=0.0, seed=3)
    left = float(ftk.adamw_moments(state)[1][0].double().mean()) / 0.001
    # 400 roundings of relative variance 0.001 / 16 at most, averaged over 65536: 7e-4; five times that
    assert abs(left / 0.999 ** 399 - 1) < 3.5e-3


@pytest.mark.parametrize("bits", [8, 32])
def test_bad_gradients_stay_in_their_block(bits):
    n = 200
    p = torch.ones(n, device=DEV)
    g = torch.full((n,), 0.1, device=DEV)
    g[40], g[150] = float("nan"), float("inf")
    state = ftk.AdamW([p], bits)
    ftk.adamw_step(state, [g], torch.ones(1, dtype=torch.int64, device=DEV))
    bad = torch.zeros(n, dtype=torch.bool, device=DEV)
    bad[[40, 150]] = True
    assert p[~bad].isfinite().all() and p[40].isnan() and p[150].isnan()
    if bits == 8:
        blocks = torch.tensor([0, 1, 0, 0, 1, 0, 0], dtype=torch.bool, device=DEV)
        assert torch.equal(state.m_scales[0] == 255, blocks) and torch.equal(state.v_scales[0] == 255, blocks)
        spread = blocks.repeat_interleave(32)[:n]
        for values in ftk.adamw_moments(state):
            assert torch.equal(values[0].isnan(), spread)
    else:
        assert state.m[0][~bad].isfinite().all()


@pytest.mark.parametrize("bits", [8, 32])
def test_graph(bits):
    """A captured step with the counter's increment, replayed: what eager steps give, bit for bit."""
    params, masters, gs = setup([3000, 65], B, B, bits, True, 6, True)
    twin, twins = [p.clone() for p in params], [m.clone() for m in masters]
    state, other = ftk.AdamW(params, bits, master=masters), ftk.AdamW(twin, bits, master=twins)
    step, count = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        ftk.adamw_step(state, gs, step, seed=8)
    for _ in range(4):
        graph.replay()
        count.add_(1)
        ftk.adamw_step(other, gs, count, seed=8)
        torch.cuda.synchronize()
        for a, b in zip(params + masters + state.m + state.v, twin + twins + other.m + other.v):
            assert torch.equal(a, b)


def test_refusals():
    p = torch.zeros(64, device=DEV)
    step = torch.ones(1, dtype=torch.int64, device=DEV)
    state = ftk.AdamW([p])
    for call in (lambda: ftk.AdamW([p, p]), lambda: ftk.AdamW([p[:40], p[30:]]), lambda: ftk.AdamW([p], m=[p]), lambda: ftk.AdamW([p[::2]]),
                 lambda: ftk.AdamW([p, p.bfloat16()]), lambda: ftk.AdamW([p], master=True), lambda: ftk.AdamW([p], 8, m=[torch.zeros_like(p)]),
                 lambda: ftk.adamw_step(state, [], step), lambda: ftk.adamw_step(state, [p[:5]], step),
                 lambda: ftk.adamw_step(state, [p.clone()], step.int()), lambda: ftk.adamw_step(state, [p.clone()], step.cpu()),
                 lambda: ftk.adamw_step(state, [p.clone()], step, lr_scale=step), lambda: ftk.adamw_moments(state),
                 lambda: ftk.adamw_step(state, [p.cpu()], step)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ftk.adamw_step(state, [p.double()], step)
    with pytest.raises(ftk.FtkError):
        ftk.adamw_step(state, [p.clone()], step, beta1=1.0)


def test_weights_that_moved():
    """Weights that a program laid elsewhere are not looked for at their old place."""
    p = torch.nn.Parameter(torch.ones(40, device=DEV))
    state, step = ftk.AdamW([p]), torch.ones(1, dtype=torch.int64, device=DEV)
    old = p.data
    p.data = old.clone()
    with pytest.raises(ValueError):
        ftk.adamw_step(state, [torch.ones_like(old)], step)
    assert (old == 1).all() and (p == 1).all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("by_scale", [True, False])
@pytest.mark.parametrize("decay", [1e-7, 3e-8, 1e-8])
def test_small_decay(decay, by_scale, bits):
    """A decay of about half a step of the weights' numbers and less, as at the end of a schedule: beside updates of all sizes, which
    spread the rounding evenly, it is kept on average, and every weight is off by that one rounding alone."""
    n = 1 << 20
    g = torch.Generator(device=DEV).manual_seed(12)
    p, grad = 1 + torch.rand(n, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
    old, gr = numpy(p), numpy(grad)
    scale = torch.full((1,), 2.0 ** -10, device=DEV) if by_scale else None
    rate = 1.024 if by_scale else 1e-3
    ftk.adamw_step(ftk.AdamW([p], bits), [grad], torch.ones(1, dtype=torch.int64, device=DEV), lr=rate, lr_scale=scale, eps=0.5,
                   weight_decay=decay / 1e-3)
    _, _, w, change = one_step(old, gr, 0 * old, 0 * old, 1, lr=1e-3, eps=0.5, weight_decay=decay / 1e-3)
    off = numpy(p) - w
    # half a step of the result: 2^-24 in [1, 2), 2^-23 from 2 on, where a weight of less may arrive; a dozen roundings of the change
    half = np.spacing(w.astype(np.float32)).astype(np.float64) / 2
    assert (abs(off) <= 1.001 * half + 40 * 2.0 ** -24 * change).all()
    # a rounding's standard deviation is a step over the root of 12; what the change's roundings have in common (40 at the most) meets
    # updates of either sign, whose mean is below five of its deviations
    limit = 5 * (2.0 ** -23 / 12 ** 0.5 + 40 * 2.0 ** -24 * 1e-3) / n ** 0.5 + 40 * 2.0 ** -24 * 2 * decay
    assert abs(off.mean()) <= limit


@pytest.mark.parametrize("grads", [F, B, H])
@pytest.mark.parametrize("pattern", [0xFFFFFFFF, 0xFFF80001, 0xFFC00000, 0x7FFFFFFF])
def test_every_nan_marks_its_block(pattern, grads):
    """Gradients that are NaN of either sign and any payload, all bits set as in memory that nobody wrote among them."""
    bits = np.full(1, pattern if grads == F else pattern >> 16, dtype=np.uint32 if grads == F else np.uint16)
    if grads == H:
        bits |= 0x7C00  # (fp16's exponent)
    bad = torch.from_numpy(bits.view(np.int32 if grads == F else np.int16)).to(DEV).view(grads)
    assert bool(bad.isnan())
    g = torch.full((96,), 0.1, device=DEV).to(grads)
    g[40] = bad[0]
    p = torch.ones(96, device=DEV)
    state = ftk.AdamW([p], 8)
    ftk.adamw_step(state, [g], torch.ones(1, dtype=torch.int64, device=DEV))
    assert state.m_scales[0].tolist()[1] == 255 and state.v_scales[0].tolist()[1] == 255
    for values in ftk.adamw_moments(state):
        assert values[0].view(3, 32).isnan().all(1).tolist() == [False, True, False] and int(values[0].isnan().sum()) == 32
    assert int(p.isnan().sum()) == 1


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [0.0, 1e-39, 1e-30, 1e-20, 1.9e-12, 2.1e-12, 1e-8])
def test_small_gradients_and_small_eps(eps, bits):
    """Second moments below the normal numbers, beside an eps that is smaller still: the update is the formula's."""
    rng = np.random.default_rng(3)
    # (a block of each magnitude, as 8-bit states share their scale)
    g = np.repeat(10.0 ** np.array([0, -5, -10, -15, -18, -18.7, -19, -19.5, -20, -20.5]), 32) * rng.uniform(0.5, 1, 320)
    g = (g * rng.choice([-1, 1], 320)).astype(np.float32)
    if eps:
        g[::7] = 0
    p = torch.full((320,), 0.25, device=DEV)
    ftk.adamw_step(ftk.AdamW([p], bits), [torch.from_numpy(g).to(DEV)], torch.ones(1, dtype=torch.int64, device=DEV), lr=0.5, eps=eps,
                   weight_decay=0.0)
    float_eps = float(np.float32(eps))
    _, _, w, change = one_step(np.full(320, 0.25), g, np.zeros(320), np.zeros(320), 1, lr=0.5, eps=float_eps, weight_decay=0.0)
    assert np.isfinite(w).all()
    # a dozen roundings of the change, two of the weight
    assert (abs(numpy(p) - w) <= 40 * 2.0 ** -24 * change + 2 * 2.0 ** -24 * abs(w)).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_states_that_were_replaced(bits):
    """Other tensors in the lists of states are refused rather than passed over; memory that a state's tensor gave up is not written
    to once it is another's."""
    n, step = 1 << 16, torch.ones(1, dtype=torch.int64, device=DEV)
    p, g = torch.zeros(n, dtype=B, device=DEV), torch.ones(n, dtype=B, device=DEV)
    for name in ("m", "v", "master") + (("m_scales", "v_scales") if bits == 8 else ()):
        state = ftk.AdamW([p], bits, master=True)
        tensors = getattr(state, name)
        tensors[0] = tensors[0].clone()
        with pytest.raises(ValueError):
            ftk.adamw_step(state, [g], step)
        if bits == 8:
            with pytest.raises(ValueError):
                ftk.adamw_moments(state)
    assert not p.any()
    state = ftk.AdamW([p], bits, master=True)
    for tensors in (state.m, state.v, state.master):
        tensors[0].data = tensors[0].data.clone()
    torch.cuda.synchronize()
    others = [torch.full((n,), 3, dtype=t.dtype, device=DEV) for t in (state.m[0], state.v[0], state.master[0]) for _ in range(3)]
    ftk.adamw_step(state, [g], step)
    assert all((t == 3).all() for t in others)
