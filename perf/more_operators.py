"""One training step of routed experts, as timed cases: the gate that learns which experts a token goes to and keeps them
evenly used (probabilities, best k, counts, balance loss, gradients), the softmax cross entropy of rows against many
classes whose logits are not kept (loss, gradients), and the update of many weights at once (AdamW, states in 32 bits or
in 8 under a power of two per 32 elements).

`own` chooses between the plain form of every operator (elementary torch operations in 32 bits) and the library's entry
points; both take the same state."""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


def _gate(name, N, E, k, dtype, normalise=True, train=True, masked=False):
    return _named(name, dict(op="gate", N=N, E=E, k=k, dtype=dtype, normalise=normalise, train=train, masked=masked))


def _loss(name, N, V, D, dtype, train=True, bias=False):
    return _named(name, dict(op="loss", N=N, V=V, D=D, dtype=dtype, train=train, bias=bias))


def _adamw(name, tensors, total, dtype, grads, bits, master, ragged):
    return _named(name, dict(op="adamw", tensors=tensors, total=total, dtype=dtype, grads=grads, bits=bits, master=master,
                             ragged=ragged))


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # one generated token: which of its experts it goes to, a launch's worth of work
        _gate("gate token", 1, 64, 2, "bf16", train=False),
        # a request's tokens forward and backward, some experts closed to them, probabilities as weights, odd sizes
        _gate("gate ragged", 3001, 77, 3, "f32", normalise=False, masked=True),
        # a batch of sequences in training, many small experts
        _gate("gate batch", 65536, 256, 8, "bf16"),
        # rows by their two nearest of as many centroids as a quantiser has
        _gate("gate wide", 16384, 4096, 2, "f16", normalise=False, train=False),
        # what a model gives the tokens of a short text: the matrix of the classes is read once
        _loss("score text", 16, 65536, 2048, "bf16", train=False),
        # odd sizes in 32 bits with a bias, loss and all gradients
        _loss("loss ragged", 777, 10007, 333, "f32", bias=True),
        # a model learns the clusters of an assignment: few classes, many rows, centroids' half norms as bias
        _loss("loss clusters", 30000, 1024, 256, "f16", bias=True),
        # the loss of a training batch over a large vocabulary
        _loss("loss batch", 8192, 65536, 2048, "bf16"),
        # the weights of a small gate: latency
        _adamw("update few", 6, 40000, "f32", "f32", 32, False, True),
        # all weights of a small model at once, 16-bit weights beside their 32-bit masters
        _adamw("update model", 200, 50000000, "bf16", "bf16", 32, True, True),
        # the same with states in 8 bits, odd sizes at odd addresses, 32-bit gradients
        _adamw("update ragged 8 bits", 40, 5000000, "f16", "f32", 8, True, True),
        # matrices of sixteen experts with states in 8 bits
        _adamw("update experts 8 bits", 32, 134217728, "bf16", "bf16", 8, False, False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["gate", "loss", "adamw"])
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        if op == "gate":
            N, E, k = log(1, 65536), log(2, 8192), rng.choice([1, 2, 2, 3, 4, 6, 8, 16])
            if rng.random() < 0.5:  # powers of two, which people choose
                E = 1 << max(1, E.bit_length() - 1)
            if k <= E and N * E <= 1 << 26:
                return _gate(None, N, E, k, dtype, rng.random() < 0.5, rng.random() < 0.6, rng.random() < 0.3)
        elif op == "loss":
            N, V, D = log(1, 32768), log(2, 131072), log(16, 4096)
            if rng.random() < 0.5:
                D = max(32, D // 64 * 64)
            if N * V <= 1 << 29 and V * D <= 1 << 28 and N * V * D <= 1 << (38 if dtype == "f32" else 40):
                return _loss(None, N, V, D, dtype, rng.random() < 0.6, rng.random() < 0.5)
        else:
            tensors, total, bits = log(1, 200), log(100, 1 << 26), rng.choice([8, 32])
            grads = rng.choice([dtype, "f32"]) if dtype != "f32" else rng.choice(["f32", "bf16"])
            if total >= 4 * tensors:
                return _adamw(None, tensors, total, dtype, grads, bits, dtype != "f32" and rng.random() < 0.6,
                              rng.random() < 0.6)


# ---- what a program has in hand ------------------------------------------------------------


def _sizes(case):
    """Elements of every tensor: some a hundred times others, odd ones where the case is ragged."""
    n = case["tensors"]
    weights = [2.0 ** (i * 7 % 14 / 2) if case["ragged"] else 1.0 for i in range(n)]
    sizes = [max(1, int(case["total"] * w / sum(weights))) for w in weights]
    return [s | 1 for s in sizes] if case["ragged"] else sizes


HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
STEP, SEED = 7, 1234567


def _blocks(n):
    return -(-n // BLOCK)


def _prepare_adamw(case, g):
    sizes = _sizes(case)
    dtype = DTYPES[case["dtype"]]
    # the tensors of each kind are views of one buffer, as programs that save or exchange them hold them
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += n if case["ragged"] else -(-n // 64) * 64
    randn = lambda scale: torch.randn(at, generator=g, device=DEV).mul_(scale)  # noqa: E731
    views = lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
    s = dict(case=case, step=torch.tensor([STEP], dtype=torch.int64, device=DEV))
    weights = randn(0.02)
    flat = dict(params=weights.to(dtype))
    if case["master"]:
        flat["master"] = weights
    grads = randn(1e-3)
    grads *= torch.where(torch.rand(at, generator=g, device=DEV) < 0.01, 30.0, 1.0)
    s["grads"] = views(grads.to(DTYPES[case["grads"]]))
    if case["bits"] == 32:
        flat["m"], flat["v"] = randn(1e-3), randn(1e-3).square_()
    else:
        flat["m"] = torch.randint(0, 256, (at,), generator=g, device=DEV, dtype=torch.uint8)
        flat["v"] = torch.randint(128, 256, (at,), generator=g, device=DEV, dtype=torch.uint8)
        blocks = [_blocks(n) for n in sizes]
        ends = torch.tensor(blocks).cumsum(0).tolist()
        for name, low in (("m_scales", 96), ("v_scales", 86)):
            t = torch.randint(low, low + 5, (ends[-1],), generator=g, device=DEV, dtype=torch.uint8)
            t[:blocks[0]] = 0  # a tensor whose states are those of a start
            flat[name], s[name] = t, [t[e - b:e] for b, e in zip(blocks, ends)]
        flat["m"][:sizes[0]] = 0
        flat["v"][:sizes[0]] = 0
        s["values"] = [torch.zeros(at, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        s["values_of"] = [views(t) for t in s["values"]]
    s["flat"] = flat
    for name, t in flat.items():
        if name not in s:
            s[name] = views(t)
    if own:  # what a program makes once, from its weights and their states
        from paper_2408_01391_amd import binding as ftk

        s["state"] = ftk.AdamW(s["params"], case["bits"], m=s["m"], v=s["v"], m_scales=s.get("m_scales"),
                               v_scales=s.get("v_scales"), master=s.get("master"))
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, generator=g, device=DEV)  # noqa: E731
    if case["op"] == "adamw":
        return _prepare_adamw(case, g)
    dtype, N = DTYPES[case["dtype"]], case["N"]
    if case["op"] == "gate":
        E, k = case["E"], case["k"]
        z = randn(N, E) * 1.5 + randn(E)  # experts that are not equally liked
        if case["masked"]:
            z[rand(N, E) < 0.1] = -INF
            if N > 2:
                z[N // 2] = -INF       # a row that no expert takes
                z[N // 3, 1:] = -INF   # a row that one expert takes
        s = dict(case=case, logits=z.to(dtype))
        if case["train"]:
            s["dweights"] = randn(N, k).mul_(1e-2)
            s["dloss"] = torch.full((1,), 0.01, device=DEV)
        return s
    V, D = case["V"], case["D"]
    X, W = randn(N, D), randn(V, D).mul_(2 * D ** -0.5)
    labels = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    if N > 1:
        labels[rand(N) < 0.03] = -1  # padding: rows that are not to be looked at
        labels[N // 2] = -1
        X[labels < 0] = float("nan")
    s = dict(case=case, X=X.to(dtype), W=W.to(dtype), labels=labels, scale=1.0, bias=None)
    if case["bias"]:
        s["bias"] = W.square().sum(1).mul_(-0.5)
    if case["train"]:
        # the mean over rows, rows weighted; what is learned in fp16 is scaled up
        s["dloss"] = (0.5 + rand(N)) * ((4096.0 if case["dtype"] == "f16" else 1.0) / N)
    return s


# ---- the plain forms -----------------------------------------------------------------------


def _plain_gate(s):
    c = s["case"]
    E, k = c["E"], c["k"]
    z = s["logits"].float() + 0.0  # (one zero)
    top = z.amax(1, keepdim=True)
    row = top > -INF
    e = torch.where(row, (z - torch.where(row, top, 0)).exp(), 0)
    total = e.sum(1, keepdim=True)
    p = torch.where(row, e / total, 0)
    lse = torch.where(row, top + total.log(), -INF).squeeze(1)
    # keys that no two experts of a row share: the value's bits in order, then the lower index first
    bits = z.view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7fffffff)) * E + (E - 1 - torch.arange(E, device=DEV))
    labels = E - 1 - key.topk(k, dim=1).values.remainder(E)
    chosen = z.gather(1, labels)
    held = chosen > -INF
    weights = torch.where(held, p.gather(1, labels), 0)
    if c["normalise"]:
        weights = torch.where(held, weights / torch.where(row, weights.sum(1, keepdim=True), 1), 0)
    labels = torch.where(held, labels, -1).int()
    counts = torch.zeros(E + 1, dtype=torch.int64, device=DEV).index_add_(0, labels[held].long(), torch.ones_like(labels[held]).long())
    T = row.sum()
    counts[E] = T
    mean = p.sum(0, dtype=torch.float64) / T.clamp(min=1)
    share = counts[:E].double() * (E / (k * T.clamp(min=1).double()))
    loss = (share * mean).sum().float().view(1)
    out = [labels, weights, lse, counts.int(), mean.float(), loss]
    if c["train"]:
        d = s["dloss"] * share.float() / T.clamp(min=1)
        dz = p * (d - (p * d).sum(1, keepdim=True))
        wdw = torch.where(held, weights * s["dweights"], 0)
        inner = wdw.sum(1, keepdim=True)
        dz = dz.scatter_add_(1, labels.clamp(min=0).long(), wdw)
        if c["normalise"]:
            dz = dz.scatter_add_(1, labels.clamp(min=0).long(), torch.where(held, -weights * inner, 0))
        else:
            dz = dz - p * inner
        out.append(dz.to(s["logits"].dtype))
    return out


def _plain_loss(s):
    dtype, labels, V = s["X"].dtype, s["labels"].long(), s["case"]["V"]
    live = (labels >= 0) & (labels < V)
    X = torch.where(live.unsqueeze(1), s["X"], 0).float()
    W = s["W"].float()
    z = (X @ W.t()).mul_(s["scale"])
    if s["bias"] is not None:
        z += s["bias"]
    top = z.amax(1)
    lse = top + (z - top.unsqueeze(1)).exp_().sum(1).log()
    at = labels.clamp(0, V - 1).unsqueeze(1)
    loss = torch.where(live, lse - z.gather(1, at).squeeze(1), 0)
    out = [loss, torch.where(live, lse, 0)]
    if s["case"]["train"]:
        d = z.sub_(lse.unsqueeze(1)).exp_()
        d.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
        d *= torch.where(live, s["dloss"], 0).unsqueeze(1)
        if s["bias"] is not None:
            out.append(d.sum(0))
        d *= s["scale"]
        out += [(d @ W).to(dtype), (d.t() @ X).to(dtype)]
    return out


BLOCK = 32  # elements of 8-bit states under one scale
# the hash that rounds stochastically: 64-bit words of (seed, step), tensor and 2^32 elements, then 32 bits an element
GOLDEN, MIX1, MIX2, MIX3, MIX4 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 0xC8E1ED59, 0x876BA2B3


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _shifted(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)


def _mix64(z):
    z = (z ^ _shifted(z, 30)) * _signed(MIX1)
    z = (z ^ _shifted(z, 27)) * _signed(MIX2)
    return z ^ _shifted(z, 31)


def _random32(key, i):
    x = (i ^ key) & 0xffffffff
    x = ((x ^ (x >> 16)) * MIX3) & 0xffffffff
    x = ((x ^ (x >> 15)) * MIX4) & 0xffffffff
    return x ^ (x >> 16)


def _power(e):
    """2^e as a 32-bit number, e from -127 to 127."""
    return torch.where(e >= -126, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _decode(codes, scales, M):
    """Values of 8-bit codes [blocks, 32] of 4 exponent and M mantissa bits under 2^(scale - 127)."""
    c = codes.int() & ((16 << M) - 1)
    e = c >> M
    n = torch.where(e > 0, ((c & ((1 << M) - 1)) + (1 << M)) << (e - 1).clamp(min=0), c)
    n = torch.where(codes >= 128, -n, n) if M == 3 else n
    return torch.where(scales.unsqueeze(1) == 255, float("nan"), n * _power(scales.int().clamp(max=254) - 127).unsqueeze(1))


def _encode(x, M, random):
    """Codes and scales of values [blocks, 32]; `random`: 23 - M bits for each, which decide what is rounded up."""
    size = x.abs().view(torch.int32)
    top = (size.amax(1) + ((1 << (23 - M)) - 1)) >> 23
    scales = (top - (M + 14)).clamp(min=0)
    y = x.abs() * _power(127 - scales).unsqueeze(1)
    low = y < (1 << M)
    bits = torch.where(low, y + (1 << M), y).view(torch.int32)
    codes = ((bits + random) >> (23 - M)) - ((126 + M) << M) - torch.where(low, 1 << M, 0)
    codes = codes + 128 * (x.view(torch.int32) < 0) if M == 3 else torch.where(x > 0, codes.clamp(min=1), codes)
    return codes.to(torch.uint8), torch.where(top >= 255, 255, scales).to(torch.uint8)


def _plain_adamw(s):
    c, h = s["case"], HYPER
    sizes, eight, flat = [t.numel() for t in s["params"]], c["bits"] == 8, s["flat"]
    padded = [_blocks(n) * BLOCK for n in sizes] if eight else sizes
    # all tensors in one, each on whole blocks where states are held by blocks
    pad = torch.nn.functional.pad
    whole = lambda ts: torch.cat([pad(t, (0, p - n)) for t, n, p in zip(ts, sizes, padded)])  # noqa: E731
    back = lambda ts, x: torch._foreach_copy_(ts, [y[:n] for y, n in zip(x.split(padded), sizes)])  # noqa: E731
    t = s["step"].double()
    c1, c2 = (1 - h["beta1"] ** t).float(), (1 - h["beta2"] ** t).float()
    p, g = whole(s["master"] if c["master"] else s["params"]).float(), whole(s["grads"]).float()
    if eight:
        m = _decode(whole(s["m"]).view(-1, BLOCK), flat["m_scales"], 3).flatten()
        v = _decode(whole(s["v"]).view(-1, BLOCK), flat["v_scales"], 4).flatten()
    else:
        m, v = whole(s["m"]), whole(s["v"])
    b1, b2 = torch.tensor([[h["beta1"], 1 - h["beta1"]], [h["beta2"], 1 - h["beta2"]]], device=DEV).unbind(0)
    m = m * b1[0] + g * b1[1]
    v = v * b2[0] + (g * g) * b2[1]
    p = p - h["lr"] * (h["weight_decay"] * p + (m / c1) / ((v / c2).sqrt() + h["eps"]))
    back(s["params"], p)
    if c["master"]:
        back(s["master"], p)
    out = [flat["params"]] + ([flat["master"]] if c["master"] else [])
    if not eight:
        back(s["m"], m)
        back(s["v"], v)
        return out + [flat["m"], flat["v"]]
    lengths = torch.tensor(padded, device=DEV)
    index = torch.arange(p.numel(), device=DEV) - (lengths.cumsum(0) - lengths).repeat_interleave(lengths, output_size=p.numel())
    key = _mix64(_mix64(s["step"] * _signed(GOLDEN) + SEED) + torch.arange(len(sizes), device=DEV))
    r = _random32(_mix64(key).repeat_interleave(lengths, output_size=p.numel()), index).view(-1, BLOCK)
    for name, x, M, u in (("m", m, 3, (r >> 16) << 4), ("v", v, 4, (r & 0xffff) << 3)):
        codes, scales = _encode(x.view(-1, BLOCK), M, u.int())
        flat[name + "_scales"].copy_(scales)
        back(s[name], codes.flatten())
        back(s["values_of"][name == "v"], _decode(codes, scales, M).flatten())
    return out + s["values"]


# ---- the library's operators ---------------------------------------------------------------


def _library(s):
    from paper_2408_01391_amd import binding as ftk

    c = s["case"]
    if c["op"] == "gate":
        gate = ftk.route_gate(s["logits"], c["k"], normalise=c["normalise"])
        out = [gate.labels, gate.weights, gate.lse, gate.counts, gate.probs, gate.loss]
        if c["train"]:
            out.append(ftk.route_gate_grad(s["logits"], gate, s["dweights"], s["dloss"]))
        return out
    if c["op"] == "loss":
        loss, lse = ftk.xent(s["X"], s["W"], s["labels"], bias=s["bias"], scale=s["scale"])
        if not c["train"]:
            return [loss, lse]
        dX, dW, dbias = ftk.xent_grad(s["X"], s["W"], s["labels"], lse, s["dloss"], bias=s["bias"], scale=s["scale"])
        return [loss, lse] + ([dbias] if c["bias"] else []) + [dX, dW]
    ftk.adamw_step(s["state"], s["grads"], s["step"], seed=SEED, **HYPER)
    out = [s["flat"]["params"]] + ([s["flat"]["master"]] if c["master"] else [])
    if c["bits"] == 32:
        return out + [s["flat"]["m"], s["flat"]["v"]]
    ftk.adamw_moments(s["state"], out=s["values_of"])
    return out + s["values"]


def run(state):
    if own:
        return _library(state)
    return {"gate": _plain_gate, "loss": _plain_loss, "adamw": _plain_adamw}[state["case"]["op"]](state)


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["op"] == "gate":
        N, E, k = case["N"], case["E"], case["k"]
        forward = N * E * size + N * (8 * k + 4) + 8 * E
        return {"bytes": forward + (2 * N * E * size + N * (12 * k + 4) + 4 * E if case["train"] else 0),
                "flops": N * E * (10 if case["train"] else 4)}
    if case["op"] == "loss":
        N, V, D = case["N"], case["V"], case["D"]
        passes = 2 if case["train"] else 1  # each array is read, and its gradient written
        return {"bytes": passes * (N + V) * D * size + 12 * N + 4 * V * passes * case["bias"],
                "flops": 2 * N * V * D * (3 if case["train"] else 1)}
    n, eight = sum(_sizes(case)), case["bits"] == 8
    states = (4 + 4 / BLOCK + 4) if eight else 16  # the values of 8-bit states are asked for beside
    return {"bytes": n * (2 * size + DTYPES[case["grads"]].itemsize + 8 * case["master"] + states), "flops": 15 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------


def _exact_gate(s):
    c = s["case"]
    N, E, k = c["N"], c["E"], c["k"]
    z = s["logits"].double()
    order = torch.sort(z + 0.0, dim=1, descending=True, stable=True)
    held = order.values[:, :k] != -INF
    labels = torch.where(held, order.indices[:, :k], -1)
    lse = torch.logsumexp(z, 1)
    some = lse != -INF
    p = torch.where(some.unsqueeze(1), torch.softmax(z, 1), 0)
    base = order.values[:, :k]
    weights = torch.softmax(base, 1) if c["normalise"] else torch.exp(base - lse.unsqueeze(1))
    weights = torch.where(held, weights, 0)
    T = int(some.sum())
    counts = torch.bincount(labels[held], minlength=E)
    mean = p.sum(0) / max(T, 1)
    loss = E * (counts.double() / max(k * T, 1) * mean).sum()
    out = [labels.int(), weights, lse, torch.cat([counts, counts.new_tensor([T])]).int(), mean, loss.view(1)]
    if c["train"]:
        dw = s["dweights"].double()
        dp = (float(s["dloss"]) * E / max(k * T, 1) / max(T, 1) * counts.double()).expand(N, E).clone()
        if c["normalise"]:
            dchosen = weights * (dw - (weights * dw).sum(1, keepdim=True))
        else:
            dp.scatter_add_(1, labels.clamp(min=0), torch.where(held, dw, 0))
            dchosen = torch.zeros_like(dw)
        dz = p * (dp - (p * dp).sum(1, keepdim=True))
        dz.scatter_add_(1, labels.clamp(min=0), torch.where(held, dchosen, 0))
        out.append(dz)
    return out


def _exact_loss(s):
    labels, V, train = s["labels"].long(), s["case"]["V"], s["case"]["train"]
    N, D = s["X"].shape
    W = s["W"].double()
    bias = torch.zeros(V, dtype=torch.float64, device=DEV) if s["bias"] is None else s["bias"].double()
    loss, lse = torch.zeros(N, dtype=torch.float64, device=DEV), torch.zeros(N, dtype=torch.float64, device=DEV)
    dX, dW, dbias = torch.zeros(N, D, dtype=torch.float64, device=DEV), torch.zeros_like(W), torch.zeros_like(bias)
    rows = torch.nonzero((labels >= 0) & (labels < V)).flatten()
    for at in rows.split(2048):
        x, l = s["X"][at].double(), labels[at]
        z = torch.addmm(bias.unsqueeze(0), x, W.t(), alpha=s["scale"])
        lse[at] = torch.logsumexp(z, 1)
        loss[at] = torch.nn.functional.cross_entropy(z, l, reduction="none")
        if train:
            d = torch.softmax(z, 1)
            d[torch.arange(at.numel(), device=DEV), l] -= 1
            d *= s["dloss"][at].double().unsqueeze(1)
            dbias += d.sum(0)
            dX[at] = s["scale"] * (d @ W)
            dW += s["scale"] * (d.t() @ x)
    return [loss, lse] + (([dbias] if s["bias"] is not None else []) + [dX, dW] if train else [])


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales, M):
    """Values of one tensor's 8-bit states, in 64 bits: every code's number of units from a table."""
    units = [float(c) if c < 1 << M else math.ldexp((1 << M) + c % (1 << M), (c >> M) - 1) for c in range(16 << M)]
    units = torch.tensor(units + ([-u for u in units] if M == 3 else []), dtype=torch.float64, device=DEV)
    return units[codes.long()] * _exact_power(scales.long() - 127).repeat_interleave(BLOCK)[:codes.numel()]


def _exact_rounded(x, M, u):
    """The values that one tensor's states x (32-bit numbers held in 64) are rounded to: between two neighbours, the upper
    one where the distance from the lower one and the random part of a step u exceed a step."""
    n = x.numel()
    blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK).abs()
    near = 2.0 ** (M + 1) - 1 + 2.0 ** (M - 23)  # from here on a number's binade may be left by rounding up
    mantissa, exponent = torch.frexp(blocks.amax(1))
    unit = (exponent - 1 + (mantissa * 2 ** (M + 1) >= near) - M - 14).clamp(min=-127)
    unit = torch.where(mantissa == 0, -127, unit)
    y = (blocks * _exact_power(-unit).unsqueeze(1)).flatten()[:n]
    step = _exact_power((torch.frexp(y).exponent - 1 - M).clamp(min=0))
    fine = (y / step).where(y >= 1 << M, (y + (1 << M)).float().double() - (1 << M))  # (below the first binade 32 bits of y + 2^M)
    low = fine.floor()
    code = (low + ((fine - low) + u >= 1)) * step
    if M == 4:
        code = torch.where(x > 0, code.clamp(min=1), code)
    return code * _exact_power(unit).repeat_interleave(BLOCK)[:n] * torch.sign(x)


def _word(*parts):
    z = 0
    for part in parts:
        z = (z + part) & (1 << 64) - 1
        z = ((z ^ z >> 30) * MIX1) & (1 << 64) - 1
        z = ((z ^ z >> 27) * MIX2) & (1 << 64) - 1
        z ^= z >> 31
    return z


def _exact_adamw(s):
    c, h = s["case"], HYPER
    results = {k: torch.zeros_like(v, dtype=torch.float64) for k, v in s["flat"].items() if k in ("params", "master", "m", "v")}
    single = lambda x: x.float().double()  # noqa: E731
    for i, (param, grad) in enumerate(zip(s["params"], s["grads"])):
        p, g = (s["master"][i] if c["master"] else param).double(), grad.double()
        eight = c["bits"] == 8
        m, v = ((_exact_values(s[k][i], s[k + "_scales"][i], M) if eight else s[k][i].double()) for k, M in (("m", 3), ("v", 4)))
        b1, b1c, b2, b2c = (float(torch.tensor(b)) for b in (h["beta1"], 1 - h["beta1"], h["beta2"], 1 - h["beta2"]))
        # the definition rounds the states' products and sums to 32 bits, one by one
        m = single(single(b1 * m) + single(b1c * g))
        v = single(single(b2 * v) + single(b2c * single(g * g)))
        mh, vh = m / (1 - h["beta1"] ** STEP), v / (1 - h["beta2"] ** STEP)
        new = p - h["lr"] * (h["weight_decay"] * p + mh / (vh.sqrt() + h["eps"]))
        if eight:
            n = param.numel()
            word = _word(SEED + GOLDEN * STEP, i, 0) & 0xffffffff
            r = torch.arange(n, device=DEV) ^ word
            for shift, factor in ((16, MIX3), (15, MIX4), (16, 1)):
                r = ((r ^ (r >> shift)) * factor) % (1 << 32)
            m, v = _exact_rounded(m, 3, (r // 65536) / 65536.0), _exact_rounded(v, 4, (r % 65536) / 65536.0)
        at = param.storage_offset()
        for k, x in (("params", new), ("master", new), ("m", m), ("v", v)):
            if k in results:
                results[k][at:at + x.numel()] = x
    if not c["ragged"]:  # what lies between the tensors stays as it was
        used = torch.zeros(results["params"].shape, dtype=torch.bool, device=DEV)
        for param in s["params"]:
            used[param.storage_offset():param.storage_offset() + param.numel()] = True
        for k, x in results.items():
            x[~used] = 0 if c["bits"] == 8 and k in "mv" else s["flat"][k][~used].double()
    return list(results.values())


def exact(case, seed):
    s = prepare(case, seed)
    return {"gate": _exact_gate, "loss": _exact_loss, "adamw": _exact_adamw}[case["op"]](s)
