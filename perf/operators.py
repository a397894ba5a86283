"""Rows routed by label to experts held in 4 bits, as timed cases: sorting rows by expert, bringing them
back with weights, the gradients of both, microscaled 4-bit floating point (blocks of 32 elements E2M1 under
a shared power of two) and the experts' products in it.

`own` chooses between the plain form of every operator (elementary torch operations in 32 bits) and the
library's entry points; both take the same state."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK, PAD = 32, 128  # elements under one scale; packed rows are whole multiples of PAD elements


def _route(name, op, N, D, k, E, dtype, align=1):
    return _named(name, dict(op=op, N=N, D=D, k=k, E=E, dtype=dtype, align=align))


def _quant(name, N, D, dtype, transpose):
    return _named(name, dict(op="quantise", N=N, D=D, dtype=dtype, transpose=transpose))


def _product(name, op, N, D, F, k, E, dtype):
    return _named(name, dict(op=op, N=N, D=D, F=F, k=k, E=E, dtype=dtype, align=128 if op == "expert_grad" else 1))


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # one step of generation for a few streams: sorting 32 tokens must cost a launch, not a sort
        _route("dispatch few", "dispatch", 32, 1024, 2, 16, "bf16"),
        # feature vectors regrouped by their nearest of many clusters, to be searched list by list
        _route("dispatch vectors", "dispatch", 60000, 1024, 1, 1024, "f32"),
        # results of a small request brought back, rows that no vector load divides
        _route("combine ragged", "combine", 777, 333, 3, 13, "f16"),
        # the same for a batch of sequences, every expert on whole tiles of 128 rows as training has them
        _route("combine batch", "combine", 65536, 1024, 2, 64, "bf16", 128),
        # backward passes: odd rows in 32 bits, and the batch
        _route("gradients ragged", "gradients", 30007, 333, 3, 77, "f32"),
        _route("gradients batch", "gradients", 65536, 1024, 2, 64, "bf16", 128),
        # packing activations (or a checkpoint's matrices) along their rows
        _quant("quantise rows", 65536, 2048, "bf16", False),
        # packing across the rows, as a weight gradient needs its operands; odd sizes in 32 bits
        _quant("quantise across", 30007, 333, "f32", True),
        # one generated token through its two experts: the weights' bytes are all there is to it
        _product("product token", "product", 1, 4096, 4096, 2, 8, "bf16"),
        # a request of some hundred tokens, no size a tile's multiple, 32-bit rows in and out
        _product("product ragged", "product", 777, 1000, 1333, 2, 13, "f32"),
        # the forward pass of a training or prefill batch
        _product("product batch", "product", 16384, 4096, 4096, 2, 16, "bf16"),
        # its backward pass: gradients of the experts' rows and of their weights (rows packed across and along)
        _product("gradients of experts", "expert_grad", 16384, 2048, 4096, 2, 8, "bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["dispatch", "dispatch", "combine", "combine", "gradients", "gradients", "quantise", "quantise",
                         "product", "product", "product", "expert_grad"])
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        N, D, F, k, E = log(1, 65536), log(16, 4096), log(16, 4096), rng.choice([1, 2, 2, 3, 4, 8]), log(2, 1024)
        if rng.random() < 0.5:  # widths that people choose, beside those that data happen to have
            D, F = max(32, D // 64 * 64), max(32, F // 64 * 64)
        if D == 3072 or F == 3072:
            continue
        if op == "quantise":
            if N * D <= 1 << 27:
                return _quant(None, N, D, dtype, rng.random() < 0.4)
            continue
        if op in ("product", "expert_grad"):
            E = min(E, 64)
        if k > E:
            continue
        if op in ("product", "expert_grad"):
            # (the plain form pads every expert to the fullest one, and holds all matrices in 32 bits)
            if (E * F * D <= 1 << 28 and N * k * D * F <= 1 << 38 and N * k * max(D, F) <= 1 << 27
                    and N * E * max(D, F) <= 1 << 31):
                return _product(None, op, N, D, F, k, E, dtype)
        elif N * k * D <= 1 << 27:
            return _route(None, op, N, D, k, E, dtype, rng.choice([1, 1, 16, 128]))


def _rows(case):
    """Rows that sorting may need: every expert that has any is filled up to a multiple of `align`."""
    slots, align = case["N"] * case["k"], case["align"]
    return (slots + min(case["E"], slots) * (align - 1)) // align * align


def _labels(case, g):
    """Experts of every token by a gate whose experts are not equally liked, the best k, a few slots dropped
    (-1); and the gate's weights."""
    N, k, E = case["N"], case["k"], case["E"]
    gate = torch.randn(N, E, generator=g, device=DEV) + torch.randn(E, generator=g, device=DEV)
    best, labels = gate.topk(k, dim=1)
    labels = labels.to(torch.int32)
    if N > 1:
        labels[torch.rand(N, k, generator=g, device=DEV) < 0.02] = -1
        labels[N // 2] = -1  # a token that nobody takes
    return labels.contiguous(), best.softmax(1).contiguous()


def _values(g, rows, cols, dtype):
    """Activations: normal values, a few features much larger than the others, a row of zeros."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    x *= torch.where(torch.rand(cols, generator=g, device=DEV) < 0.01, 20.0, 1.0)
    if rows > 2:
        x[rows // 3] = 0
    return x.to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    op, N, D, dtype = case["op"], case["N"], case["D"], case["dtype"]
    s = dict(case=case)
    if op == "quantise":
        s["X"] = _values(g, N, D, dtype)
        return s
    labels, weights = _labels(case, g)
    R = s["R"] = _rows(case)
    if op == "dispatch":
        return dict(s, X=_values(g, N, D, dtype), labels=labels)
    offsets, counts, order, pos = _plan(labels, case["E"], case["align"], R)
    s.update(weights=weights, offsets=offsets, counts=counts, order=order, pos=pos)
    if op in ("combine", "gradients"):
        s["Y"] = _values(g, R, D, dtype)
        if op == "gradients":
            s["dOut"] = _values(g, N, D, dtype)
            s["dRows"] = _values(g, R, D, dtype)
        return s
    F, E = case["F"], case["E"]
    s["most"] = int(counts.max())  # rows of the fullest expert, for the plain form's padding
    W = torch.randn(E * F, D, generator=g, device=DEV).mul_(D ** -0.5)
    if op == "product":
        s["X"] = _values(g, N, D, dtype)
        s["W"] = _pack(*_quantise(W))
        return s
    # rows as sorting leaves them: those that hold no token are zero
    held = (order >= 0).unsqueeze(1)
    s["X"] = torch.where(held, _values(g, R, D, dtype), 0).contiguous()
    s["dY"] = torch.where(held, _values(g, R, F, dtype) * 2.0 ** -10, 0).contiguous()
    s["W"] = _pack(*_quantise(W.view(E, F, D).transpose(1, 2).reshape(E * D, F)))
    return s


# ---- the plain forms ----------------------------------------------------------------------


def _plan(labels, E, align, R):
    """offsets [E+1], counts [E], slot of every sorted row (-1: none), sorted row of every slot (-1: dropped)."""
    flat = labels.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    counts = (torch.zeros(E + 1, dtype=torch.int64, device=DEV).index_add_(0, key, torch.ones_like(key)))[:E]
    ends = torch.cumsum((counts + align - 1) // align * align, 0)
    offsets = torch.cat([torch.zeros_like(ends[:1]), ends])
    by_key, slot = torch.sort(key, stable=True)
    first = torch.cumsum(counts, 0) - counts
    routed = by_key < E
    safe = by_key.clamp(max=E - 1)
    place = torch.where(routed, offsets[safe] + torch.arange(key.numel(), device=DEV) - first[safe], R)
    order = torch.full((R + 1,), -1, dtype=torch.int64, device=DEV).index_put_((place,), torch.where(routed, slot, -1))[:R]
    pos = torch.empty_like(key).index_put_((slot,), torch.where(routed, place, -1))
    return offsets.int(), counts.int(), order.int(), pos.int().view(labels.shape)


def _gather(X, order, k):
    return torch.where((order >= 0).unsqueeze(1), X[order.clamp(min=0).long() // k], 0)


def _combine(Y, pos, weights=None):
    held = (pos >= 0).unsqueeze(2)
    rows = torch.where(held, Y[pos.clamp(min=0).long()].float(), 0)
    if weights is not None:
        rows = torch.where(held, rows * weights.unsqueeze(2), 0)
    return rows.sum(1).to(Y.dtype)


def _combine_grad(dOut, Y, order, pos, weights):
    k = pos.shape[1]
    token = order.clamp(min=0).long()
    dY = torch.where((order >= 0).unsqueeze(1), dOut[token // k].float() * weights.reshape(-1)[token].unsqueeze(1), 0)
    dots = (dOut.float().unsqueeze(1) * Y[pos.clamp(min=0).long()].float()).sum(2)
    return dY.to(dOut.dtype), torch.where(pos >= 0, dots, 0)


def _table():
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)


def _quantise(X):
    """Indices of the magnitudes, signs and exponents of the shared scales: [rows, blocks, 32], same, [rows, blocks]."""
    x = torch.nn.functional.pad(X.float(), (0, -X.shape[1] % PAD)).view(X.shape[0], -1, BLOCK)
    top = x.abs().amax(2)
    exponent = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(min=-127)
    m = torch.ldexp(x, -exponent.unsqueeze(2)).abs()
    index = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5))
    return index, torch.signbit(x), exponent


def _pack(index, sign, exponent):
    """Two elements a byte, the first in the low half; scales as exponent + 127."""
    code = (index + 8 * sign.to(torch.uint8)).view(index.shape[0], -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).contiguous(), (exponent + 127).to(torch.uint8).contiguous()


def _values_of(index, sign, exponent):
    v = _table()[index.long()]
    return torch.ldexp(torch.where(sign, -v, v), exponent.unsqueeze(2)).flatten(1)


def _unpack(codes, scales, D):
    code = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1, BLOCK)
    return _values_of(code & 7, code > 7, scales.int() - 127)[:, :D]


def _rounded(X):
    return _values_of(*_quantise(X))[:, : X.shape[1]]


def _by_expert(rows, s):
    """Sorted rows [R, .] as [E, most, .], filled up with zeros, and the place of every sorted row in it."""
    offsets, counts, E, most = s["offsets"].long(), s["counts"].long(), s["case"]["E"], s["most"]
    at = torch.arange(most, device=DEV)
    inside = at < counts.unsqueeze(1)
    source = torch.where(inside, offsets[:-1].unsqueeze(1) + at, 0)
    p = torch.arange(rows.shape[0], device=DEV)
    expert = (torch.searchsorted(offsets, p, right=True) - 1).clamp(max=E - 1)
    return torch.where(inside.unsqueeze(2), rows[source], 0), expert * most + (p - offsets[expert]).clamp(max=most - 1)


def _grouped(A, W, s):
    """Sorted rows A [R, D] by their experts' matrices W [E, F, D]; rows without a token are zero."""
    padded, place = _by_expert(A, s)
    out = torch.bmm(padded, W.transpose(1, 2)).flatten(0, 1)
    return torch.where((s["order"] >= 0).unsqueeze(1), out[place], 0)


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "dispatch":
        plan = _plan(s["labels"], c["E"], c["align"], s["R"])
        return (_gather(s["X"], plan[2], c["k"]), *plan)
    if op == "combine":
        return _combine(s["Y"], s["pos"], s["weights"])
    if op == "gradients":
        return (*_combine_grad(s["dOut"], s["Y"], s["order"], s["pos"], s["weights"]), _combine(s["dRows"], s["pos"]))
    dt = DTYPES[c["dtype"]]
    if op == "quantise":
        return _rounded(s["X"].t() if c["transpose"] else s["X"]).to(dt)
    E, D, F = c["E"], c["D"], c["F"]
    if op == "product":
        W = _unpack(*s["W"], D).view(E, F, D)
        return _grouped(_gather(_rounded(s["X"]), s["order"], c["k"]), W, s).to(dt)
    W = _unpack(*s["W"], F).view(E, D, F)
    dX = _grouped(_rounded(s["dY"]), W, s)
    # the sum over an expert's rows: 32 rows share a scale, and every expert starts at a multiple of 128
    left, right = _by_expert(_rounded(s["dY"].t()).t(), s)[0], _by_expert(_rounded(s["X"].t()).t(), s)[0]
    return dX.to(dt), torch.bmm(left.transpose(1, 2), right).to(dt)


# ---- the library's operators --------------------------------------------------------------


def _library(s):
    from paper_2408_01391_amd import binding as ftk

    c = s["case"]
    op = c["op"]
    if op == "dispatch":
        rows, r = ftk.route_dispatch(s["X"], s["labels"], c["E"], align=c["align"])
        return rows, r.offsets, r.counts, r.order, r.pos
    if op == "quantise":
        return ftk.mx4_dequantize(ftk.mx4_quantize(s["X"], transpose=c["transpose"]), s["X"].dtype)
    r = ftk.Route(s["offsets"], s["counts"], s["order"], s["pos"], c["align"])
    if op == "combine":
        return ftk.route_combine(s["Y"], r, s["weights"])
    if op == "gradients":
        return (*ftk.route_combine_grad(s["dOut"], s["Y"], r, s["weights"]), ftk.route_combine(s["dRows"], r))
    if op == "product":
        return ftk.mx4_linear(s["X"], ftk.Mx4(*s["W"], c["D"]), route=r, gather=True)
    dX = ftk.mx4_linear(s["dY"], ftk.Mx4(*s["W"], c["F"]), route=r)
    dW = ftk.mx4_outer(ftk.mx4_quantize(s["dY"], transpose=True), ftk.mx4_quantize(s["X"], transpose=True), r,
                       out_dtype=s["X"].dtype)
    return dX, dW


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    op, N, D = case["op"], case["N"], case["D"]
    size = DTYPES[case["dtype"]].itemsize
    packed = lambda rows, cols: rows * (-(-cols // PAD) * PAD) * 17 // 32  # noqa: E731
    if op == "quantise":
        rows, cols = (D, N) if case["transpose"] else (N, D)
        return {"bytes": 2 * N * D * size + 2 * packed(rows, cols), "flops": 2 * N * D}
    k, E, R = case["k"], case["E"], _rows(case)
    slots = N * k
    if op == "dispatch":
        return {"bytes": (N + R) * D * size + 8 * slots + 4 * R + 8 * E, "flops": 0}
    if op == "combine":
        return {"bytes": (N + slots) * D * size + 8 * slots, "flops": 2 * slots * D}
    if op == "gradients":
        return {"bytes": (2 * N + 2 * slots + R) * D * size + 12 * slots + 4 * R, "flops": 4 * slots * D}
    F, used = case["F"], min(E, slots)
    if op == "product":
        return {"bytes": N * D * size + packed(used * F, D) + R * F * size + 8 * slots, "flops": 2 * slots * D * F}
    return {"bytes": R * (2 * D + F) * size + packed(used * D, F) + E * F * D * size + 4 * R, "flops": 4 * slots * D * F}


# ---- the definitions in 64 bits -----------------------------------------------------------


def _exact_plan(labels, E, align, R):
    flat = labels.reshape(-1).cpu().numpy().astype(np.int64)
    slots = np.flatnonzero((flat >= 0) & (flat < E))
    by = slots[np.lexsort((slots, flat[slots]))]
    counts = np.bincount(flat[slots], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(-(-counts // align) * align)])
    order, pos = np.full(R, -1, np.int64), np.full(flat.size, -1, np.int64)
    pos[by] = offsets[flat[by]] + np.arange(by.size) - (np.cumsum(counts) - counts)[flat[by]]
    order[pos[by]] = by
    return tuple(torch.from_numpy(a.astype(np.int32)).to(DEV) for a in (offsets, counts, order, pos.reshape(labels.shape)))


def _exact_rounded(X):
    """Every block of 32 along the rows as the nearest multiples of its steps, ties to the even multiple."""
    rows, cols = X.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=DEV)
    lines = max(1, (1 << 25) // max(cols, 1))
    for r in range(0, rows, lines):
        x = X[r:r + lines].double()
        x = torch.cat([x, x.new_zeros(x.shape[0], -cols % BLOCK)], 1).unflatten(1, (-1, BLOCK))
        top = x.abs().amax(2, keepdim=True)
        scale = torch.exp2((torch.floor(torch.log2(top)) - 2).clamp(min=-127))
        y = x / scale
        step = torch.exp2(torch.floor(torch.log2(y.abs())).clamp(min=0) - 1)
        y = (torch.round(y / step) * step).clamp(-6, 6) * scale
        out[r:r + lines] = torch.where(top > 0, y, 0).flatten(1)[:, :cols]
    return out


def _exact_matrix(W, e, rows, cols):
    """Rows of one expert's packed matrix."""
    codes, scales = (t[e * rows:(e + 1) * rows].long() for t in W)
    code = torch.stack((codes % 16, codes // 16), 2).flatten(1)
    index = code % 8
    v = torch.where(index < 2, index * 0.5, (2.0 + index % 2).double() * torch.exp2((index // 2 - 2).double()))
    v = torch.where(code >= 8, -v.double(), v.double()) * torch.exp2((scales - 127).double()).repeat_interleave(BLOCK, 1)
    return v[:, :cols]


def _exact_back(rows, pos, weights=None):
    out = torch.zeros(pos.shape[0], rows.shape[1], dtype=torch.float64, device=DEV)
    for j in range(pos.shape[1]):
        t = torch.nonzero(pos[:, j] >= 0).flatten()
        part = rows[pos[t, j].long()].double()
        out[t] += part if weights is None else part * weights[t, j].double().unsqueeze(1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantise":
        return _exact_rounded(s["X"].t() if case["transpose"] else s["X"])
    k, E, D = case["k"], case["E"], case["D"]
    if op == "dispatch":
        plan = _exact_plan(s["labels"], E, case["align"], s["R"])
        rows = torch.zeros(s["R"], D, dtype=torch.float64, device=DEV)
        held = torch.nonzero(plan[2] >= 0).flatten()
        rows[held] = s["X"][plan[2][held].long() // k].double()
        return (rows, *plan)
    order, pos, weights = s["order"], s["pos"], s["weights"]
    held = torch.nonzero(order >= 0).flatten()
    slot = order[held].long()
    if op == "combine":
        return _exact_back(s["Y"], pos, weights)
    if op == "gradients":
        dY = torch.zeros(s["R"], D, dtype=torch.float64, device=DEV)
        dY[held] = s["dOut"][slot // k].double() * weights.flatten()[slot].double().unsqueeze(1)
        dw = torch.zeros(case["N"] * k, dtype=torch.float64, device=DEV)
        dw[slot] = (s["dOut"][slot // k].double() * s["Y"][held].double()).sum(1)
        return dY, dw.view(-1, k), _exact_back(s["dRows"], pos)
    F = case["F"]
    offsets, counts = s["offsets"].tolist(), s["counts"].tolist()
    if op == "product":
        A = _exact_rounded(s["X"])
        out = torch.zeros(s["R"], F, dtype=torch.float64, device=DEV)
        for e, (o, c) in enumerate(zip(offsets, counts)):
            if c:
                out[o:o + c] = A[order[o:o + c].long() // k] @ _exact_matrix(s["W"], e, F, D).t().contiguous()
        return out
    A, left, right = _exact_rounded(s["dY"]), _exact_rounded(s["dY"].t()), _exact_rounded(s["X"].t())
    dX = torch.zeros(s["R"], D, dtype=torch.float64, device=DEV)
    dW = torch.zeros(E, F, D, dtype=torch.float64, device=DEV)
    for e, (o, c) in enumerate(zip(offsets, counts)):
        if c:
            dX[o:o + c] = A[o:o + c] @ _exact_matrix(s["W"], e, D, F).t().contiguous()
            dW[e] = left[:, o:o + c] @ right[:, o:o + c].t().contiguous()
    return dX, dW
