"""The operators of cluster experts - a model per cluster, fed by a soft assignment of every row to a few clusters - with
the sizes they are measured at and their plain forms.

Four operators: the assignment (a row's t best clusters of k scores, their softmax weights, the rows grouped by cluster, and
the gradient of the scores), the product of every group with its cluster's matrix (and the gradients of both factors), the
weighted sum that brings a row's t results together again (and its gradients), and the product with both factors held in 8
bits, a power of two as scale for every block of 128 along the contraction, with the conversion to and from that form.

With `own` false `run` computes them with elementary torch operations in 32 bits, rounded once at the end; with `own` true it
calls the library.  `exact` computes the same outputs in 64 bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 128          # values that share a scale in the 8-bit form
E4M3_MAX = 448.0     # largest value of the 8-bit type: 1.75 * 2^8


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one step of serving a handful of rows: all latency
        dict(name="route_8", kind="route", n=8, k=64, t=4, dtype="f32", mask="none", normalize=True, backward=False),
        # a training step's assignment with its gradient
        dict(name="route_train_32k", kind="route", n=32768, k=128, t=8, dtype="bf16", mask="none", normalize=True,
             backward=True),
        # every point of a large set over many clusters, pairs ruled out by a mask, weights that do not add up to one
        dict(name="route_masked_100k", kind="route", n=100_003, k=500, t=2, dtype="f32", mask="pairs", normalize=False,
             backward=True),
        # serving 16 rows: a few rows a cluster, the matrices of the clusters that were met are read
        dict(name="product_16", kind="product", n=16, t=4, groups=64, K=2048, N=1024, dtype="bf16", skew=0.5, train=False),
        # local linear models on the rows of a clustered point set, one cluster a row, odd sizes, single precision
        dict(name="product_points_100k", kind="product", n=100_003, t=1, groups=100, K=90, N=100, dtype="f32", skew=1.0,
             train=True),
        # a training step: product and both gradients
        dict(name="product_train_8k", kind="product", n=8192, t=2, groups=16, K=1024, N=2048, dtype="bf16", skew=0.5,
             train=True),
        # the largest: many rows, many wide clusters of uneven size
        dict(name="product_16k_4", kind="product", n=16384, t=4, groups=64, K=2048, N=2048, dtype="bf16", skew=0.5,
             train=False),
        # serving from 8-bit matrices: conversion of the rows and product
        dict(name="e4m3_24", kind="e4m3", n=24, t=2, groups=32, K=4096, N=2048, dtype="bf16", skew=0.5),
        # the largest, from 8-bit matrices
        dict(name="e4m3_16k_4", kind="e4m3", n=16384, t=4, groups=64, K=2048, N=2048, dtype="bf16", skew=0.5),
        # matrices of a length that ends inside a block, to 8 bits and back
        dict(name="blocks_25k_1000", kind="blocks", rows=25_003, K=1000, dtype="bf16"),
        # serving: the results of a few rows brought together
        dict(name="combine_16", kind="combine", n=16, t=4, d=2048, dtype="bf16", dropped=0.0, weights=True, backward=False),
        # training: the sum and its gradients, some rows without a cluster
        dict(name="combine_train_32k", kind="combine", n=32768, t=4, d=1024, dtype="bf16", dropped=0.02, weights=True,
             backward=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: any, or (as models mostly have it) a multiple of 64."""
    v = _log_int(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["route", "route", "product", "product", "product", "e4m3", "e4m3", "blocks", "combine", "combine"])
    if kind == "route":
        k = _log_int(rng, 2, 2000)
        n = min(_log_int(rng, 1, 100_000), 40_000_000 // k)
        return dict(kind=kind, n=n, k=k, t=rng.randint(1, min(8, k)), dtype=rng.choice(["f32", "bf16", "f16"]),
                    mask=rng.choice(["none", "clusters", "pairs"]), normalize=rng.random() < 0.5,
                    backward=rng.random() < 0.6)
    if kind == "blocks":
        K = _width(rng, 32, 4096)
        return dict(kind=kind, rows=max(1, min(_log_int(rng, 1, 100_000), 25_000_000 // K)), K=K,
                    dtype=rng.choice(["f32", "bf16", "f16"]))
    if kind == "combine":
        d = _width(rng, 16, 4096)
        t = rng.randint(1, 8)
        return dict(kind=kind, n=max(1, min(_log_int(rng, 1, 60_000), 100_000_000 // (d * t))), t=t, d=d,
                    dtype=rng.choice(["f32", "bf16", "f16"]), dropped=rng.choice([0.0, 0.1]), weights=rng.random() < 0.7,
                    backward=rng.random() < 0.6)
    groups = _log_int(rng, 2, 128)
    t = rng.randint(1, min(4, groups))
    K, N = _width(rng, 32, 2048), _width(rng, 32, 2048)
    while groups * K * N > 1 << 28:
        groups = max(t, groups // 2)
    skew = rng.choice([0.0, 0.5, 1.5])
    if kind == "e4m3":
        return dict(kind=kind, n=_log_int(rng, 1, 16384), t=t, groups=groups, K=K, N=N,
                    dtype=rng.choice(["f32", "bf16", "f16"]), skew=skew)
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    train = rng.random() < 0.5
    # the rate of 32-bit products is a sixteenth of that of 16-bit ones, a training step has three products
    most = 2.5e11 / (16 if dtype == "f32" else 1) / (3 if train else 1)
    return dict(kind=kind, n=max(1, min(_log_int(rng, 1, 32768), int(most / (t * K * N)))), t=t, groups=groups, K=K, N=N,
                dtype=dtype, skew=skew, train=train)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 4242)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _grouping(idx, k):
    """Slots (row * t + place in the row) sorted by cluster, stably: offsets (k + 1), order, place; -1 = no cluster."""
    flat = idx.reshape(-1).long()
    flat = torch.where(flat < 0, k, flat)
    at = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=k + 1)[:k]
    offsets = torch.zeros(k + 1, dtype=torch.int64, device=idx.device)
    offsets[1:] = torch.cumsum(counts, 0)
    pos = torch.arange(flat.numel(), device=idx.device)
    used = pos < offsets[k]
    place = torch.empty_like(pos)
    place[at] = torch.where(used, pos, -1)
    order = torch.where(used, at, -1)
    return offsets.int(), order.int(), place.reshape(idx.shape).int()


def _assigned(g, n, t, k, skew, dropped=0.0):
    """t different clusters for every row, clusters of uneven popularity; a share of the slots without one."""
    lean = skew * _normal(g, k)
    idx = torch.topk(lean + torch.empty(n, k, device=DEV).exponential_(generator=g).log_().neg_(), t, dim=1).indices.int()
    if dropped > 0.0:
        idx[torch.rand(n, t, generator=g, device=DEV) < dropped] = -1
    return idx


def _scaled(v, e):
    """v * 2^e, e a whole number from -254 to 254: two factors made from their bits, as a power function may be off in its
    last place."""
    half = e >> 1
    for h in (half, e - half):
        v = v * ((h + 127).int() << 23).view(torch.float32)
    return v


def _codes(x):
    """8-bit form of the rows of x: (values of the type, exponents), rows padded with zeros to whole blocks."""
    rows, K = x.shape
    pad = -K % BLOCK
    v = torch.nn.functional.pad(x.float(), (0, pad)).reshape(rows, -1, BLOCK)
    most = v.abs().amax(-1)
    m, e = torch.frexp(most)                                  # most = m * 2^e, m in [1/2, 1)
    e = torch.where(m <= 0.875, e - 9, e - 8)                 # smallest e with most <= 448 * 2^e
    e = torch.where(most > 0, e, torch.zeros_like(e)).clamp(min=-127)
    v = _scaled(v, -e[..., None])
    a = v.abs()
    step = _scaled(torch.ones_like(a), torch.frexp(a)[1].clamp(min=-5) - 4)   # 3 bits after the leading one
    return (torch.round(v / step) * step).reshape(rows, -1), e


def _values(q, e):
    """What the 8-bit form stands for."""
    rows, Kp = q.shape
    return _scaled(q.reshape(rows, -1, BLOCK), e[..., None]).reshape(rows, Kp)


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    st = dict(case)
    dt = TYPES[case["dtype"]]
    if kind == "route":
        n, k = case["n"], case["k"]
        # scores of a trained assignment: a few clusters stand out
        s = _normal(g, n, k) + 0.5 * _normal(g, k)
        if k >= 8:
            s += 4.0 * (torch.rand(n, k, generator=g, device=DEV) < 3.0 / k)
        st["allowed"] = None
        if case["mask"] == "clusters":
            st["allowed"] = torch.rand(k, generator=g, device=DEV) < 0.8
        elif case["mask"] == "pairs":
            allowed = torch.rand(n, k, generator=g, device=DEV) < 0.7
            allowed[torch.rand(n, generator=g, device=DEV) < 0.01] = False      # rows for which nothing is left
            junk = torch.rand(n, k, generator=g, device=DEV)                    # what masked places hold does not count
            s = torch.where(allowed, s, torch.where(junk < 0.3, float("nan"), torch.where(junk < 0.6, float("inf"), s)))
            s = torch.where(allowed & (junk > 0.95), float("-inf"), s)
            st["allowed"] = allowed
        st["scores"] = s.to(dt)
        st["dweight"] = _normal(g, n, case["t"])
        return st
    if kind == "blocks":
        x = _normal(g, case["rows"], case["K"]) * torch.exp(2.0 * _normal(g, case["rows"], 1))
        x[:, torch.rand(case["K"], generator=g, device=DEV) < 0.01] *= 30.0     # a few large coordinates
        x[torch.rand(case["rows"], generator=g, device=DEV) < 0.001] = 0.0
        st["x"] = x.to(dt)
        return st
    if kind == "combine":
        n, t, d = case["n"], case["t"], case["d"]
        idx = _assigned(g, n, t, max(t, 64), 0.5, case["dropped"])
        st["offsets"], st["order"], st["place"] = _grouping(idx, max(t, 64))
        st["z"] = _normal(g, n * t, d).to(dt)
        st["weight"] = torch.rand(n, t, generator=g, device=DEV) if case["weights"] else None
        st["dout"] = _normal(g, n, d).to(dt)
        return st
    n, t, G, K, N = case["n"], case["t"], case["groups"], case["K"], case["N"]
    st["idx"] = _assigned(g, n, t, G, case["skew"])
    st["offsets"], st["order"], _ = _grouping(st["idx"], G)
    st["bounds"] = st["offsets"].tolist()
    x = _normal(g, n, K)
    w = _normal(g, G, N, K) / math.sqrt(K)
    if kind == "e4m3":
        x[:, torch.rand(K, generator=g, device=DEV) < 0.01] *= 20.0
        st["x"] = x.to(dt)
        q, e = _codes(w.reshape(G * N, K))
        st["wq"] = q.to(torch.float8_e4m3fn).reshape(G, N, -1)
        st["wscale"] = (e + 127).to(torch.uint8).reshape(G, N, -1)
        return st
    st["x"], st["w"] = x.to(dt), w.to(dt)
    if case["train"]:
        st["dy"] = _normal(g, n * t, N).to(dt)
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _plain_route(st):
    n, k, t = st["n"], st["k"], st["t"]
    s = st["scores"].float()
    ok = s > float("-inf")                                    # not for NaN either
    if st["allowed"] is not None:
        ok = ok & st["allowed"]
    s = torch.where(ok, s + 0.0, float("-inf"))
    val, at = torch.sort(s, dim=1, descending=True, stable=True)
    val, at = val[:, :t], at[:, :t]
    chosen = val > float("-inf")
    top = torch.where(chosen[:, :1], val[:, :1], 0.0)
    e = torch.where(chosen, torch.exp(val - top), 0.0)
    total = e.sum(1, keepdim=True) if st["normalize"] else torch.exp(s - top).sum(1, keepdim=True)
    weight = torch.where(chosen, e / total, 0.0)
    idx = torch.where(chosen, at, -1).int()
    offsets, order, place = _grouping(idx, k)
    out = [idx, weight, offsets, order, place]
    if st["backward"]:
        dw = torch.where(chosen, st["dweight"], 0.0)
        c = (weight * dw).sum(1, keepdim=True)
        if st["normalize"]:
            ds = torch.zeros_like(s).scatter_add_(1, at, weight * (dw - c))
        else:
            p = torch.where(ok, torch.exp(s - top) / total, 0.0)
            ds = p * (torch.zeros_like(s).scatter_add_(1, at, dw) - c)
        out.append(ds.to(st["scores"].dtype))
    return out


def _plain_product(st):
    x, w, b, t, dt = st["x"], st["w"], st["bounds"], st["t"], st["x"].dtype
    src = torch.div(st["order"].long(), t, rounding_mode="floor")
    xg = x.float()[src]
    y = torch.zeros(xg.shape[0], st["N"], device=DEV)
    for g in range(st["groups"]):
        if b[g + 1] > b[g]:
            y[b[g]:b[g + 1]] = xg[b[g]:b[g + 1]] @ w[g].float().t()
    if not st["train"]:
        return y.to(dt)
    dy = st["dy"].float()
    dx = torch.zeros_like(xg)
    dw = torch.zeros_like(w)
    for g in range(st["groups"]):
        if b[g + 1] > b[g]:
            dyg = dy[b[g]:b[g + 1]]
            dx[b[g]:b[g + 1]] = dyg @ w[g].float()
            dw[g] = (dyg.t() @ xg[b[g]:b[g + 1]]).to(dt)
    return [y.to(dt), dx.to(dt), dw]


def _plain_e4m3(st):
    q, e = _codes(st["x"])
    x = _values(q, e)
    b = st["bounds"]
    src = torch.div(st["order"].long(), st["t"], rounding_mode="floor")
    y = torch.zeros(src.numel(), st["N"], device=DEV)
    for g in range(st["groups"]):
        if b[g + 1] > b[g]:
            w = _values(st["wq"][g].float(), st["wscale"][g].int() - 127)
            y[b[g]:b[g + 1]] = x[src[b[g]:b[g + 1]]] @ w.t()
    return y.to(st["x"].dtype)


def _plain_combine(st):
    place, weight, z = st["place"].long(), st["weight"], st["z"].float()
    dt = st["z"].dtype
    used = place >= 0
    w = torch.where(used, 1.0 if weight is None else weight, 0.0)
    rows = z[place.clamp(min=0)]
    out = [(w[..., None] * rows).sum(1).to(dt)]
    if st["backward"]:
        dout = st["dout"].float()
        dz = torch.zeros_like(z)
        dz[place[used]] = (w[..., None] * dout[:, None, :])[used]
        out.append(dz.to(dt))
        if weight is not None:
            out.append(torch.where(used, (rows * dout[:, None, :]).sum(-1), 0.0))
    return out


def _plain_blocks(st):
    q, e = _codes(st["x"])
    return [_values(q, e)[:, :st["K"]].contiguous(), e + 127]


# ---- the library's calls ----------------------------------------------------------------------------------------------
def _own_route(st):
    from paper_1802_04450_amd import binding as sc
    idx, weight, offsets, order, place = sc.sc_route(st["scores"], st["t"], allowed=st["allowed"],
                                                     normalize=st["normalize"])
    out = [idx, weight, offsets, order, place]
    if st["backward"]:
        out.append(sc.sc_route_backward(st["scores"], idx, weight, st["dweight"], allowed=st["allowed"],
                                        normalize=st["normalize"]))
    return out


def _own_product(st):
    from paper_1802_04450_amd import binding as sc
    y = sc.sc_grouped_product(st["x"], st["w"], st["offsets"], order=st["order"], slots=st["t"])
    if not st["train"]:
        return y
    dx = sc.sc_grouped_product(st["dy"], st["w"], st["offsets"], transpose=True)
    dw = sc.sc_grouped_gradient(st["dy"], st["x"], st["offsets"], order=st["order"], slots=st["t"])
    return [y, dx, dw]


def _own_e4m3(st):
    from paper_1802_04450_amd import binding as sc
    q, scale = sc.sc_quantize_blocks(st["x"])
    return sc.sc_grouped_product_e4m3(q, scale, st["wq"], st["wscale"], st["offsets"], order=st["order"], slots=st["t"],
                                      dtype=st["x"].dtype)


def _own_combine(st):
    from paper_1802_04450_amd import binding as sc
    out = [sc.sc_group_combine(st["z"], st["place"], st["weight"])]
    if st["backward"]:
        dz, dweight = sc.sc_group_combine_backward(st["dout"], st["z"], st["place"], st["weight"], st["order"])
        out.append(dz)
        if st["weight"] is not None:
            out.append(dweight)
    return out


def _own_blocks(st):
    from paper_1802_04450_amd import binding as sc
    q, scale = sc.sc_quantize_blocks(st["x"])
    return [sc.sc_dequantize_blocks(q, scale, st["K"]), scale.int()]


def run(state):
    """One pass through the case's operator, as a program calls it."""
    kind = state["kind"]
    forms = {"route": (_plain_route, _own_route), "product": (_plain_product, _own_product),
             "e4m3": (_plain_e4m3, _own_e4m3), "combine": (_plain_combine, _own_combine),
             "blocks": (_plain_blocks, _own_blocks)}
    return forms[kind][1 if own else 0](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind == "route":
        n, k, t = case["n"], case["k"], case["t"]
        b = n * k * size + {"none": 0, "clusters": k, "pairs": n * k}[case["mask"]] + 16 * n * t + 4 * (k + 1)
        if case["backward"]:
            b += n * t * 4 + n * k * size
        return {"bytes": b, "flops": n * k * (4 if case["backward"] else 2)}
    if kind == "blocks":
        scales = -(-case["K"] // BLOCK)
        # the values in, the values that the 8-bit form stands for and its exponents out
        return {"bytes": case["rows"] * (case["K"] * (size + 4) + 4 * scales), "flops": 3 * case["rows"] * case["K"]}
    if kind == "combine":
        n, t, d = case["n"], case["t"], case["d"]
        used = n * t * (1.0 - case["dropped"])
        per_slot = 4 + (4 if case["weights"] else 0)
        b = used * d * size + n * d * size + n * t * per_slot
        f = 2 * used * d
        if case["backward"]:
            b += n * d * size + n * t * d * size + n * t * 4
            f += 3 * used * d
        return {"bytes": int(b), "flops": int(f)}
    n, t, G, K, N = case["n"], case["t"], case["groups"], case["K"], case["N"]
    rows = n * t
    met = G * (1.0 - (1.0 - t / G) ** n) if t < G else G      # clusters that some row meets, were they all as popular
    wsize = 1.0 + 1.0 / BLOCK if kind == "e4m3" else size
    b = n * K * size + met * N * K * wsize + rows * N * size + 4 * rows + 4 * G
    f = 2 * rows * N * K
    if kind == "product" and case["train"]:
        b += rows * N * size + rows * K * size + G * N * K * size
        f *= 3
    return {"bytes": int(b), "flops": int(f)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def _exact_route(st):
    n, k, t = st["n"], st["k"], st["t"]
    s = st["scores"].double().cpu().numpy()
    ok = np.isfinite(s) | (s == np.inf)
    if st["allowed"] is not None:
        ok &= st["allowed"].cpu().numpy()
    left = np.where(ok, s, -np.inf)
    top = np.where(ok.any(1), left.max(1), 0.0)
    p = np.where(ok, np.exp(left - top[:, None]), 0.0)
    idx = np.full((n, t), -1, dtype=np.int32)
    row = np.arange(n)
    for j in range(t):
        a = left.argmax(1)                                    # the first of the largest
        good = left[row, a] > -np.inf
        idx[good, j] = a[good]
        left[row, a] = -np.inf
    chosen = idx >= 0
    part = np.where(chosen, np.take_along_axis(p, np.maximum(idx, 0), 1), 0.0)
    total = (part if st["normalize"] else p).sum(1)
    total[total == 0.0] = 1.0
    weight = part / total[:, None]
    groups = [np.flatnonzero(idx.reshape(-1) == g) for g in range(k)] if n * t * k < 1e8 else None
    if groups is None:
        flat = idx.reshape(-1)
        at = np.lexsort((np.arange(flat.size), np.where(flat < 0, k, flat)))
        slots = at[:int(chosen.sum())]
        counts = np.bincount(flat[flat >= 0], minlength=k)
    else:
        slots = np.concatenate(groups)
        counts = np.array([len(a) for a in groups])
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    order = np.full(n * t, -1, dtype=np.int32)
    order[:slots.size] = slots
    place = np.full(n * t, -1, dtype=np.int32)
    place[slots] = np.arange(slots.size, dtype=np.int32)
    out = [idx, weight, offsets, order, place.reshape(n, t)]
    if st["backward"]:
        dw = np.where(chosen, st["dweight"].double().cpu().numpy(), 0.0)
        c = (weight * dw).sum(1)
        given = np.zeros((n, k))
        for j in range(t):
            given[row, np.maximum(idx[:, j], 0)] += dw[:, j]
        share = p / total[:, None]
        if st["normalize"]:
            kept = np.zeros((n, k), dtype=bool)
            for j in range(t):
                kept[row[chosen[:, j]], idx[chosen[:, j], j]] = True
            share = np.where(kept, share, 0.0)
        out.append(share * (given - c[:, None]))
    return [torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in out]


def _members(st):
    """For every cluster its slots, found one cluster at a time."""
    flat = st["idx"].reshape(-1)
    return [torch.nonzero(flat == g).reshape(-1) for g in range(st["groups"])]


def _exact_product(st):
    x, w = st["x"].double(), st["w"]
    parts, dxs, dws, done = [], [], [], 0
    for g, slots in enumerate(_members(st)):
        xg, wg = x[slots // st["t"]], w[g].double()
        parts.append(torch.mm(xg, wg.t().contiguous()))
        if st["train"]:
            dyg = st["dy"][done:done + slots.numel()].double()
            done += slots.numel()
            dxs.append(torch.mm(dyg, wg))
            dws.append(torch.mm(dyg.t().contiguous(), xg))
    y = torch.cat(parts)
    return [y, torch.cat(dxs), torch.stack(dws)] if st["train"] else y


def _table():
    """The values of the 8-bit type that are not negative, by code: 4 bits of exponent (bias 7), 3 of fraction."""
    c = torch.arange(127, dtype=torch.int64)
    e, f = c >> 3, (c & 7).double()
    return torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (e.double() - 7))


def _power(e):
    """2^e, e a whole number in 64 bits from -160 to 160."""
    tab = torch.tensor([2.0 ** i for i in range(-160, 161)], dtype=torch.float64, device=e.device)
    return tab[e.long() + 160]


def _exact_codes(x):
    rows, K = x.shape
    v = torch.zeros(rows, K + -K % BLOCK, dtype=torch.float64, device=x.device)
    v[:, :K] = x.double()
    v = v.reshape(rows, -1, BLOCK)
    most = v.abs().amax(-1)
    e = torch.ceil(torch.log2(torch.where(most > 0, most, E4M3_MAX) / E4M3_MAX))
    e = torch.where(most > E4M3_MAX * _power(e), e + 1, e)     # the logarithm's rounding
    e = torch.where(most <= E4M3_MAX * _power(e - 1), e - 1, e)
    e = torch.where(most > 0, e, 0.0).clamp(min=-127)
    v = v * _power(-e)[..., None]
    tab = _table().to(x.device)
    mid = (tab[1:] + tab[:-1]) / 2
    a = v.abs()
    lo = torch.searchsorted(mid, a)                           # codes whose upper midpoint lies below
    tie = a == mid[lo.clamp(max=125)]
    code = torch.where(tie & (lo % 2 == 1), lo + 1, lo)
    return (torch.sign(v) * tab[code] * _power(e)[..., None]).reshape(rows, -1), e


def _exact_e4m3(st):
    x, _ = _exact_codes(st["x"])
    parts = []
    for g, slots in enumerate(_members(st)):
        wg = st["wq"][g].double().reshape(st["N"], -1, BLOCK) \
            * _power(st["wscale"][g].double() - 127)[..., None]
        parts.append(torch.mm(x[slots // st["t"]], wg.reshape(st["N"], -1).t().contiguous()))
    return torch.cat(parts)


def _exact_combine(st):
    n, t, d = st["n"], st["t"], st["d"]
    out = torch.zeros(n, d, dtype=torch.float64, device=DEV)
    dz = torch.zeros(n * t, d, dtype=torch.float64, device=DEV)
    dw = torch.zeros(n, t, dtype=torch.float64, device=DEV)
    for j in range(t):
        row = torch.nonzero(st["place"][:, j] >= 0).reshape(-1)
        at = st["place"][row, j].long()
        z = st["z"][at].double()
        w = torch.ones(row.numel(), 1, dtype=torch.float64, device=DEV) if st["weight"] is None \
            else st["weight"][row, j].double()[:, None]
        out[row] += w * z
        dz[at] = w * st["dout"][row].double()
        dw[row, j] = (z * st["dout"][row].double()).sum(1)
    if not st["backward"]:
        return [out]
    return [out, dz] + ([dw] if st["weight"] is not None else [])


def _exact_blocks(st):
    v, e = _exact_codes(st["x"])
    return [v[:, :st["K"]].contiguous(), (e + 127).int()]


def exact(case, seed):
    st = prepare(case, seed)
    forms = {"route": _exact_route, "product": _exact_product, "e4m3": _exact_e4m3, "combine": _exact_combine,
             "blocks": _exact_blocks}
    return forms[case["kind"]](st)
