"""What is timed of the operators around a mixture whose samples are routed to its components.

  route     per sample the most probable components, their weights and the mixture's log-density; with `train` the
            gradients of the scores and of the log coefficients too (the E-step of a mixture)
  exchange  slots (sample, choice) sorted by component, rows carried to their components and, weighted, back; with
            `train` the gradients of the rows on both sides and of the weights too
  choose    one entry per row of logits under temperature, top-k, top-p and min-p, from given uniforms

`run` makes the framework's calls where `own` is true and computes the same with elementary operations elsewhere.
`exact` computes it in 64 bits with NumPy.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _route(name, N, M, top, dtype="float32", by="component", coef=True, renormalise=False, train=False, masked=False):
    return dict(name=name, op="route", N=N, M=M, top=top, dtype=dtype, by=by, coef=coef, renormalise=renormalise,
                train=train, masked=masked)


def _exchange(name, N, M, top, H, dtype="float32", train=False, dropped=False, padded=False):
    return dict(name=name, op="exchange", N=N, M=M, top=top, H=H, dtype=dtype, train=train, dropped=dropped, padded=padded)


def _choose(name, B, V, dtype="float32", filters="none", per_row=False, masked=False):
    return dict(name=name, op="choose", B=B, V=V, dtype=dtype, filters=filters, per_row=per_row, masked=masked)


def listed():
    return [
        # one sample of a small mixture, as a service answers it: latency only
        _route("route_one", 1, 8, 2),
        # the E-step of the coefficients of a mixture of 100 circuits on a mini-batch of 500, some components closed
        _route("route_mixture", 500, 100, 1, train=True, masked=True),
        # a router's logits, a row per token, in a training step: eight of 128, weights summing to one
        _route("route_rows", 16001, 128, 8, "bfloat16", "sample", False, True, True),
        # assigning a whole training set to its clusters
        _route("route_dataset", 262144, 64, 2),
        # a handful of grey images to their components and back
        _exchange("exchange_few", 3, 8, 2, 784),
        # 64x64 colour images, each to the one component it was assigned to, and the answers back
        _exchange("exchange_images", 1000, 100, 1, 12288),
        # a prompt's rows to two of eight experts, slots over capacity dropped, rows inside a wider buffer
        _exchange("exchange_ragged", 4097, 8, 2, 4096, "bfloat16", dropped=True, padded=True),
        # a training step of a layer with 64 experts, four per row, with all gradients
        _exchange("exchange_train", 8192, 64, 4, 2048, "bfloat16", train=True),
        # a component for each of a batch of samples, from the mixture's posterior
        _choose("choose_component", 500, 100),
        # a grey value for every pixel of 64 images of 28x28, tails cut off
        _choose("choose_values", 50176, 256, filters="top_p"),
        # the next entry of a single sequence over a long vocabulary: latency
        _choose("choose_one", 1, 100003, "bfloat16", "all"),
        # the same for a batch, every row with settings of its own, entries masked out
        _choose("choose_batch", 64, 131077, filters="all", per_row=True, masked=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    while True:
        op = rng.choice(["route", "exchange", "choose"])
        dtype = rng.choice(["float32", "float32", "bfloat16", "float16"])
        if op == "route":
            M = _log_int(rng, 2, 512)
            c = _route("", _log_int(rng, 1, 262144), M, min(M, rng.choice([1, 1, 2, 3, 4, 6, 8])), dtype,
                       rng.choice(["component", "sample"]), rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5,
                       rng.random() < 0.3)
            small = c["N"] * M <= 1.6e7
        elif op == "exchange":
            M = _log_int(rng, 1, 512)
            c = _exchange("", _log_int(rng, 1, 65536), M, min(M, rng.choice([1, 2, 2, 4, 8])), _log_int(rng, 1, 12288), dtype,
                          rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3)
            small = c["N"] * c["top"] * c["H"] <= 6.4e7
        else:
            c = _choose("", _log_int(rng, 1, 50000), _log_int(rng, 2, 150000), dtype,
                        rng.choice(["none", "top_k", "top_p", "min_p", "all"]), rng.random() < 0.5, rng.random() < 0.3)
            small = c["B"] * c["V"] <= 8.4e6
        if small:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------------ inputs

def _wide(g, rows, H, dtype, padded):
    """[rows, H] standard normal values, inside a buffer of longer rows if `padded`."""
    t = torch.randn(rows, H + 8 if padded else H, generator=g, device="cuda").to(dtype)
    return t[:, :H]


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = dict(generator=g, device="cuda")
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "route":
        N, M, top = c["N"], c["M"], c["top"]
        # log-densities of images, or logits
        scale, shift = (40.0, -700.0) if c["by"] == "component" and dtype == torch.float32 else (2.0, 0.0)
        shape = (M, N) if c["by"] == "component" else (N, M)
        scores = torch.randn(shape, **dev).mul_(scale).add_(shift)
        if c["masked"]:
            scores.masked_fill_(torch.rand(shape, **dev) < 0.2, float("-inf"))
        scores = scores.to(dtype)
        s = dict(scores=scores if c["by"] == "component" else scores.t(), top=top, renormalise=c["renormalise"],
                 train=c["train"], coef=None, dweights=None, dlogp=None)
        if c["coef"]:
            s["coef"] = torch.log_softmax(torch.randn(M, **dev), 0)
            if c["masked"]:
                s["coef"].masked_fill_(torch.rand(M, **dev) < 0.1, float("-inf"))
        if c["train"]:
            s["dweights"] = torch.randn(N, top, **dev)
            s["dlogp"] = torch.ones(N, device="cuda") if c["coef"] else torch.randn(N, **dev)
    elif c["op"] == "exchange":
        N, M, top, H = c["N"], c["M"], c["top"], c["H"]
        popularity = torch.randn(M, **dev)
        ids = (popularity + torch.randn(N, M, **dev)).topk(top, 1).indices.to(torch.int32)
        if c["dropped"]:
            ids.masked_fill_(torch.rand(N, top, **dev) < 0.1, -1)
        w = torch.rand(N, top, **dev)
        s = dict(M=M, top=top, train=c["train"], ids=ids, weights=w / w.sum(1, keepdim=True),
                 x=_wide(g, N, H, dtype, c["padded"]), ys=_wide(g, N * top, H, dtype, c["padded"]),
                 xs=torch.zeros(N * top, H, dtype=dtype, device="cuda"))
        if c["train"]:
            s.update(dy=_wide(g, N, H, dtype, c["padded"]), dxs=_wide(g, N * top, H, dtype, c["padded"]),
                     dys=torch.zeros(N * top, H, dtype=dtype, device="cuda"))
    else:
        B, V = c["B"], c["V"]
        logits = torch.randn(B, V, **dev).mul_(3.0)
        if c["masked"]:
            logits.masked_fill_(torch.rand(B, V, **dev) < 0.3, float("-inf"))
            logits[B // 2].fill_(float("-inf"))
        # uniforms in the middle of 2^23 equal steps
        u = (torch.randint(1 << 23, (B,), **dev).float() + 0.5) / (1 << 23)
        n = B if c["per_row"] else 1
        f = c["filters"]
        settings = dict(temperature=0.5 + torch.rand(n, **dev), top_k=torch.zeros(n, dtype=torch.int32, device="cuda"),
                        top_p=torch.ones(n, device="cuda"), min_p=torch.zeros(n, device="cuda"))
        if f in ("top_k", "all"):
            settings["top_k"] = torch.randint(2, 200, (n,), **dev).to(torch.int32)
        if f in ("top_p", "all"):
            settings["top_p"] = 0.5 + 0.49 * torch.rand(n, **dev)
        if f in ("min_p", "all"):
            settings["min_p"] = 0.1 * torch.rand(n, **dev)
        if not c["per_row"]:
            settings = {k: v.item() for k, v in settings.items()}
        s = dict(logits=logits.to(dtype), u=u, **settings)
    s["op"] = c["op"]
    return s


# --------------------------------------------------------------------------------------------------- the passes

def run(s):
    return {"route": _run_route, "exchange": _run_exchange, "choose": _run_choose}[s["op"]](s)


def _run_route(s):
    if own:
        import paper_2004_06231_amd as P
        ids, weights, logp = P.einet_route(s["scores"], s["coef"], s["top"], renormalise=s["renormalise"])
        if not s["train"]:
            return ids, weights, logp
        dscores, dcoef = P.einet_route_backward(s["scores"], s["coef"], ids, weights, s["dweights"], s["dlogp"],
                                                renormalise=s["renormalise"])
        return ids, weights, logp, dscores, dcoef
    # sums of score and coefficient and their differences in 64 bits: neighbours are close to each other and large
    t = s["scores"].t().double()
    if s["coef"] is not None:
        t = t + s["coef"].double()
    values, order = torch.sort(t, dim=1, descending=True, stable=True)
    m = values[:, :1]
    e = torch.where(t == m, 0.0, t - m).float().exp()
    e = torch.where(t == float("-inf"), 0.0, e)
    z = e.sum(1, keepdim=True)
    p = torch.where(z > 0, e / z, 0.0)
    logp = (m + z.log().double()).float().squeeze(1)
    there = values[:, :s["top"]] > float("-inf")
    chosen = order[:, :s["top"]]
    ids = torch.where(there, chosen, -1).to(torch.int32)
    weights = torch.where(there, p.gather(1, chosen), 0.0)
    if s["renormalise"]:
        total = weights.sum(1, keepdim=True)
        weights = torch.where(total > 0, weights / total, 0.0)
    if not s["train"]:
        return ids, weights, logp
    dw, dlogp = s["dweights"], s["dlogp"][:, None]
    mean = (dw * weights).sum(1, keepdim=True)
    dt = p * (dlogp if s["renormalise"] else dlogp - mean)
    dt = dt.scatter_add(1, chosen, weights * (dw - mean) if s["renormalise"] else weights * dw)
    return ids, weights, logp, dt.t().to(s["scores"].dtype), dt.sum(0)


def _run_exchange(s):
    M, top, x, ys, weights = s["M"], s["top"], s["x"], s["ys"], s["weights"]
    if own:
        import paper_2004_06231_amd as P
        first, place = P.einet_sort(s["ids"], M)
        xs = P.einet_dispatch(x, place, out=s["xs"])
        y = P.einet_combine(ys, place, weights)
        if not s["train"]:
            return first, place, xs, y
        dys, dweights = P.einet_combine_backward(s["dy"], ys, place, weights, out=s["dys"])
        dx = P.einet_combine(s["dxs"], place)
        return first, place, xs, y, dys, dweights, dx
    flat = s["ids"].reshape(-1).long()
    there = (flat >= 0) & (flat < M)
    key, order = torch.sort(torch.where(there, flat, M), stable=True)
    slots = torch.arange(flat.numel(), device=flat.device)
    first = torch.searchsorted(key, torch.arange(M + 1, device=flat.device))
    place = torch.where(there, torch.empty_like(order).scatter_(0, order, slots), -1).reshape(s["ids"].shape)
    filled = (slots < first[M])[:, None]
    xs = torch.where(filled, x[order // top], s["xs"])
    at, has = place.clamp(min=0), (place >= 0)[:, :, None]
    rows = torch.where(has, ys[at].float(), 0.0)
    y = (weights[:, :, None] * rows).sum(1).to(x.dtype)
    first, place = first.to(torch.int32), place.to(torch.int32)
    if not s["train"]:
        return first, place, xs, y
    dy = s["dy"].float()
    dys = torch.where(filled, (weights.reshape(-1)[order, None] * dy[order // top]).to(x.dtype), s["dys"])
    dweights = (rows * dy[:, None, :]).sum(2)
    dx = torch.where(has, s["dxs"][at].float(), 0.0).sum(1).to(x.dtype)
    return first, place, xs, y, dys, dweights, dx


def _setting(v, device):
    return torch.as_tensor(v, dtype=torch.float32, device=device).double().reshape(-1, 1)


def _run_choose(s):
    if own:
        import paper_2004_06231_amd as P
        return P.einet_choose(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                              min_p=s["min_p"])
    # weights and their running sums in 64 bits: the choice is a comparison with one of very many close values
    x = s["logits"].double()
    V, device = x.shape[1], x.device
    x = torch.where(torch.isnan(x), float("-inf"), x)
    values, order = torch.sort(x, dim=1, descending=True, stable=True)
    temperature, top_k, top_p, min_p = (_setting(s[k], device) for k in ("temperature", "top_k", "top_p", "min_p"))
    m = values[:, :1]
    w = torch.where(values == m, 0.0, values - m) / torch.where(temperature > 0, temperature, 1.0)
    w = torch.where(values > float("-inf"), w.exp(), 0.0)
    rank = torch.arange(V, device=device)
    keep = ((top_k <= 0) | (rank < top_k)) & (values > float("-inf"))
    running = torch.where(keep, w, 0.0).cumsum(1)
    before = torch.cat([torch.zeros_like(m), running[:, :-1]], 1)
    keep &= (top_p >= 1) | (before < top_p * running[:, -1:])
    keep &= w >= min_p.clamp(max=1.0)
    keep &= (temperature > 0) | (rank == 0)
    keep[:, 0] = True
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    running = kept.cumsum(1)
    total = running[:, -1:]
    at = (running > s["u"].double()[:, None] * total).to(torch.uint8).argmax(1, keepdim=True)
    alive = total > 0
    index = torch.where(alive, at, -1).to(torch.int32).squeeze(1)
    logq = torch.where(alive, (kept.gather(1, at) / total).log(), float("-inf")).float().squeeze(1)
    return index, logq


def work(c):
    """Bytes: every input read and every output written once.  Flops: a handful per score, the weighted sums of rows, an
    exponential and a sum per logit."""
    e = 4 if c["dtype"] == "float32" else 2
    if c["op"] == "route":
        N, M, top = c["N"], c["M"], c["top"]
        b = N * M * e + (4 * M if c["coef"] else 0) + N * (8 * top + 4)
        if c["train"]:
            b += N * M * e + 4 * M + N * (4 * top + 4)
        return {"bytes": float(b), "flops": 4.0 * N * M * (2 if c["train"] else 1)}
    if c["op"] == "exchange":
        N, M, top, H = c["N"], c["M"], c["top"], c["H"]
        slots = N * top
        b = 12 * slots + 4 * (M + 1) + 2 * e * H * (N + slots)
        f = 2.0 * slots * H
        if c["train"]:
            b += 4 * slots + 2 * e * H * (N + slots)
            f += 4.0 * slots * H
        return {"bytes": float(b), "flops": f}
    B, V = c["B"], c["V"]
    return {"bytes": float(B * V * e + 12 * B + (16 * B if c["per_row"] else 0)), "flops": 4.0 * B * V}


# ------------------------------------------------------------------------------------------------------ 64 bits

def _host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def exact(c, seed):
    s = prepare(c, seed)
    with np.errstate(all="ignore"):
        return {"route": _exact_route, "exchange": _exact_exchange, "choose": _exact_choose}[c["op"]](s)


def _exact_route(s):
    t = _host(s["scores"])
    if s["coef"] is not None:
        t = t + _host(s["coef"])[:, None]
    M, N = t.shape
    top = s["top"]
    m = t.max(0)
    e = np.exp(t - np.where(np.isfinite(m), m, 0.0))
    z = e.sum(0)
    p = np.divide(e, z, out=np.zeros_like(e), where=z > 0)
    logp = m + np.log(np.where(z > 0, z, 1.0))
    ids, weights, left = np.full((N, top), -1, np.int32), np.zeros((N, top)), t.copy()
    every = np.arange(N)
    for k in range(top):
        best = left.argmax(0)
        there = left[best, every] > -np.inf
        ids[:, k] = np.where(there, best, -1)
        weights[:, k] = np.where(there, p[best, every], 0.0)
        left[best, every] = -np.inf
    if s["renormalise"]:
        total = weights.sum(1, keepdims=True)
        weights = np.divide(weights, total, out=np.zeros_like(weights), where=total > 0)
    if not s["train"]:
        return ids, weights, logp
    dw, dlogp = _host(s["dweights"]), _host(s["dlogp"])
    # through the softmax: d p[j] / d t[c] = p[j] ([j = c] - p[c]), and through the quotient of the weights
    g = dw.copy()
    if s["renormalise"]:
        mass = np.where(ids >= 0, p[np.maximum(ids, 0), every[:, None]], 0.0).sum(1, keepdims=True)
        g = np.divide(dw - (dw * weights).sum(1, keepdims=True), mass, out=np.zeros_like(dw), where=mass > 0)
    dp = np.zeros_like(t)
    for k in range(top):
        there = ids[:, k] >= 0
        dp[ids[there, k], every[there]] += g[there, k]
    dt = p * (dp - (p * dp).sum(0)) + p * dlogp
    return ids, weights, logp, dt, dt.sum(1)


def _exact_exchange(s):
    ids, weights = _host(s["ids"]), _host(s["weights"])
    N, top = ids.shape
    x, ys, xs = _host(s["x"]), _host(s["ys"]), _host(s["xs"])
    M = s["M"]
    place, first, rows = np.full(N * top, -1, np.int32), np.zeros(M + 1, np.int32), []
    flat = ids.reshape(-1)
    for c in range(M):
        mine = np.flatnonzero(flat == c)
        place[mine] = first[c] + np.arange(mine.size, dtype=np.int32)
        first[c + 1] = first[c] + mine.size
        rows.append(mine)
    rows = np.concatenate(rows)
    xs[:rows.size] = x[rows // top]
    place = place.reshape(N, top)
    y = np.zeros_like(x)
    for k in range(top):
        there = place[:, k] >= 0
        y[there] += weights[there, k, None] * ys[place[there, k]]
    if not s["train"]:
        return first, place, xs, y
    dy, dxs, dys = _host(s["dy"]), _host(s["dxs"]), _host(s["dys"])
    dys[:rows.size] = weights.reshape(-1)[rows, None] * dy[rows // top]
    dweights, dx = np.zeros((N, top)), np.zeros_like(x)
    for k in range(top):
        there = place[:, k] >= 0
        dweights[there, k] = np.einsum("nh,nh->n", dy[there], ys[place[there, k]])
        dx[there] += dxs[place[there, k]]
    return first, place, xs, y, dys, dweights, dx


def _exact_choose(s):
    x, u = _host(s["logits"]), _host(s["u"])
    B, V = x.shape
    settings = [np.broadcast_to(_host(torch.as_tensor(s[k], dtype=torch.float32)).reshape(-1), (B,))
                for k in ("temperature", "top_k", "top_p", "min_p")]
    index, logq = np.full(B, -1, np.int32), np.full(B, -np.inf)
    for b in range(B):
        T, k, p, mp = (v[b] for v in settings)
        row = x[b]
        left = np.flatnonzero(row > -np.inf)
        if left.size == 0:
            continue
        left = left[np.argsort(-row[left], kind="stable")]
        if T <= 0:
            index[b], logq[b] = left[0], 0.0
            continue
        if k > 0:
            left = left[:int(k)]
        w = np.exp((row[left] - row[left[0]]) / T)
        if p < 1:
            running = np.cumsum(w)
            n = max(1, 1 + np.count_nonzero(running[:-1] < p * running[-1]))
            left, w = left[:n], w[:n]
        n = max(1, np.count_nonzero(w >= min(mp, 1.0)))
        back = np.argsort(left[:n])
        left, w = left[back], w[back]
        running = np.cumsum(w)
        at = np.searchsorted(running, u[b] * running[-1], side="right")
        index[b], logq[b] = left[at], np.log(w[at] / running[-1])
    return index, logq
