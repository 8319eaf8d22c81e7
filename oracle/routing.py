"""Float64 oracle of the operators around a mixture whose samples are routed to its components: the most probable
components of a sample, slots sorted by component, rows there and back with their gradients, and a choice from logits
under temperature, top-k, top-p and min-p.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain loops over the definitions; pinned by
tests/test_oracle_routing.py (gradients against differences, choices against enumerated distributions)."""
import math

import numpy as np


def route(scores, log_coef=None, top=1, renormalise=False):
    """scores [M, N].  Returns ids [N, top], weights [N, top], logp [N] and the posteriors p [M, N]."""
    t = np.asarray(scores, np.float64)
    if log_coef is not None:
        with np.errstate(invalid="ignore"):
            t = t + np.asarray(log_coef, np.float64)[:, None]
    M, N = t.shape
    t = np.where(np.isnan(t), -np.inf, t)
    ids, weights = np.full((N, top), -1, np.int32), np.zeros((N, top))
    logp, p = np.full(N, -np.inf), np.zeros((M, N))
    for n in range(N):
        m = t[:, n].max()
        if m == -np.inf:
            continue
        e = np.array([1.0 if v == m else (0.0 if m == np.inf else math.exp(v - m)) for v in t[:, n]])
        p[:, n] = e / e.sum()
        logp[n] = m + math.log(e.sum())
        order = sorted((c for c in range(M) if t[c, n] > -np.inf), key=lambda c: (-t[c, n], c))[:top]
        ids[n, :len(order)] = order
        weights[n, :len(order)] = p[order, n]
        if renormalise:
            weights[n] /= weights[n].sum()
    return ids, weights, logp, p


def route_backward(scores, log_coef, ids, dweights=None, dlogp=None, renormalise=False):
    """dscores [M, N], dlog_coef [M]: the sum over the weights of dweights times their derivatives, written out."""
    top = 1 if ids is None else ids.shape[1]
    _, w, _, p = route(scores, log_coef, top, renormalise)
    M, N = p.shape
    g = np.zeros((M, N))
    for n in range(N):
        if dlogp is not None:
            g[:, n] += dlogp[n] * p[:, n]
        if dweights is None:
            continue
        chosen = [c for c in ids[n] if c >= 0]
        for s, c in enumerate(chosen):
            for k in range(M):
                if renormalise:
                    dw = w[n, s] * ((k == c) - (w[n, chosen.index(k)] if k in chosen else 0.0))
                else:
                    dw = w[n, s] * ((k == c) - p[k, n])
                g[k, n] += dweights[n, s] * dw
    return g, g.sum(1)


def sort(ids, M):
    """first [M + 1], place like ids."""
    flat = np.asarray(ids).reshape(-1)
    first, place = np.zeros(M + 1, np.int32), np.full(flat.size, -1, np.int32)
    at = 0
    for c in range(M):
        mine = np.flatnonzero(flat == c)
        place[mine] = at + np.arange(mine.size)
        at += mine.size
        first[c + 1] = at
    return first, place.reshape(np.shape(ids))


def dispatch(x, place, out):
    out = out.copy()
    for (n, s), at in np.ndenumerate(place):
        if 0 <= at < out.shape[0]:
            out[at] = x[n]
    return out


def combine(rows, place, weights=None):
    rows = np.asarray(rows, np.float64)
    out = np.zeros((place.shape[0],) + rows.shape[1:])
    for (n, s), at in np.ndenumerate(place):
        if 0 <= at < rows.shape[0]:
            out[n] += (1.0 if weights is None else float(weights[n, s])) * rows[at]
    return out


def combine_backward(dout, rows, place, weights, drows):
    drows, dweights = np.asarray(drows, np.float64).copy(), np.zeros(place.shape)
    for (n, s), at in np.ndenumerate(place):
        if 0 <= at < rows.shape[0]:
            drows[at] = float(weights[n, s]) * np.asarray(dout[n], np.float64)
            dweights[n, s] = np.sum(np.asarray(dout[n], np.float64) * np.asarray(rows[at], np.float64))
    return drows, dweights


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The kept entries of one row, {index: weight}; empty where no entry is left."""
    x = [float(v) for v in logits]
    left = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: (-x[i], i))
    if not left:
        return {}
    if not temperature > 0:
        return {left[0]: 1.0}
    m = x[left[0]]
    w = {i: 1.0 if x[i] == m else (0.0 if m == math.inf else math.exp((x[i] - m) / temperature)) for i in left}
    if top_k > 0:
        left = left[:top_k]
    if top_p < 1:
        total, before, keep = math.fsum(w[i] for i in left), 0.0, []
        for i in left:
            if keep and not before < top_p * total:
                break
            keep.append(i)
            before += w[i]
        left = keep
    return {i: w[i] for i in left if w[i] >= min(min_p, 1.0)}


def choose(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(index, log of its share) of one row."""
    k = kept(logits, temperature, top_k, top_p, min_p)
    if not k:
        return -1, -math.inf
    total, run = math.fsum(k.values()), 0.0
    u = u if u > 0 else 0.0
    for i in sorted(k):
        run += k[i]
        if run > u * total and k[i] > 0:
            return i, math.log(k[i] / total)
    last = max(i for i in k if k[i] > 0)
    return last, math.log(k[last] / total)
