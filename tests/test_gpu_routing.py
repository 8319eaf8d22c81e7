"""The operators around a mixture whose samples are routed to its components, against the float64 oracle.

Tolerances.  u = 2^-24 is half a step of float32.
  route     a posterior is exp(d) / z: d = t - m is exact in float64 and rounded to float32 (u |d| relative), exp is within
            2 steps (4 u), z adds at most 16 terms in a lane and 6 times across lanes after errors of its own terms of the same
            kind (their d weighted by their share, below 8 on average for up to 1024 terms), and one quotient, two where
            the weights are renormalised: u (|d| + 48) relative.  logp adds m (float64) and log z (z's relative error
            and 4 u of log z < 7), rounded once: u (|logp| + 96).
  gradient  a sum of products of such numbers with dweights and dlogp, at most 16 + 6 additions long: u (|d| + 96) times
            the sum of the terms' magnitudes, and half a step of the type that is written.  Over n samples: a lane adds up
            at most n / 1024 + 16 of them, which bounds the relative error of a sum of magnitudes by as many u.
  combine   top products and additions in float32: u (top + 2) of the sum of magnitudes, and half a step of the type.
  dweights  products and sums over a row of H: at most H / 64 + 64 additions in a lane and 16 across: u (H / 64 + 82) of
            the sum of magnitudes.
  choose    the index is the oracle's; its log-share comes from float64 numbers (2^-36 for their sums and logarithms, which stay
            below 2^7) and from a total of V weights, each rounded to a multiple of 2^-(61 - ceil(log2 V)) of the largest: off
            by V / 2 such units of a total of one at least, rounded once: u |logq| + 2^-36 + V 2^-(62 - ceil(log2 V)).
"""
import math

import numpy as np
import pytest
import torch

import paper_2004_06231_amd as P
from oracle import routing as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}            # half a step, relative to the value
SMALLEST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}   # below: absolute error


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def close(got, want, tol):
    got, want = host(got), np.asarray(want, np.float64)
    assert got.shape == want.shape
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin])
    err = np.abs(got[fin] - want[fin])
    tol = np.broadcast_to(tol, want.shape)[fin]
    assert np.all(err <= tol), f"worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of its tolerance"


# ------------------------------------------------------------------------------------------------------ route

def check_route(scores, coef, top, renormalise, grad=True, seed=0):
    ids, w, logp = P.einet_route(scores, coef, top, renormalise=renormalise)
    s, a = host(scores), None if coef is None else host(coef)
    rid, rw, rlogp, p = R.route(s, a, top, renormalise)
    assert np.array_equal(host(ids), rid)
    with np.errstate(all="ignore"):
        t = s if a is None else s + a[:, None]
        t = np.where(np.isnan(t), -np.inf, t)
        m = t.max(0)
        d = np.where(t == m, 0.0, m - t)
        d = np.where(np.isfinite(d), d, 0.0)
    dsel = np.where(rid >= 0, d[np.maximum(rid, 0), np.arange(d.shape[1])[:, None]], 0.0)
    # (a share of the selected ones: the largest of them is the largest of all, d = 0)
    close(w, rw, U * (dsel + 48) * rw + 2.0 ** -125)
    fin = np.where(np.isfinite(rlogp), np.abs(rlogp), 0.0)
    close(logp, rlogp, U * (fin + 96))
    if not grad:
        return
    rng = np.random.default_rng(seed)
    n, M = d.shape[1], d.shape[0]
    dw, dl = rng.normal(size=(n, top)).astype(np.float32), rng.normal(size=n).astype(np.float32)
    for use_w, use_l in ((True, True), (True, False), (False, True)):
        gw, gl = dw if use_w else None, dl if use_l else None
        g, ga = P.einet_route_backward(scores, coef, ids, w, None if gw is None else torch.tensor(gw).cuda(),
                                       None if gl is None else torch.tensor(gl).cuda(), renormalise=renormalise)
        rg, rga = R.route_backward(s, a, rid, gw, gl, renormalise)
        mag = np.zeros_like(d)
        if use_l:
            mag += p * np.abs(dl)
        if use_w:
            each = np.abs(dw) * rw
            mag += (0.0 if renormalise else p) * each.sum(1)
            for k in range(top):
                there = rid[:, k] >= 0
                mag[rid[there, k], np.flatnonzero(there)] += each[there, k] + (rw[there, k] * each[there].sum(1) if renormalise else 0.0)
        tol = U * (d + 96 + (48 if use_w else 0)) * mag + 2.0 ** -120
        assert g.dtype == scores.dtype and g.shape == scores.shape
        close(g, rg, tol + HALF[g.dtype] * np.abs(rg) * 1.01 + SMALLEST[g.dtype])
        close(ga, rga, (tol + U * (n / 1024 + 16 + 16) * mag).sum(1) + U * np.abs(rga))


@pytest.mark.parametrize("M,N,top", [(1, 1, 1), (2, 3, 2), (3, 1, 3), (8, 5, 2), (7, 300, 5), (16, 65, 16), (33, 70, 9), (64, 130, 4),
                                     (100, 501, 1), (128, 37, 8), (129, 20, 3), (257, 33, 2), (512, 9, 16), (1000, 11, 4), (1024, 5, 8)])
@pytest.mark.parametrize("by", ["component", "sample"])
def test_route_matches_oracle(M, N, top, by):
    rng = np.random.default_rng(M * 1000 + N)
    for i, name in enumerate(TYPES):
        x = rng.normal(-700.0 if name == "float32" and by == "component" else 0.0, 5.0, (M, N)).astype(np.float32)
        if i != 2 and M > 1:
            x[rng.random((M, N)) < 0.2] = -np.inf
        x = torch.tensor(x).cuda().to(TYPES[name])
        x = x if by == "component" else x.t().contiguous().t()
        coef = torch.tensor(np.log(rng.dirichlet(np.ones(M))).astype(np.float32)).cuda() if i != 1 else None
        print("route", M, N, top, by, name, flush=True)
        check_route(x, coef, top, renormalise=(M + i) % 2 == 0)


def test_route_of_many_samples_and_strided_scores():
    rng = np.random.default_rng(3)
    x = torch.tensor(rng.normal(0, 2, (5, 20011)).astype(np.float32)).cuda()
    check_route(x, None, 2, True)
    wide = torch.tensor(rng.normal(0, 2, (24, 77)).astype(np.float32)).cuda()
    for view in (wide[::2, :], wide[:, ::3], wide[3:13, 5:50], wide.t()[1::2], wide[:, 4:5].expand(24, 9)):
        check_route(view, None, 3, False)
        check_route(view.to(torch.bfloat16) if view.stride(1) else view, None, 1, True)


@pytest.mark.parametrize("M,N,top,dtype,with_coef,renormalise", [
    (16, 70001, 1, "float32", True, False), (5, 65537, 3, "bfloat16", False, True), (1, 66000, 1, "float32", True, True),
    (64, 131073, 2, "float32", True, True), (33, 140000, 4, "float16", True, False), (64, 131072, 1, "float32", False, False),
    (64, 131072, 6, "float32", True, True), (17, 8193, 2, "float32", True, False), (100, 9001, 5, "bfloat16", True, True),
    (300, 8200, 16, "float32", True, False), (512, 8199, 3, "float16", False, False), (1000, 8500, 8, "float32", True, True)])
def test_route_of_many_samples_next_to_each_other(M, N, top, dtype, with_coef, renormalise):
    """The kernels that scores [n_components, n] of many samples get, against the formulas in float64 over whole arrays."""
    print("route many", M, N, top, dtype, with_coef, renormalise, flush=True)
    rng = np.random.default_rng(M + N)
    x = rng.normal(-50.0, 5.0, (M, N)).astype(np.float32)
    x[rng.random((M, N)) < 0.15] = -np.inf
    x[:, 7] = -np.inf
    x[:, N - 1] = 3.0
    x = torch.tensor(x).cuda().to(TYPES[dtype])
    coef = np.log(rng.dirichlet(np.ones(M))).astype(np.float32) if with_coef else None
    dev_coef = None if coef is None else torch.tensor(coef).cuda()
    ids, w, logp = P.einet_route(x, dev_coef, top, renormalise=renormalise)
    t = host(x) + (0.0 if coef is None else coef.astype(np.float64)[:, None])
    m = t.max(0)
    alive = m > -np.inf
    e = np.where(alive, np.exp(np.minimum(t - np.where(alive, m, 0.0), 0.0)), 0.0)
    z = np.where(alive, e.sum(0), 1.0)
    p = e / z
    order = np.argsort(-t, axis=0, kind="stable")[:top].T
    n = np.arange(N)[:, None]
    rid = np.where(t[order, n] > -np.inf, order, -1)
    rw = np.where(rid >= 0, p[order, n], 0.0)
    if renormalise:
        rw = rw / np.where(alive, rw.sum(1), 1.0)[:, None]
    rlogp = np.where(alive, np.where(alive, m, 0.0) + np.log(z), -np.inf)
    assert np.array_equal(host(ids), rid)
    d = np.where(np.isfinite(t) & alive, m - np.where(np.isfinite(t), t, 0.0), 0.0)
    dsel = np.where(rid >= 0, d[order, n], 0.0)
    close(w, rw, U * (dsel + 48) * rw + 2.0 ** -125)
    close(logp, rlogp, U * (np.where(alive, np.abs(rlogp), 0.0) + 96))
    dw, dl = rng.normal(size=(N, top)).astype(np.float32), rng.normal(size=N).astype(np.float32)
    for use_w, use_l in ((True, True), (False, True)):
        g, ga = P.einet_route_backward(x, dev_coef, ids, w, torch.tensor(dw).cuda() if use_w else None, torch.tensor(dl).cuda() if use_l else None,
                                       renormalise=renormalise)
        lw, ll = dw.astype(np.float64) * use_w, dl.astype(np.float64) * use_l
        a = (lw * rw).sum(1)
        rg = p * (ll if renormalise else ll - a)
        mag = p * (np.abs(ll) + (0.0 if renormalise else (np.abs(lw) * rw).sum(1)))
        for k in range(top):
            there = rid[:, k] >= 0
            at = (rid[there, k], np.flatnonzero(there))
            rg[at] += (rw * (lw - a[:, None] if renormalise else lw))[there, k]
            mag[at] += (rw * (np.abs(lw) + (np.abs(lw) * rw).sum(1)[:, None] if renormalise else np.abs(lw)))[there, k]
        tol = U * (d + 96 + (48 if use_w else 0)) * mag + 2.0 ** -120
        close(g, rg, tol + HALF[g.dtype] * np.abs(rg) * 1.01 + SMALLEST[g.dtype])
        close(ga, rg.sum(1), (tol + U * (N / 1024 + 32) * mag).sum(1) + U * np.abs(rg.sum(1)))


def test_route_rows_where_nothing_or_little_is_left():
    nan, inf, low = math.nan, math.inf, torch.finfo(torch.float32).min
    cols = [[-inf] * 4, [nan] * 4, [nan, -inf, 1.0, nan], [low, low, 0.0, low], [low] * 4, [inf, 0.0, inf, -inf], [inf, nan, 1.0, -3e38],
            [0.0, -0.0, 0.0, -0.0], [1e-45, -1e-45, 0.0, 3e38], [5.0, 5.0, 5.0, 5.0]]
    x = torch.tensor(cols, device="cuda").t().contiguous()
    for renormalise in (False, True):
        for top in (1, 3, 4):
            ids, w, logp = P.einet_route(x, None, top, renormalise=renormalise)
            rid, rw, rlogp, p = R.route(host(x), None, top, renormalise)
            assert np.array_equal(host(ids), rid)
            close(w, rw, 48 * U * rw + 2.0 ** -125)
            close(logp, rlogp, U * (np.where(np.isfinite(rlogp), np.abs(rlogp), 0) + 96))
            g, ga = P.einet_route_backward(x, None, ids, w, torch.ones_like(w), torch.ones_like(logp), renormalise=renormalise)
            rg, rga = R.route_backward(host(x), None, rid, np.ones(rid.shape), np.ones(len(cols)), renormalise)
            assert bool(torch.isfinite(g).all()) and bool(torch.isfinite(ga).all())
            close(g, rg, 200 * U * (1 + top))
            close(ga, rga, 200 * U * (1 + top) * len(cols))
    # a closed component hides what it would have said
    closed = torch.tensor([0.0, -inf, 0.0, 0.0], device="cuda")
    x = torch.tensor([[0.0, nan], [inf, 7.0], [1.0, 1.0], [nan, -inf]], device="cuda")
    ids, w, logp = P.einet_route(x, closed, 2)
    assert host(ids).tolist() == [[2, 0], [2, -1]] and float(logp[1]) == 1.0


def test_route_gradient_is_the_mixtures_e_step():
    rng = np.random.default_rng(5)
    x = torch.tensor(rng.normal(-300, 3, (12, 700)).astype(np.float32)).cuda()
    coef = torch.tensor(np.log(rng.dirichlet(np.ones(12))).astype(np.float32)).cuda()
    g, counts = P.einet_route_backward(x, coef, None, None, None, torch.ones(700, device="cuda"))
    p = R.route(host(x), host(coef), 1)[3]
    close(g, p, U * 200 * p + 2.0 ** -125)
    close(counts, p.sum(1), U * 250 * p.sum(1))
    assert abs(float(counts.double().sum()) - 700) < 700 * 250 * U


# --------------------------------------------------------------------------------------------------- exchange

@pytest.mark.parametrize("N,top,M", [(0, 2, 3), (1, 1, 1), (1, 3, 7), (63, 1, 2), (64, 1, 1), (65, 2, 1024), (1000, 1, 100), (777, 5, 13),
                                     (4096, 4, 64), (30011, 2, 257), (5, 8, 900), (70001, 1, 3), (150001, 8, 512)])
def test_sort_matches_oracle(N, top, M):
    rng = np.random.default_rng(N + top)
    for kind in range(3):
        ids = rng.integers(0, M, (N, top)).astype(np.int32)
        if kind == 1:                                            # most slots in one component, some nowhere
            ids[rng.random((N, top)) < 0.7] = M // 2
            drop = rng.random((N, top))
            ids[drop < 0.1] = -1
            ids[drop > 0.95] = M + 5
        if kind == 2:
            ids[:] = -1 if N % 2 else M - 1
        print("sort", N, top, M, kind, flush=True)
        first, place = P.einet_sort(torch.tensor(ids).cuda(), M)
        rfirst, rplace = R.sort(ids, M)
        assert np.array_equal(host(first), rfirst) and np.array_equal(host(place), rplace)


def rows_in(t, layout):
    """The rows of t: dense, inside wider rows, or from an address that only the element's size divides."""
    if layout == "dense":
        return t.contiguous()
    wide = torch.zeros(t.shape[0], t.shape[1] + (16 if layout == "wide" else 3), dtype=t.dtype, device=t.device)
    view = wide[:, 8:8 + t.shape[1]] if layout == "wide" else wide[:, 1:1 + t.shape[1]]
    view.copy_(t)
    return view


CASES = [(1, 1, 1, 1), (3, 2, 8, 784), (5, 1, 2, 7), (64, 2, 5, 64), (33, 8, 16, 130), (257, 4, 7, 33), (40, 3, 100, 1000), (9, 2, 3, 4097),
         (500, 1, 10, 2), (1200, 2, 64, 3), (130, 16, 20, 96), (17, 2, 4, 12288), (700, 6, 9, 8), (300, 2, 8, 256)]


@pytest.mark.parametrize("N,top,M,H", CASES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd"])
def test_rows_there_and_back_match_oracle(N, top, M, H, layout):
    rng = np.random.default_rng(N * 7 + H)
    for name, dtype in TYPES.items():
        ids = np.stack([rng.permutation(max(M, top))[:top] for _ in range(N)]).astype(np.int32)
        if H % 2:
            ids[rng.random((N, top)) < 0.25] = -1
        print("exchange", N, top, M, H, layout, name, flush=True)
        first, place = P.einet_sort(torch.tensor(ids).cuda(), M)
        x, rows, dy = (rows_in(torch.tensor(rng.normal(size=(n, H)).astype(np.float32)).cuda().to(dtype), layout) for n in (N, N * top, N))
        w = torch.tensor(rng.random((N, top)).astype(np.float32)).cuda()
        pl = host(place)
        used = int(first[M])
        xs = rows_in(torch.full((N * top, H), 7.0, device="cuda", dtype=dtype), layout)
        assert P.einet_dispatch(x, place, out=xs) is xs
        want = R.dispatch(host(x), pl, np.full((N * top, H), 7.0))
        assert np.array_equal(host(xs), want) and (want[used:] == 7.0).all()
        for weights in (w, None):
            y = P.einet_combine(rows, place, weights)
            ry = R.combine(host(rows), pl, None if weights is None else host(w))
            mag = R.combine(np.abs(host(rows)), pl, None if weights is None else host(w))
            close(y, ry, U * (top + 2) * mag + HALF[dtype] * 1.01 * np.abs(ry) + SMALLEST[dtype])
        drows = rows_in(torch.full((N * top, H), 7.0, device="cuda", dtype=dtype), layout)
        drows, dw = P.einet_combine_backward(dy, rows, place, w, out=drows)
        rdrows, rdw = R.combine_backward(host(dy), host(rows), pl, host(w), np.full((N * top, H), 7.0))
        mag = R.combine_backward(np.abs(host(dy)), np.abs(host(rows)), pl, host(w), rdrows)[1]
        close(drows, rdrows, (2 * U + HALF[dtype] * 1.01) * np.abs(rdrows) + SMALLEST[dtype])
        assert (host(drows)[used:] == 7.0).all()
        close(dw, rdw, U * (H / 64 + 82) * mag + 2.0 ** -125)


def test_rows_of_any_type_and_shape_are_carried():
    rng = np.random.default_rng(11)
    ids = torch.tensor(rng.integers(0, 4, (37, 2)).astype(np.int32)).cuda()
    first, place = P.einet_sort(ids, 4)
    for shape, dtype in (((5, 7), torch.uint8), ((3,), torch.uint8), ((16,), torch.int64), ((2, 3, 2), torch.float64), ((9, 3), torch.float32)):
        x = torch.tensor(rng.integers(0, 100, (37,) + shape)).cuda().to(dtype)
        xs = P.einet_dispatch(x, place)
        assert np.array_equal(host(xs), R.dispatch(host(x), host(place), np.zeros((74,) + shape)))
    # one row for all samples
    x = torch.arange(6.0, device="cuda")[None].expand(37, 6)
    assert bool((P.einet_dispatch(x, place) == x[0]).all())
    # a batch without samples, rows without elements
    empty, nowhere = torch.zeros(0, 6, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    assert P.einet_dispatch(empty, nowhere).shape == (0, 6) and P.einet_combine(empty, nowhere).shape == (0, 6)
    assert P.einet_combine(torch.zeros(74, 0, device="cuda"), place).shape == (37, 0)
    d, dw = P.einet_combine_backward(torch.zeros(37, 0, device="cuda"), torch.zeros(74, 0, device="cuda"), place, torch.ones(37, 2, device="cuda"))
    assert d.shape == (74, 0) and not bool(dw.any())


def test_batches_and_rows_of_length_zero():
    dev = dict(device="cuda")
    scores = torch.zeros(5, 0, **dev)
    ids, w, logp = P.einet_route(scores, torch.zeros(5, **dev), 3)
    assert ids.shape == (0, 3) and w.shape == (0, 3) and logp.shape == (0,)
    g, ga = P.einet_route_backward(scores, None, ids, w, w, logp)
    assert g.shape == (5, 0) and ga.tolist() == [0.0] * 5
    first, place = P.einet_sort(torch.zeros(0, 2, dtype=torch.int32, **dev), 3)
    assert first.tolist() == [0] * 4 and place.shape == (0, 2)
    # no sorted rows: every slot goes nowhere
    nowhere = torch.full((4, 2), -1, dtype=torch.int32, **dev)
    assert not bool(P.einet_combine(torch.empty(0, 6, **dev), nowhere, torch.ones(4, 2, **dev)).any())
    d, dw = P.einet_combine_backward(torch.ones(4, 6, **dev), torch.empty(0, 6, **dev), nowhere, torch.ones(4, 2, **dev))
    assert d.shape == (0, 6) and not bool(dw.any())
    assert P.einet_dispatch(torch.ones(4, 6, **dev), nowhere, out=torch.empty(0, 6, **dev)).shape == (0, 6)
    with pytest.raises(P.EinetError):
        P.einet_choose(torch.zeros(3, 0, **dev), torch.zeros(3, **dev))


def test_positions_out_of_range_go_nowhere():
    place = torch.tensor([[0, 99], [-7, 3], [2 ** 31 - 1, -1]], dtype=torch.int32, device="cuda")
    x = torch.arange(24.0, device="cuda").reshape(3, 8)
    out = torch.full((5, 8), -1.0, device="cuda")
    P.einet_dispatch(x, place, out=out)
    want = torch.full((5, 8), -1.0, device="cuda")
    want[0], want[3] = x[0], x[1]
    assert torch.equal(out, want)
    rows = torch.arange(40.0, device="cuda").reshape(5, 8)
    w = torch.ones(3, 2, device="cuda")
    assert torch.equal(P.einet_combine(rows, place, w), torch.stack([rows[0], rows[3], torch.zeros(8, device="cuda")]))
    d, dw = P.einet_combine_backward(x, rows, place, w, out=out.fill_(-1.0))
    assert torch.equal(d, want) and host(dw).tolist() == [[float((x[0] * rows[0]).sum()), 0.0], [0.0, float((x[1] * rows[3]).sum())], [0.0, 0.0]]


# ----------------------------------------------------------------------------------------------------- choose

def check_choose(logits, u, **settings):
    index, logq = P.einet_choose(logits, u, **settings)
    x, uu = host(logits), host(u)
    each = {k: np.broadcast_to(host(v) if torch.is_tensor(v) else np.float32(v), (len(uu),)) for k, v in settings.items()}
    want = [R.choose(x[b], uu[b], **{k: (int(v[b]) if k == "top_k" else float(v[b])) for k, v in each.items()}) for b in range(len(uu))]
    assert host(index).tolist() == [i for i, _ in want]
    q = np.array([v for _, v in want])
    V = x.shape[1]
    close(logq, q, U * np.where(np.isfinite(q), np.abs(q), 0) + 2.0 ** -36 + V * 2.0 ** -(62 - (V - 1).bit_length()))
    return index


def uniforms(rng, n):
    return torch.tensor(((rng.integers(0, 1 << 23, n) + 0.5) / (1 << 23)).astype(np.float32)).cuda()


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=5, temperature=1.3), dict(top_p=0.9), dict(top_p=0.3, temperature=0.5),
            dict(min_p=0.05), dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.02), dict(temperature=0.0, top_k=3), dict(temperature=30.0, top_p=0.99)]


@pytest.mark.parametrize("V", [1, 2, 3, 31, 64, 65, 100, 255, 256, 257, 511, 1000, 1023, 1024, 1025, 2049, 5000, 16384, 32769])
def test_choose_matches_oracle(V):
    rng = np.random.default_rng(V)
    B = 24 if V <= 1100 else 3
    for i, settings in enumerate(SETTINGS):
        for name, dtype in TYPES.items():
            x = rng.normal(0, 3, (B, V)).astype(np.float32)
            if i % 2:
                x[rng.random((B, V)) < 0.3] = -np.inf
            print("choose", V, settings, name, flush=True)
            check_choose(torch.tensor(x).cuda().to(dtype), uniforms(rng, B), **settings)


@pytest.mark.parametrize("B,V", [(1, 100003), (2, 65536), (5, 150001)])
def test_choose_from_long_rows(B, V):
    rng = np.random.default_rng(V)
    for settings in SETTINGS:
        for name, dtype in TYPES.items():
            x = torch.tensor(rng.normal(0, 3, (B, V)).astype(np.float32)).cuda().to(dtype)
            print("choose", B, V, settings, name, flush=True)
            check_choose(x, uniforms(rng, B), **settings)


@pytest.mark.parametrize("V", [7, 300, 3000, 40000])
def test_choose_with_settings_of_every_row(V):
    rng = np.random.default_rng(V)
    B = 16
    x = torch.tensor(rng.normal(0, 2, (B, V)).astype(np.float32)).cuda()
    t = rng.uniform(0.2, 2, B).astype(np.float32)
    t[3], t[4] = 0.0, 1e-6
    settings = dict(temperature=torch.tensor(t).cuda(), top_k=torch.tensor(rng.integers(0, min(V, 60), B).astype(np.int32)).cuda(),
                    top_p=torch.tensor(rng.uniform(0.3, 1.0, B).astype(np.float32)).cuda(),
                    min_p=torch.tensor(rng.uniform(0.0, 0.2, B).astype(np.float32)).cuda())
    check_choose(x, uniforms(rng, B), **settings)
    for name in settings:
        check_choose(x, uniforms(rng, B), **{name: settings[name]})


@pytest.mark.parametrize("V", [4, 200, 1500, 20000, 70000])
def test_choose_among_equal_and_masked_logits(V):
    rng = np.random.default_rng(V)
    nan, inf = math.nan, math.inf
    low = torch.finfo(torch.float32).min
    rows = [np.zeros(V), np.full(V, -inf), np.full(V, nan), np.full(V, low), rng.integers(0, 2, V) * 1.0, np.where(rng.random(V) < 0.5, 0.0, -0.0),
            np.where(rng.random(V) < 0.9, low, 1.0), np.where(rng.random(V) < 0.5, nan, 2.0), np.where(rng.random(V) < 0.9, -inf, 1e30),
            np.where(np.arange(V) % 3 == 1, inf, 5.0), np.where(np.arange(V) == V - 1, -3.0, -inf), np.where(np.arange(V) == V // 2, 0.0, low),
            np.linspace(-3e38, 3e38, V), np.full(V, 1e-45), rng.integers(0, 3, V) * 1e-40]
    x = torch.tensor(np.stack(rows).astype(np.float32)).cuda()
    for settings in (dict(), dict(top_k=max(1, V // 3)), dict(top_p=0.5), dict(min_p=1.0), dict(top_k=V), dict(top_k=V + 5, top_p=0.25),
                     dict(temperature=0.0), dict(top_p=0.0), dict(temperature=1e-30), dict(top_k=V - 1, top_p=0.999, min_p=0.5, temperature=2.0)):
        print("choose ties", V, settings, flush=True)
        check_choose(x, uniforms(rng, len(rows)), **settings)
        if V <= 20000:
            check_choose(x.to(torch.bfloat16), uniforms(rng, len(rows)), **settings)


@pytest.mark.parametrize("V", [5, 1000, 3000, 50000])
def test_choose_at_the_ends_of_the_uniforms(V):
    x = torch.zeros(6, V, device="cuda")
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, math.nan, math.inf], device="cuda")
    index, logq = P.einet_choose(x, u)
    assert host(index).tolist() == [0, V - 1, V - 1, 0, 0, V - 1]
    close(logq, np.full(6, -math.log(V)), U * math.log(V) + 2.0 ** -36)
    index, _ = P.einet_choose(x, u, top_k=3)
    assert host(index).tolist() == [0, 2, 2, 0, 0, 2]
    # no entry without weight is ever chosen
    x[:, ::2] = -math.inf
    last = V - 1 if (V - 1) % 2 else V - 2
    assert host(P.einet_choose(x, u)[0]).tolist() == [1, last, last, 1, 1, last]
    x[:, 1::2] = -1000.0
    x[:, 3] = 0.0
    assert host(P.einet_choose(x, u)[0]).tolist() == [3] * 6


def test_choose_rows_in_wider_rows_and_the_same_row_for_all():
    rng = np.random.default_rng(8)
    for V in (100, 1030, 5001, 66000):
        wide = torch.tensor(rng.normal(0, 2, (5, V + 7)).astype(np.float32)).cuda()
        for dtype in TYPES.values():
            check_choose(wide.to(dtype)[:, 3:3 + V], uniforms(rng, 5), top_p=0.8)
        check_choose(wide[:1, 1:V].expand(40 if V < 2000 else 4, V - 1), uniforms(rng, 40 if V < 2000 else 4), top_k=50)
    assert P.einet_choose(torch.zeros(0, 9, device="cuda"), torch.zeros(0, device="cuda"))[0].shape == (0,)


@pytest.mark.parametrize("B,V", [(1100, 4100), (600, 8192), (2100, 5000), (1025, 20000)])
def test_choose_from_many_long_rows(B, V):
    """Rows enough for several batches: the same choices as from the rows alone, and the oracle's for some of them."""
    rng = np.random.default_rng(B)
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    x = torch.randn(B, V, generator=g, device="cuda") * 3
    u = uniforms(rng, B)
    t, k, p, m = (torch.rand(B, generator=g, device="cuda") for _ in range(4))
    settings = dict(temperature=t + 0.3, top_k=(k * 90).int(), top_p=0.5 + 0.6 * p, min_p=0.1 * m)
    for use in (dict(), dict(top_p=0.9), settings):
        print("choose", B, V, list(use), flush=True)
        index, logq = P.einet_choose(x, u, **use)
        for lo, hi in ((0, 9), (1020, 1030), (B - 7, B)):
            part = {k: v[lo:hi].contiguous() if torch.is_tensor(v) else v for k, v in use.items()}
            i, q = P.einet_choose(x[lo:hi], u[lo:hi].contiguous(), **part)
            assert torch.equal(i, index[lo:hi]) and torch.equal(q, logq[lo:hi])
        last = {k: v[B - 2:].contiguous() if torch.is_tensor(v) else v for k, v in use.items()}
        assert torch.equal(check_choose(x[B - 2:], u[B - 2:].contiguous(), **last), index[B - 2:])


def test_choices_have_the_frequencies_of_the_kept_distribution():
    n = 200000
    logits = torch.log(torch.tensor([0.05, 0.3, 0.15, 0.5], device="cuda"))
    u = (torch.arange(n, device="cuda") + 0.5) / n
    index, _ = P.einet_choose(logits[None].expand(n, 4), u.float(), top_k=3)
    got = torch.bincount(index.long(), minlength=4).double().cpu().numpy() / n
    # (stratified uniforms, rounded to float32: a share is off by two strata and a few roundings)
    np.testing.assert_allclose(got, [0.0, 0.3 / 0.95, 0.15 / 0.95, 0.5 / 0.95], atol=4 / n + 1e-6)


# --------------------------------------------------------------------------------------------------- together

def pass_of(x, scores, coef, dy, u):
    ids, w, logp = P.einet_route(scores, coef, 2, renormalise=True)
    first, place = P.einet_sort(ids, scores.shape[0])
    xs = P.einet_dispatch(x, place, out=torch.zeros(2 * x.shape[0], x.shape[1], device="cuda"))
    ys = xs * 2.0 - 1.0
    y = P.einet_combine(ys, place, w)
    dys, dw = P.einet_combine_backward(dy, ys, place, w, out=torch.zeros_like(ys))
    dx = P.einet_combine(dys * 2.0, place)
    ds, da = P.einet_route_backward(scores, coef, ids, w, dw, torch.ones_like(logp), renormalise=True)
    index, logq = P.einet_choose(y, u, top_p=0.9)
    return ids, w, logp, first, place, xs, y, dys, dw, dx, ds, da, index, logq


def inputs(seed, N=700, M=9, H=50):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    return [r(N, H), r(M, N), torch.log_softmax(r(M), 0), r(N, H), torch.rand(N, generator=g, device="cuda")]


def test_whole_pass_matches_oracle_and_differences():
    x, scores, coef, dy, u = inputs(1, N=40, M=5, H=6)
    out = pass_of(x, scores, coef, dy, u)
    X, S, A, D = (host(t) for t in (x, scores, coef, dy))

    def loss(X, S, A):
        ids, w, logp, _ = R.route(S, A, 2, True)
        y = np.zeros_like(X)
        for n in range(X.shape[0]):
            y[n] = sum(w[n, s] * (X[n] * 2 - 1) for s in range(2))
        return (y * D).sum() + logp.sum()

    h = 1e-6
    rng = np.random.default_rng(2)
    for t, g in ((X, out[9]), (S, out[10]), (A, out[11])):
        g = host(g)
        for _ in range(30):
            i = tuple(rng.integers(0, k) for k in t.shape)
            e = np.zeros_like(t)
            e[i] = h
            arg = [X, S, A]
            up = loss(*[a + e if a is t else a for a in arg])
            down = loss(*[a - e if a is t else a for a in arg])
            # float32 gradients of sums of at most 6 * 2 terms below 100; differences of float64 values of about 500 by 2e-6
            assert (up - down) / (2 * h) == pytest.approx(g[i], abs=1e-4)


def test_captured_pass_replays_on_new_inputs():
    """The pass captured once and replayed on other inputs, with eager work and synchronisations between the replays; a second
    graph of the same pass replayed on another stream at the same time."""
    state = inputs(3)
    pass_of(*state)
    torch.cuda.synchronize()
    other = inputs(4)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        out1 = pass_of(*state)
    with torch.cuda.graph(g2):
        out2 = pass_of(*other)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for rep in range(4):
        for t, v in zip(state, inputs(10 + rep)):
            t.copy_(v)
        for t, v in zip(other, inputs(20 + rep)):
            t.copy_(v)
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            g1.replay()
        with torch.cuda.stream(s2):
            g2.replay()
        torch.cuda.synchronize()
        for out, st in ((out1, state), (out2, other)):
            want = pass_of(*st)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {rep}"


def test_pass_on_another_stream_and_twice_the_same():
    state = inputs(5, N=3001, M=64, H=77)
    want = pass_of(*state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [pass_of(*state) for _ in range(2)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_offsets_beyond_32_bits():
    """Tensors of more than 2^31 elements and 2^32 bytes: the last rows are where a 32-bit offset would go wrong."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    # rows: 300001 samples with two slots of 4096 bf16 values
    N, H = 300001, 4096
    x = torch.randn(N, H, generator=g, device="cuda", dtype=torch.bfloat16)
    first, place = P.einet_sort(torch.randint(0, 5, (N, 2), generator=g, device="cuda", dtype=torch.int32), 5)
    print("dispatch and combine beyond 2^31 elements", flush=True)
    xs = P.einet_dispatch(x, place)
    assert xs.numel() > 2 ** 31
    for n in (0, 1, 262143, 262144, N - 2, N - 1):
        assert torch.equal(xs[place[n].long()], x[n].expand(2, H))
    at = torch.randint(0, N, (1000,), generator=g, device="cuda")
    assert torch.equal(xs[place[at].long().reshape(-1)], x[at].repeat_interleave(2, 0))
    half = torch.full((N, 2), 0.5, device="cuda")
    assert torch.equal(P.einet_combine(xs, place, half), x)
    d, dw = P.einet_combine_backward(x, xs, place, half)
    assert torch.equal(d[place[at].long().reshape(-1)], (x[at].float() * 0.5).bfloat16().repeat_interleave(2, 0))
    want = x[at].double().square().sum(1)
    assert bool(((dw[at].double() - want[:, None]).abs() <= U * (H / 64 + 82) * want[:, None]).all())
    del x, xs, d, place, half
    # logits: 70000 rows of 32768
    logits = torch.randn(70000, 32768, generator=g, device="cuda", dtype=torch.bfloat16)
    u = uniforms(np.random.default_rng(1), 70000)
    print("choose beyond 2^31 elements", flush=True)
    index, logq = P.einet_choose(logits, u, top_p=0.9)
    for lo, hi in ((0, 3), (65530, 65540), (69995, 70000)):
        i, q = P.einet_choose(logits[lo:hi].clone(), u[lo:hi].contiguous(), top_p=0.9)
        assert torch.equal(i, index[lo:hi]) and torch.equal(q, logq[lo:hi])
    del logits
    # scores: 64 components of 34 million samples
    scores = torch.randn(64, 34000001, generator=g, device="cuda")
    print("route beyond 2^31 elements", flush=True)
    ids, w, logp = P.einet_route(scores, None, 1)
    ds, dc = P.einet_route_backward(scores, None, ids, w, None, torch.ones_like(logp))
    at = torch.cat([torch.randint(0, scores.shape[1], (1000,), generator=g, device="cuda"), torch.tensor([0, scores.shape[1] - 1], device="cuda")])
    few = scores[:, at].double()
    assert torch.equal(ids[at, 0].long(), few.argmax(0))
    close(logp[at], host(few.logsumexp(0)), U * (host(few.logsumexp(0).abs()) + 96))
    p = host(few.softmax(0))
    close(ds[:, at], p, U * 120 * p)
    assert abs(float(dc.double().sum()) - scores.shape[1]) <= U * 400 * scores.shape[1]


def test_more_rows_than_a_launch_has_lanes_for():
    """A launch holds fewer than 2^32 lanes: rows that are one row over and over need little memory and more lanes than that."""
    B = 2 ** 26 + 5                                               # (64 lanes to a row)
    u = torch.zeros(B, device="cuda")
    tail = torch.tensor([0.0, 0.3, 0.6, 0.9, 0.99], device="cuda")
    u[-5:] = tail
    u[2 ** 26 - 16:2 ** 26 - 11] = tail
    for V in (3, 700):
        print("choose", B, V, flush=True)
        row = torch.linspace(-1.0, 1.0, V, device="cuda")
        index, logq = P.einet_choose(row.expand(B, V), u, top_p=0.95)
        few, share = P.einet_choose(row.expand(5, V), tail, top_p=0.95)
        for at in (slice(B - 5, B), slice(2 ** 26 - 16, 2 ** 26 - 11)):
            assert torch.equal(index[at], few) and torch.equal(logq[at], share)
        assert torch.equal(index[:2 ** 26 - 16], few[:1].expand(2 ** 26 - 16)) and torch.equal(index[2 ** 26 - 11:B - 5], few[:1].expand(11))
    B = 2 ** 24 + 5                                               # (256 lanes to a row)
    print("choose", B, 2000, flush=True)
    row = torch.linspace(-1.0, 1.0, 2000, device="cuda")
    index, logq = P.einet_choose(row.expand(B, 2000), u[-B:])
    few, share = P.einet_choose(row.expand(5, 2000), tail)
    assert torch.equal(index[-5:], few) and torch.equal(logq[-5:], share) and torch.equal(index[:5], few[:1].expand(5))
    del u, index, logq
    # scores of 1024 components: 64 lanes to a sample
    N = 2 ** 26 + 5
    print("route", N, flush=True)
    score = torch.linspace(-3.0, 2.0, 1024, device="cuda")
    ids, w, logp = P.einet_route(score[:, None].expand(1024, N), None, 1)
    assert bool((ids == 1023).all()) and bool((w == w[0, 0]).all()) and bool((logp == logp[0]).all())
    close(logp[-1:], [np.logaddexp.reduce(host(score))], U * 110)                  # (|logp| < 14)
    del ids, w, logp
    # rows: all samples are one row and few of them go anywhere
    for name, H, n in (("a wave to a row", 256, 2 ** 26 + 5), ("a workgroup to a row", 300, 2 ** 24 + 5)):
        print("rows,", name, n, flush=True)
        place = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
        went = torch.tensor([0, 1, 2 ** 24 - 5, 2 ** 24 - 4, 2 ** 24, n - 2, n - 1], device="cuda")
        place[went, 0] = torch.arange(7, dtype=torch.int32, device="cuda")
        x = torch.randn(1, H, device="cuda")
        out = torch.zeros(8, H, device="cuda")
        P.einet_dispatch(x.expand(n, H), place, out=out)
        assert torch.equal(out[:7], x.expand(7, H)) and not bool(out[7].any())
        weight = torch.full((n, 1), 2.0, device="cuda")
        d, dw = P.einet_combine_backward(x.expand(n, H), out, place, weight)
        assert torch.equal(d[:7], 2.0 * x.expand(7, H))
        want = float(x.double().square().sum())
        assert bool(((dw[went, 0].double() - want).abs() <= U * (H / 64 + 82) * want).all())
        assert int(dw.count_nonzero()) == 7


# ------------------------------------------------------------------------------------------------ choose, very long rows
#
# A row of more than 2^19 entries holds its weights as whole multiples of at most 1.5 * 2^-60 of their total Z (of the largest:
# 1): a weight is off by half of that, V of them by V 2^-60 of the total at most, so a log-share by U |logq| + 2^-36 + V 2^-60 (up to 2^19
# entries by V 2^-43, as above).  Among entries of weight W a running sum that is off by V 2^-60 Z is off by V 2^-60 Z / W entries, twice
# (the sum and the total), and by one where a quotient is rounded down.

def longest_tolerance(V, logq):
    return U * np.abs(logq) + 2.0 ** -36 + V * (2.0 ** -60 if V > 1 << 19 else 2.0 ** -43)


@pytest.mark.parametrize("V,dtype", [((1 << 19) + 1, "float32"), ((1 << 20) + 3, "float16"), ((1 << 23) + 1, "bfloat16"), ((1 << 26) + 5, "float32"),
                                     (1 << 30, "bfloat16")])
def test_choose_keeps_the_mass_of_many_small_weights(V, dtype):
    """One entry at 0, all others so far below it that each is less than half of 2^-(61 - ceil(log2 V)), together up to a fifth of
    the mass: their shares, and which of them a uniform falls on."""
    print("choose among many small weights", V, dtype, flush=True)
    level = -math.ceil((62 - (V - 1).bit_length()) * math.log(2.0) * 4 + 0.2) / 4       # (a multiple of 1/4 below 32: exact in every type)
    W, big = math.exp(level), V // 3
    Z = 1.0 + (V - 1) * W
    row = torch.full((1, V), level, device="cuda", dtype=TYPES[dtype])
    row[0, big] = 0.0
    u = np.array([0.0, 2.0 ** -27, 2.0 ** -25, 0.3, 0.5, 0.999, 1.0 - 2.0 ** -24], np.float32)
    index, logq = P.einet_choose(row.expand(len(u), V), torch.tensor(u).cuda())
    slack = 2 * V * 2.0 ** -60 * Z / W + 2
    for i, q, t in zip(host(index).tolist(), host(logq).tolist(), u.astype(np.float64) * Z):
        want = int(t / W) if t < big * W else big if t < big * W + 1.0 else big + 1 + int((t - big * W - 1.0) / W)
        assert 0 <= i < V and abs(i - want) <= (0 if want == big and i == big else slack), (i, want, slack)
        share = (0.0 if i == big else level) - math.log(Z)
        assert abs(q - share) <= longest_tolerance(V, share), (i, q, share)
    if V > 1 << 21:
        return
    # the cut of top_p among them (entries of one weight are kept from the lowest index on): the last kept entry
    p = float(np.float32(1.0 - 2.0 ** -24))
    kept = math.ceil((p * Z - 1.0) / W)
    index, _ = P.einet_choose(row, torch.ones(1, device="cuda"), top_p=p)
    want = kept - 1 if kept <= big else kept
    assert abs(int(index) - want) <= slack, (int(index), want)


@pytest.mark.parametrize("V", [(1 << 19), (1 << 19) + 1, (1 << 22) + 7])
def test_choose_from_very_long_rows_matches_the_formula(V):
    """Against sorted weights summed in 80-bit floats."""
    rng = np.random.default_rng(V)
    B = 3
    x = rng.normal(0, 3, (B, V)).astype(np.float32)
    x[1, rng.random(V) < 0.4] = -np.inf
    x[2] = -30.0 - 0.001 * np.abs(x[2])
    x[2, 12345] = 0.0
    dev = torch.tensor(x).cuda()
    u = uniforms(rng, B)
    for settings in (dict(), dict(temperature=0.7, top_k=300), dict(top_p=0.95), dict(min_p=1e-3), dict(temperature=1.5, top_p=0.999, min_p=1e-7), dict(top_k=5000)):
        print("choose", V, settings, flush=True)
        index, logq = P.einet_choose(dev, u, **settings)
        T, k, p, mp = (settings.get(n, d) for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)))
        T, p, mp = (float(np.float32(v)) for v in (T, p, mp))
        for b in range(B):
            left = np.flatnonzero(x[b] > -np.inf)
            left = left[np.argsort(-x[b][left], kind="stable")]
            if k > 0:
                left = left[:k]
            top = np.longdouble(x[b][left[0]])
            w = np.exp((x[b][left].astype(np.longdouble) - top) / np.longdouble(T))
            if p < 1:
                run = np.cumsum(w)
                n = 1 + int(np.count_nonzero(run[:-1] < np.longdouble(p) * run[-1]))
                left, w = left[:n], w[:n]
            left, w = left[w >= mp], w[w >= mp]
            back = np.argsort(left)
            left, w = left[back], w[back]
            run = np.cumsum(w)
            at = int(np.searchsorted(run, np.longdouble(float(u[b])) * run[-1], side="right"))
            assert int(index[b]) == left[at], (b, int(index[b]), int(left[at]))
            share = float(np.log(w[at] / run[-1]))
            assert abs(float(logq[b]) - share) <= longest_tolerance(V, share), (b, float(logq[b]), share)


def test_choose_from_very_long_rows_that_are_flat_empty_or_infinite():
    V = (1 << 19) + 3
    x = torch.zeros(5, V, device="cuda")
    x[1] = -math.inf
    x[2, 1::3] = math.inf
    x[3] = torch.finfo(torch.float32).min
    x[4, 77] = 1.0
    u = torch.tensor([0.75, 0.5, 0.5, 0.25, 0.5], device="cuda")
    t = torch.tensor([1.0, 1.0, 2.0, 0.5, 0.0], device="cuda")
    index, logq = P.einet_choose(x, u, temperature=t)
    n = (V + 1) // 3                                 # entries at 1, 4, 7, ...
    assert host(index).tolist() == [int(0.75 * V), -1, 1 + 3 * (n // 2), int(0.25 * V), 77]
    want = np.array([-math.log(V), -math.inf, -math.log(n), -math.log(V), 0.0])
    close(logq, want, longest_tolerance(V, np.where(np.isfinite(want), want, 0.0)))


def test_numbers_beyond_32_bits_are_not_cut():
    """C takes numbers of components, entries and choices as ints: one beyond is refused, and a top_k beyond keeps all."""
    dev = dict(device="cuda")
    column = torch.zeros(1, 3, **dev)
    with pytest.raises(AssertionError, match="32 bits"):
        P.einet_route(column.expand(2 ** 32 + 2, 3))
    with pytest.raises(AssertionError, match="32 bits"):
        P.einet_route(torch.zeros(4, 0, **dev), top=2 ** 32 + 1)
    with pytest.raises(AssertionError, match="32 bits"):
        P.einet_sort(torch.zeros(0, 1, dtype=torch.int32, **dev), 2 ** 32 + 1)
    with pytest.raises(AssertionError, match="32 bits"):
        P.einet_choose(torch.zeros(0, 2 ** 32 + 5, **dev), torch.zeros(0, **dev))
    with pytest.raises(AssertionError, match="32 bits"):
        P.einet_dispatch(torch.zeros(0, 2, **dev), torch.zeros(0, 2 ** 32 + 1, dtype=torch.int32, **dev))
    rng = np.random.default_rng(1)
    x, u = torch.tensor(rng.normal(0, 1, (50, 7)).astype(np.float32)).cuda(), uniforms(rng, 50)
    want = P.einet_choose(x, u)
    for k in (7, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 2 ** 63 - 1):
        assert all(torch.equal(a, b) for a, b in zip(P.einet_choose(x, u, top_k=k), want))
    for k in (-1, -2 ** 32, -2 ** 63):
        with pytest.raises(P.EinetError):
            P.einet_choose(x, u, top_k=k)


@pytest.mark.parametrize("M", [257, 512, 1024])
def test_captured_route_and_sort_of_many_components(M):
    """Kernels whose workgroups have more than 64 KiB of LDS (scores of 512 components through LDS, their gradient for 257 to 512 and
    1024, the sort of 1024), captured and replayed with eager work between."""
    print("captured", M, flush=True)
    N = 8200

    def all_of(scores, coef, dw, dl):
        ids, w, logp = P.einet_route(scores, coef, 2)
        ds, da = P.einet_route_backward(scores, coef, ids, w, dw, dl)
        return (ids, w, logp, ds, da) + P.einet_sort(ids, M)

    def fresh(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        return [torch.randn(*s, generator=g, device="cuda") for s in ((M, N), (M,), (N, 2), (N,))]

    state = fresh(0)
    all_of(*state)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = all_of(*state)
    for rep in range(3):
        for t, v in zip(state, fresh(rep + 1)):
            t.copy_(v)
        g.replay()
        torch.cuda.synchronize()
        want = all_of(*state)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {rep}"
    t = state[0].double() + state[1].double()[:, None]
    assert torch.equal(out[0][:, 0].long(), t.argmax(0))
    close(out[2], host(t.logsumexp(0)), U * (host(t.logsumexp(0).abs()) + 96))


def test_combine_of_more_rows_than_a_launch_has_lanes_for():
    """Sums of more rows than one launch of 2^32 lanes has a wave for (64 lanes to 264 float16): rows on both sides of the border
    between the launches, with weights and without, and zeros everywhere else."""
    H, n = 264, 2 ** 26 + 5
    border = (2 ** 32 - 1024) // 64
    print("combine", H, n, flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rows = torch.randn(9, H, generator=g, device="cuda").half()
    place = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
    went = torch.tensor([0, 1, border - 2, border - 1, border, border + 1, n - 3, n - 2, n - 1], device="cuda")
    place[went, 0] = torch.arange(9, dtype=torch.int32, device="cuda")
    weight = torch.zeros(n, 1, device="cuda")
    weight[went, 0] = 2.0
    out = torch.full((n, H), 7.0, dtype=torch.float16, device="cuda")
    for w in (weight, None):
        P.einet_combine(rows, place, w, out=out)
        assert torch.equal(out[went], rows * 2.0 if w is not None else rows)
        step = 2 ** 22
        assert sum(int(out[b:b + step].any(1).sum()) for b in range(0, n, step)) == 9
        out.fill_(7.0)


@pytest.mark.parametrize("V", [50, 1500, 6000, 20000, 600000])
def test_choose_at_the_ends_of_the_temperatures(V):
    """An infinite temperature makes all entries that take part equal (those at +inf, where there are any); the smallest one leaves
    the largest alone."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 4, (3, V)).astype(np.float32)
    x[1, ::2] = -np.inf
    x[2, 5::7] = np.inf
    u = np.array([0.6, 0.3, 0.7], np.float32)
    dev, du = torch.tensor(x).cuda(), torch.tensor(u).cuda()
    part = [np.flatnonzero(x[0] > -np.inf), np.flatnonzero(x[1] > -np.inf), np.flatnonzero(x[2] == np.inf)]
    for t in (math.inf, torch.full((3,), math.inf, device="cuda")):
        for k in (0, 4):
            print("choose, infinite temperature", V, k, flush=True)
            index, logq = P.einet_choose(dev, du, temperature=t, top_k=k)
            # (of equal weights the first top_k of the order: by logit, then by index)
            kept = [np.sort(p[np.argsort(-x[b][p], kind="stable")][:k]) if k else p for b, p in enumerate(part)]
            assert host(index).tolist() == [int(p[int(float(u[b]) * len(p))]) for b, p in enumerate(kept)]
            want = np.array([-math.log(len(p)) for p in kept])
            close(logq, want, longest_tolerance(V, want) + V * 2.0 ** -(62 - (V - 1).bit_length()) * (V <= 1 << 19))
    for t in (2.0 ** -149, torch.full((3,), 2.0 ** -149, device="cuda")):
        for settings in (dict(), dict(top_k=4), dict(top_p=0.5)):
            index, logq = P.einet_choose(dev[:2], du[:2], temperature=t if not torch.is_tensor(t) else t[:2], **settings)
            assert host(index).tolist() == x[:2].argmax(1).tolist() and not bool(logq.any())


@pytest.mark.parametrize("B,V", [(3, 3001), (3, 20000), (2, (1 << 19) + 5)])
def test_captured_choices_replay_on_new_logits(B, V):
    def fresh(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        return [torch.randn(B, V, generator=g, device="cuda") * 2, torch.rand(B, generator=g, device="cuda"),
                torch.randint(1, 900, (B,), generator=g, device="cuda", dtype=torch.int32)]

    def choices(x, u, k):
        return P.einet_choose(x, u) + P.einet_choose(x, u, top_p=0.9) + P.einet_choose(x, u, temperature=0.7, top_k=k, min_p=1e-4)

    state = fresh(0)
    choices(*state)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = choices(*state)
    for rep in range(3):
        for t, v in zip(state, fresh(rep + 1)):
            t.copy_(v)
        g.replay()
        torch.cuda.synchronize()
        want = choices(*state)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {rep}"
