"""What the routing operators refuse: every call returns before it touches a device, so these need none."""
import ctypes as C

import pytest
import torch

import paper_2004_06231_amd as P

X = C.c_void_p(4096)                    # an aligned address that no refused call reads
ODD = C.c_void_p(4097)
BIG = 1 << 31


def _refused(rc, *words):
    lib = P.load_library()
    assert rc == -1
    why = lib.einet_last_error(None).decode()
    assert all(w in why for w in words), why


def test_route_refusals():
    lib = P.load_library()

    def call(score=X, dtype=0, sc=8, sn=1, coef=None, M=4, n=8, top=2, ids=X, w=X, lp=X):
        return lib.einet_route(score, dtype, sc, sn, coef, M, n, top, 0, ids, w, lp, None)

    _refused(call(dtype=3), "einet_route", "dtype")
    for M in (0, -1, 1025):
        _refused(call(M=M), "n_components")
    for top in (0, 5, 17, -1):
        _refused(call(top=top), "top")
    _refused(call(M=64, top=17), "top")
    _refused(call(n=-1), "n must be")
    _refused(call(n=BIG // 2), "2^31")
    _refused(call(sc=-1), "strides")
    for name in ("score", "ids", "w", "lp"):
        _refused(call(**{name: None}), "NULL")
        _refused(call(**{name: ODD}), "aligned")
    _refused(call(coef=ODD), "aligned")
    assert call(n=0, score=None, ids=None, w=None, lp=None) == 0


def test_route_backward_refusals():
    lib = P.load_library()
    size = C.c_size_t()
    assert lib.einet_route_workspace(4, 800, C.byref(size)) == 0 and size.value > 0
    _refused(lib.einet_route_workspace(0, 8, C.byref(size)), "n_components")
    _refused(lib.einet_route_workspace(4, 8, None), "bytes")

    def call(score=X, M=4, n=800, top=2, ids=X, w=X, dw=X, dl=X, ds=X, dsc=8, dsn=1, da=X, ws=X, size=size.value):
        return lib.einet_route_backward(score, 0, 8, 1, None, M, n, top, 0, ids, w, dw, dl, ds, dsc, dsn, da, ws, size, None)

    _refused(call(M=0), "n_components")
    _refused(call(top=5), "top")
    _refused(call(dsn=-1), "strides")
    for name in ("score", "ids", "w", "ds"):
        _refused(call(**{name: None}), "NULL")
        _refused(call(**{name: ODD}), "aligned")
    _refused(call(ws=None), "workspace")
    _refused(call(size=size.value - 1), "workspace")
    _refused(call(ws=C.c_void_p(4100)), "workspace")


def test_sort_refusals():
    lib = P.load_library()
    size = C.c_size_t()
    assert lib.einet_sort_workspace(100, 8, C.byref(size)) == 0
    _refused(lib.einet_sort_workspace(-1, 8, C.byref(size)), "n_slots")
    _refused(lib.einet_sort_workspace(BIG, 8, C.byref(size)), "n_slots")

    def call(ids=X, n=100, M=8, first=X, place=X):
        return lib.einet_sort(ids, n, M, first, place, X, size.value, None)

    for M in (0, 1025):
        _refused(call(M=M), "n_components")
    for n in (-1, BIG):
        _refused(call(n=n), "n_slots")
    for name in ("ids", "first", "place"):
        _refused(call(**{name: None}), "NULL")
        _refused(call(**{name: ODD}), "aligned")


def test_row_refusals():
    lib = P.load_library()

    def dispatch(x=X, width=64, stride=64, n=4, top=2, place=X, out=X, out_stride=64, rows=8):
        return lib.einet_dispatch(x, width, stride, n, top, place, out, out_stride, rows, None)

    def combine(rows=X, dtype=0, width=16, stride=16, m=8, place=X, w=X, n=4, top=2, out=X, out_stride=16):
        return lib.einet_combine(rows, dtype, width, stride, m, place, w, n, top, out, out_stride, None)

    def backward(g=X, rows=X, dtype=0, width=16, m=8, place=X, w=X, n=4, top=2, out=X, out_stride=16, dw=X):
        return lib.einet_combine_backward(g, 16, rows, dtype, width, 16, m, place, w, n, top, out, out_stride, dw, None)

    for call in (dispatch, combine, backward):
        _refused(call(top=0), "top")
        _refused(call(n=-1), "n must")
        _refused(call(n=BIG // 2), "2^31")
        _refused(call(width=-1), "negative")
        _refused(call(out_stride=15), "overlap")
        _refused(call(place=None), "NULL")
        _refused(call(out=None), "NULL")
        _refused(call(place=ODD), "aligned")
        assert call(n=0) == 0
    _refused(dispatch(rows=-1), "sorted rows")
    _refused(dispatch(x=None), "NULL")
    for call in (combine, backward):
        _refused(call(m=-1), "sorted rows")
        _refused(call(dtype=9), "dtype")
        _refused(call(rows=None), "NULL")
        _refused(call(out=ODD), "aligned")
        _refused(call(w=ODD), "aligned")
    _refused(backward(w=None), "NULL")
    _refused(backward(dw=None), "NULL")
    _refused(backward(g=None), "NULL")


def test_choose_refusals():
    lib = P.load_library()
    size = C.c_size_t()
    _refused(lib.einet_choose_workspace(-1, 8, C.byref(size)), "n_rows")
    _refused(lib.einet_choose_workspace(1, 0, C.byref(size)), "n_entries")
    assert lib.einet_choose_workspace(1, 300000, C.byref(size)) == 0
    need = size.value

    def call(x=X, dtype=0, stride=300000, n=1, V=300000, u=X, tp=None, t=1.0, kp=None, k=0, pp=None, p=1.0, mp=None, m=0.0, index=X,
             logq=X, ws=X, size=need):
        return lib.einet_choose(x, dtype, stride, n, V, u, tp, t, kp, k, pp, p, mp, m, index, logq, ws, size, None)

    nan = float("nan")
    _refused(call(dtype=-1), "dtype")
    _refused(call(n=-1), "n_rows")
    for V in (0, (1 << 30) + 1):
        _refused(call(V=V), "n_entries")
    _refused(call(stride=-1), "row_stride")
    for t in (-0.5, nan):
        _refused(call(t=t), "temperature")
    _refused(call(k=-1), "top_k")
    for v in (-0.1, 1.5, nan):
        _refused(call(p=v), "top_p")
        _refused(call(m=v), "min_p")
    for name in ("x", "u", "index"):
        _refused(call(**{name: None}), "NULL")
        _refused(call(**{name: ODD}), "aligned")
    for name in ("tp", "kp", "pp", "mp", "logq"):
        _refused(call(**{name: ODD}), "aligned")
    if need:
        _refused(call(ws=None), "workspace")
        _refused(call(size=need - 1), "workspace")
        _refused(call(ws=C.c_void_p(4112)), "workspace")
    assert call(n=0) == 0


def test_binding_takes_no_tensors_of_the_host():
    x, place = torch.zeros(4, 3), torch.zeros(4, 1, dtype=torch.int32)
    for call in (lambda: P.einet_route(x), lambda: P.einet_route_backward(x, None, None, None), lambda: P.einet_sort(place, 3),
                 lambda: P.einet_dispatch(x, place), lambda: P.einet_combine(x, place),
                 lambda: P.einet_combine_backward(x, x, place, torch.ones(4, 1)), lambda: P.einet_choose(x, torch.zeros(4))):
        with pytest.raises(AssertionError):
            call()


def test_rows_too_long_for_a_launch_are_refused():
    lib = P.load_library()
    for width in ((1 << 35) + 1, 1 << 62):
        _refused(lib.einet_dispatch(X, width, 0, 4, 2, X, X, width, 8, None), "einet_dispatch", "2^35")
    for dtype, most in ((0, 1 << 33), (1, 1 << 34), (2, 1 << 34)):
        for width in (most + 1, 1 << 61):
            _refused(lib.einet_combine(X, dtype, width, 0, 8, X, X, 4, 2, X, width, None), "einet_combine", "2^35")
            _refused(lib.einet_combine_backward(X, 0, X, dtype, width, 0, 8, X, X, 4, 2, X, width, X, None), "2^35")


def test_every_thread_reads_the_reason_of_its_own_refusal():
    """Calls without a handle may be refused in several threads at once: nobody reads another call's reason."""
    import threading
    lib = P.load_library()
    calls = [(lambda: lib.einet_route(X, 9, 8, 1, None, 4, 8, 2, 0, X, X, X, None), b"einet_route: unknown dtype"),
             (lambda: lib.einet_choose(X, 0, 8, -1, 8, X, None, 1.0, None, 0, None, 1.0, None, 0.0, X, X, X, 0, None),
              b"einet_choose: n_rows must be at least 0 and n_entries in 1..EINET_CHOOSE_MAX_ENTRIES"),
             (lambda: lib.einet_sort(X, 8, 0, X, X, X, 0, None), b"einet_sort: n_components must be in 1..EINET_ROUTE_MAX_COMPONENTS"),
             (lambda: lib.einet_dispatch(X, 64, 64, 4, 0, X, X, 64, 8, None), b"einet_dispatch: top must be at least 1")]
    wrong = []
    start = threading.Barrier(len(calls))

    def refused(call, reason):
        start.wait()
        for _ in range(20000):
            call()
            got = lib.einet_last_error(None)
            if got != reason:
                wrong.append((reason, got))
                return

    threads = [threading.Thread(target=refused, args=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
