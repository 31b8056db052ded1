"""What the calls on rows by index refuse, before anything is enqueued: no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2511_10442_amd import binding as B

N = 2147418112          # FG_MAX_N
BF16, F32 = B.FG_BF16, B.FG_F32


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def sizes(fn, *args):
    out = ctypes.c_size_t(77)
    return fn(*args, ctypes.byref(out)), out.value


def test_index_sort(lib):
    f, need = lib.fg_index_sort, lib.fg_index_sort_workspace_size
    assert need(10, 10, None) == B.FG_ERR_NULL
    for m, n in [(-1, 5), (5, -1), (N + 1, 5), (5, N + 1), (2 ** 40, 5)]:
        assert sizes(need, m, n)[0] == B.FG_ERR_BAD_SHAPE
        assert f(8, m, n, 8, 8, 8, 256, 1 << 50, None) == B.FG_ERR_BAD_SHAPE
    assert sizes(need, N, N)[0] == B.FG_OK and sizes(need, N, N)[1] > 4 * 4 * N
    assert f(None, 10, 5, 8, 8, 8, 256, 1 << 30, None) == B.FG_ERR_NULL
    assert f(8, 10, 5, None, 8, 8, 256, 1 << 30, None) == B.FG_ERR_NULL
    assert f(8, 10, 5, 8, 8, None, 256, 1 << 30, None) == B.FG_ERR_NULL
    assert f(None, 0, 5, None, None, None, None, 0, None) == B.FG_ERR_NULL
    enough = sizes(need, 100000, 5000)[1]
    assert f(8, 100000, 5000, 8, 8, 8, None, 0, None) == B.FG_ERR_WORKSPACE
    assert f(8, 100000, 5000, 8, 8, 8, 256, enough // 2, None) == B.FG_ERR_WORKSPACE
    assert f(8, 100000, 5000, 8, 8, 8, 257, enough * 2, None) == B.FG_ERR_WORKSPACE


def test_lookup(lib):
    f = lib.fg_lookup
    ok = dict(table=256, type=BF16, n=5, c=8, ts=8, index=8, m=3, scale=1.0, out=512, os=8)
    call = lambda **k: f(*dict(ok, **k).values(), None)      # noqa: E731
    assert call(type=3) == call(type=-1) == B.FG_ERR_UNSUPPORTED
    assert call(c=0) == call(c=-3) == call(c=(1 << 18) + 1) == B.FG_ERR_BAD_SHAPE
    assert call(ts=-8) == call(ts=(1 << 29) + 1) == call(os=7) == call(os=0) == call(os=(1 << 29) + 1) == B.FG_ERR_BAD_SHAPE
    assert call(m=-1) == call(m=N + 1) == call(n=-1) == call(n=N + 1) == B.FG_ERR_BAD_SHAPE
    assert call(table=None) == call(index=None) == call(out=None) == B.FG_ERR_NULL
    assert call(table=257) == call(out=513) == call(type=F32, table=258) == B.FG_ERR_UNSUPPORTED
    assert call(m=0, table=None, index=None, out=None) == B.FG_OK


def test_lookup_backward(lib):
    f, need = lib.fg_lookup_backward, lib.fg_lookup_backward_workspace_size
    assert need(10, 5, 8, BF16, None) == B.FG_ERR_NULL
    assert sizes(need, 10, 5, 8, 5)[0] == B.FG_ERR_UNSUPPORTED
    assert sizes(need, 10, 5, 0, BF16)[0] == sizes(need, -1, 5, 8, BF16)[0] == sizes(need, N + 1, 5, 8, BF16)[0] == sizes(need, 10, -1, 8, BF16)[0] == B.FG_ERR_BAD_SHAPE
    assert sizes(need, 1024, 5000, 512, BF16) == (B.FG_OK, 0) and sizes(need, 1025, 5000, 512, BF16)[1] >= 32 * 512 * 4
    ok = dict(grad=256, type=BF16, m=10000, c=8, gs=8, index=8, order=8, bounds=8, n=5, scale=1.0, acc=0, to=256, gt=F32, ts=8, ws=256, bytes=1 << 30)
    call = lambda **k: f(*dict(ok, **k).values(), None)      # noqa: E731
    assert call(type=7) == call(gt=B.FG_F16) == call(type=F32, gt=BF16) == B.FG_ERR_UNSUPPORTED
    assert call(c=0) == call(gs=-1) == call(ts=7) == call(m=-1) == call(n=-1) == call(n=N + 1) == B.FG_ERR_BAD_SHAPE
    assert call(grad=None) == call(index=None) == call(order=None) == call(bounds=None) == call(to=None) == B.FG_ERR_NULL
    assert call(grad=257) == call(to=258) == B.FG_ERR_UNSUPPORTED
    assert call(ws=None) == call(ws=264) == call(bytes=16) == B.FG_ERR_WORKSPACE
    assert call(n=0) == B.FG_OK


def test_dispatch(lib):
    f = lib.fg_dispatch
    ok = dict(x=256, type=BF16, t=5, c=8, xs=8, place=8, k=2, n=10, out=256, os=8)
    call = lambda **k: f(*dict(ok, **k).values(), None)      # noqa: E731
    assert call(type=9) == call(x=257) == call(out=257) == B.FG_ERR_UNSUPPORTED
    assert call(c=0) == call(xs=-1) == call(os=7) == call(t=-1) == call(k=0) == call(k=129) == call(n=-1) == B.FG_ERR_BAD_SHAPE
    assert call(t=N, k=2) == call(t=N // 2 + 1, k=2) == B.FG_ERR_BAD_SHAPE
    assert call(x=None) == call(place=None) == call(out=None) == B.FG_ERR_NULL
    assert call(t=0) == call(n=0) == B.FG_OK


def test_combine(lib):
    f = lib.fg_combine
    ok = dict(rows=256, type=BF16, n=10, c=8, rs=8, index=8, w=8, t=5, k=2, walk=None, out=256, os=8)
    call = lambda **k: f(*dict(ok, **k).values(), None)      # noqa: E731
    assert call(type=9) == call(rows=257) == call(out=257) == B.FG_ERR_UNSUPPORTED
    assert call(c=0) == call(rs=-1) == call(os=7) == call(t=-1) == call(k=0) == call(k=129) == call(n=-1) == call(t=N, k=2) == B.FG_ERR_BAD_SHAPE
    assert call(rows=None) == call(index=None) == call(out=None) == B.FG_ERR_NULL
    assert call(t=0) == B.FG_OK


def test_combine_backward(lib):
    f, need = lib.fg_combine_backward, lib.fg_combine_backward_workspace_size
    assert need(10, 2, 9, 8, BF16, None) == B.FG_ERR_NULL
    assert sizes(need, 10, 2, 9, 8, 5)[0] == B.FG_ERR_UNSUPPORTED
    assert sizes(need, 10, 0, 9, 8, BF16)[0] == sizes(need, N, 2, 9, 8, BF16)[0] == sizes(need, 10, 2, 9, 0, BF16)[0] == sizes(need, 10, 2, -1, 8, BF16)[0] == B.FG_ERR_BAD_SHAPE
    ok = dict(grad=256, type=BF16, t=500, c=8, gs=8, rows=256, n=10, rs=8, index=8, w=8, k=2, order=8, bounds=8, walk=None, gr=256, grs=8, gw=8, ws=256, bytes=1 << 30)
    call = lambda **k: f(*dict(ok, **k).values(), None)      # noqa: E731
    assert call(type=9) == call(grad=257) == call(rows=257) == call(gr=257) == B.FG_ERR_UNSUPPORTED
    assert call(c=0) == call(gs=-1) == call(rs=-1) == call(grs=7) == call(t=-1) == call(k=0) == call(k=129) == call(n=-1) == B.FG_ERR_BAD_SHAPE
    assert call(grad=None) == call(rows=None) == call(index=None) == call(order=None) == call(bounds=None) == B.FG_ERR_NULL
    assert call(ws=None) == call(ws=264) == call(bytes=16) == B.FG_ERR_WORKSPACE
    assert call(gr=None, gw=None) == B.FG_OK
    assert call(t=0, n=0) == call(t=0, order=None, bounds=None) == B.FG_OK


def test_sizes_of_types_that_there_are_not():
    for size in (lambda: B.fg_lookup_backward_workspace_size(5, 5, 5, torch.float64), lambda: B.fg_combine_backward_workspace_size(5, 5, 5, 5, torch.int32)):
        with pytest.raises(B.FgError):
            size()


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    i, x = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 8))
    by = B.IndexSort(i, 4, torch.zeros(8 + 5 + 8, dtype=torch.int32), True)
    for call in (lambda: B.fg_index_sort(i, 4), lambda: B.fg_lookup(x, i), lambda: B.fg_lookup_backward(torch.zeros((8, 8)), by),
                 lambda: B.fg_dispatch(x, i), lambda: B.fg_combine(x, i), lambda: B.fg_combine_backward(x, x, i)):
        with pytest.raises(ValueError):
            call()


def test_pointers_that_int32_and_float32_may_not_have(lib):
    """Indexes, orders, bounds and weights between two elements' places are refused as rows are"""
    bad = lambda f, args, names: [n for n in names if f(*dict(args, **{n: args[n] + 2}).values(), None) != B.FG_ERR_UNSUPPORTED]      # noqa: E731
    sort = dict(index=8, m=100000, n=5000, order=8, place=8, bounds=8, ws=256, bytes=1 << 30)
    assert not bad(lib.fg_index_sort, sort, ["index", "order", "place", "bounds"])
    look = dict(table=256, type=BF16, n=5, c=8, ts=8, index=8, m=3, scale=1.0, out=512, os=8)
    assert not bad(lib.fg_lookup, look, ["index"])
    back = dict(grad=256, type=BF16, m=10000, c=8, gs=8, index=8, order=8, bounds=8, n=5, scale=1.0, acc=0, to=256, gt=BF16, ts=8, ws=256, bytes=1 << 30)
    assert not bad(lib.fg_lookup_backward, back, ["index", "order", "bounds"])
    send = dict(x=256, type=BF16, t=5, c=8, xs=8, place=8, k=2, n=10, out=256, os=8)
    assert not bad(lib.fg_dispatch, send, ["place"])
    take = dict(rows=256, type=BF16, n=10, c=8, rs=8, index=8, w=8, t=5, k=2, walk=8, out=256, os=8)
    assert not bad(lib.fg_combine, take, ["index", "w", "walk"])
    grads = dict(grad=256, type=BF16, t=500, c=8, gs=8, rows=256, n=10, rs=8, index=8, w=8, k=2, order=8, bounds=8, walk=8, gr=256, grs=8, gw=8, ws=256, bytes=1 << 30)
    assert not bad(lib.fg_combine_backward, grads, ["index", "w", "order", "bounds", "walk", "gw"])
