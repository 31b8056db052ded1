"""Rows by index on the GPU: sort by index, lookup, expert order, weighted sums and all gradients against plain sums in 64 bits."""
import numpy as np
import pytest
import torch

import rows_oracle as R
from paper_2511_10442_amd import binding as B
from paper_2511_10442_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def values(rng, n, c, dtype):
    return dev(rng.standard_normal((n, c)).astype(np.float32)).to(dtype)


def some_index(rng, shape, n_rows, kind="uniform"):
    """int32; a few entries name no row, in all the ways there are"""
    n = int(np.prod(shape))
    if kind == "one":
        index = np.full(n, n_rows // 2)
    elif kind == "frequent":
        index = np.minimum((n_rows + 1.0) ** rng.random(n), n_rows).astype(np.int64) - 1
    else:
        index = rng.integers(0, max(1, n_rows), size=n)
    none = rng.random(n) < 0.1
    index = np.where(none, rng.choice([-1, n_rows, -2 ** 31, 2 ** 31 - 1], size=n), index)
    return index.astype(np.int32).reshape(shape)


# ---- sort --------------------------------------------------------------------------------------------------------------

def check_sort(index, n_rows, **kw):
    got = B.fg_index_sort(dev(index), n_rows, **kw)
    order, bounds, place = R.sort(index, n_rows)
    assert np.array_equal(got.order.cpu().numpy(), order)
    assert np.array_equal(got.bounds.cpu().numpy(), bounds)
    if kw.get("place", True):
        assert got.place.shape == index.shape and np.array_equal(got.place.cpu().numpy(), place)
    else:
        assert got.place is None


# counted by 4 lanes and by 16, one workgroup with 1, 4 and 8 entries a lane, many workgroups with 4; bounds from the keys, from the digits, by search
@pytest.mark.parametrize("m", [0, 1, 63, 64, 65, 256, 257, 512, 513, 1024, 1025, 4096, 4097, 8192, 8193, 20011])
@pytest.mark.parametrize("n_rows", [0, 1, 2, 7, 64, 1000, 1023, 1024, 4096, 4097, 12287, 12288, 31743, 31744, 70001, 261631, 261632])
def test_sort(m, n_rows):
    rng = np.random.default_rng(m * 31 + n_rows)
    for kind in ("uniform", "one", "frequent"):
        check_sort(some_index(rng, (m,), n_rows, kind), n_rows)


@pytest.mark.parametrize("m,n_rows", [(1048576, 300), (1048577, 300), (1200003, 100003), (30000, 1048575), (30000, 1048576), (1300000, 1300000),
                                      (32768, 1023), (32769, 1023), (65536, 131072), (65537, 131072), (131072, 2047), (262144, 127), (262145, 127), (262145, 8), (700000, 40000)])
def test_sort_many(m, n_rows):
    rng = np.random.default_rng(m)
    check_sort(some_index(rng, (m,), n_rows, "frequent"), n_rows)
    check_sort(some_index(rng, (m,), n_rows), n_rows, place=False)


def test_sort_keeps_shape_and_takes_a_workspace():
    rng = np.random.default_rng(5)
    ws = torch.full((B.fg_index_sort_workspace_size(30000, 5000),), 0xee, dtype=torch.uint8, device=DEV)
    check_sort(some_index(rng, (10000, 3), 5000), 5000, workspace=ws)
    check_sort(some_index(rng, (5, 4, 3), 60), 60)


def test_sort_of_four_digits():
    """Row numbers up to 2^30 and more; the bounds, 4 GB, are looked at in samples"""
    n_rows, m = (1 << 30) + 5, 20000
    rng = np.random.default_rng(9)
    index = some_index(rng, (m,), n_rows)
    got = B.fg_index_sort(dev(index), n_rows)
    key = np.where(R.names(index.astype(np.int64), n_rows), index, n_rows)
    order = np.lexsort((np.arange(m), key))
    assert np.array_equal(got.order.cpu().numpy(), order)
    at = np.unique(np.concatenate([[0, 1, n_rows - 1, n_rows], key, np.minimum(key + 1, n_rows), rng.integers(0, n_rows, size=1000)]))
    assert np.array_equal(got.bounds[dev(at)].cpu().numpy(), np.searchsorted(key[order], at))


# ---- lookup ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 2, 3, 7, 8, 9, 64, 257, 1000, 4099])
def test_lookup(c, dtype):
    rng = np.random.default_rng(c)
    for m, n_rows, scale in [(1, 1, 1.0), (65, 7, -3.5), (1001, 4003, 64.0)]:
        table, index = values(rng, n_rows, c, dtype), some_index(rng, (m,), n_rows)
        ref = R.lookup(R.wide(table), index, scale)
        R.check(B.fg_lookup(table, dev(index), scale), ref, abs(ref), 0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_lookup_many(dtype):
    """Enough pieces of rows for several to a lane, the last turn not full"""
    rng = np.random.default_rng(3)
    c = 999
    m = 1024 * 256 * 4 * (16 // torch.empty((), dtype=dtype).element_size()) // c + 77
    table, index = values(rng, 5001, c, dtype), some_index(rng, (m,), 5001)
    got = B.fg_lookup(table, dev(index), 0.3)
    at = dev(index).long()
    ref = torch.where(((at >= 0) & (at < 5001))[:, None], table.double()[at.clamp(0, 5000)] * float(np.float32(0.3)), 0.0)
    assert bool(((got.double() - ref).abs() <= (2.0 ** -24 + R.STEP[dtype]) * 1.01 * ref.abs() + R.LEAST[dtype]).all())


def test_lookup_of_nothing():
    assert B.fg_lookup(torch.zeros((5, 8), device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV)).shape == (0, 8)
    got = B.fg_lookup(torch.zeros((0, 8), device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV))
    assert got.shape == (3, 8) and not bool(got.any())
    # entries that name no row give zeros whatever the scale, and read nothing
    table = torch.full((4, 9), float("nan"), device=DEV)
    got = B.fg_lookup(table, dev(np.array([-1, 2, 4], dtype=np.int32)), float("inf"))
    assert not bool(got[[0, 2]].any()) and bool(got[1].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows_and_what_lies_between(dtype):
    """Rows as parts of wider ones, at odd elements, for every operator: what lies between the rows stays as it was"""
    rng = np.random.default_rng(8)
    t, k, n, c, wide = 37, 3, 50, 21, 29
    index = some_index(rng, (t, k), n)
    w = dev(rng.random((t, k)).astype(np.float32))
    part = slice(5, 5 + c)

    def place_for(rows, like=None):
        whole = torch.full((rows, wide), 7.0, dtype=dtype, device=DEV)
        return whole, whole[:, part]

    def between(whole):
        whole = whole.clone()
        whole[:, part] = 7.0
        return bool((whole == 7.0).all())
    table = values(rng, n, wide, dtype)[:, part]
    grad = values(rng, t, wide, dtype)[:, part]
    flat = dev(index.reshape(-1))
    whole, out = place_for(t * k)
    ref = R.lookup(R.wide(table), index.reshape(-1), 2.0)
    R.check(B.fg_lookup(table, flat, 2.0, out=out), ref, abs(ref), 0, dtype)
    assert between(whole)
    whole, out = place_for(t)
    ref, mass = R.combine(R.wide(table), index, R.wide(w))
    R.check(B.fg_combine(table, dev(index), w, out=out), ref, mass, k, dtype)
    assert between(whole)
    whole, out = place_for(n)
    by = B.fg_index_sort(dev(index), n)
    ref, mass, count = R.row_sums(R.wide(grad), index, R.wide(w), n)
    got, gw = B.fg_combine_backward(grad, table, dev(index), w, sort=by, grad_rows=out)
    R.check(got, ref, mass, count[:, None], dtype)
    R.check(gw, *R.dots(R.wide(grad), R.wide(table), index), c, torch.float32)
    assert between(whole)
    whole, out = place_for(t * k)
    B.fg_dispatch(grad, by.place, out)
    ref = np.full((t * k, c), 7.0)
    for (i, j), p in np.ndenumerate(by.place.cpu().numpy()):
        if p >= 0:
            ref[p] = R.wide(grad)[i]
    assert np.array_equal(R.wide(out), ref) and between(whole)
    # a gradient that is one row for all (a mean's, a sum's)
    one = values(rng, 1, c, dtype)
    ref, mass, count = R.row_sums(np.repeat(R.wide(one), t * k, 0), index, None, n)
    R.check(B.fg_lookup_backward(one.expand(t * k, c), B.fg_index_sort(flat, n)), ref, mass, count[:, None], dtype)


# ---- the lookup's gradient ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "one", "frequent"])
@pytest.mark.parametrize("m,n_rows,c", [(0, 5, 8), (1, 1, 1), (64, 3, 9), (127, 2, 40), (129, 1, 3), (1000, 700, 257), (1024, 128, 70), (1025, 4000, 24), (900, 300, 5), (9001, 40, 100), (5000, 9000, 36)])
def test_lookup_backward(m, n_rows, c, kind, dtype):
    rng = np.random.default_rng(m + n_rows + c)
    index, grad = some_index(rng, (m,), n_rows, kind), values(rng, m, c, dtype)
    by = B.fg_index_sort(dev(index), n_rows)
    ref, mass, count = R.row_sums(R.wide(grad), index, None, n_rows, 0.7)
    for out in {dtype, torch.float32}:
        got = B.fg_lookup_backward(grad, by, 0.7, dtype=out)
        assert got.dtype == out
        R.check(got, ref, mass, count[:, None], out)
        assert torch.equal(got, B.fg_lookup_backward(grad, by, 0.7, dtype=out))                  # the same bits again
        there = values(rng, n_rows, c, out)
        was = there.clone()
        B.fg_lookup_backward(grad, by, 0.7, grad_table=there, accumulate=True)
        R.check(there, ref + R.wide(was), mass + abs(R.wide(was)), count[:, None] + 1, out)
        assert torch.equal(there[dev(count == 0)], was[dev(count == 0)])


def test_rows_that_begin_and_end_around_chunks():
    """Rows of 1 to 200 entries one after the other: every way in which one lies over 64 entries of the order"""
    rng = np.random.default_rng(2)
    index = np.repeat(np.arange(150), rng.integers(1, 200, size=150)).astype(np.int32)
    index = np.concatenate([index[rng.permutation(index.size)], np.full(300, -1, dtype=np.int32)])
    grad = values(rng, index.size, 12, torch.float32)
    ref, mass, count = R.row_sums(R.wide(grad), index, None, 150)
    R.check(B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 150)), ref, mass, count[:, None], torch.float32)


def test_one_row_named_by_many():
    """Half a million entries of one row and a few of its neighbours"""
    rng = np.random.default_rng(4)
    m = 500_003
    index = np.full(m, 3, dtype=np.int32)
    index[rng.integers(0, m, size=100)] = rng.integers(0, 7, size=100)
    grad = values(rng, m, 8, torch.bfloat16)
    ref, mass, count = R.row_sums(R.wide(grad), index, None, 7)
    got = B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 7), dtype=torch.float32)
    R.check(got, ref, mass, count[:, None], torch.float32)


def test_a_row_of_five_million_entries():
    """Enough for larger chunks: those of a row are added up by one lane"""
    rng = np.random.default_rng(11)
    m = 5_000_011
    index = np.full(m, 1, dtype=np.int32)
    index[:70] = 0
    index[-5:] = -1
    grad = values(rng, m, 4, torch.float16)
    got = B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 3), dtype=torch.float32)
    wide = R.wide(grad)
    ref = np.stack([wide[:70].sum(0), wide[70:-5].sum(0), np.zeros(4)])
    mass = np.stack([abs(wide[:70]).sum(0), abs(wide[70:-5]).sum(0), np.zeros(4)])
    # no sum here is longer than some 5000 terms in a row (a chunk, the chunks of one, those): far fewer roundings than entries
    R.check(got, ref, mass, 5000, torch.float32)


@pytest.mark.parametrize("m,n_rows,c", [(20, 40, 64), (5000, 9000, 33), (5000, 9000, 1024)])
@pytest.mark.parametrize("scale", [float("inf"), float("nan")])
def test_a_scale_that_is_not_finite_leaves_rows_without_entries_zero(m, n_rows, c, scale):
    index = dev(np.arange(m, dtype=np.int32) * 2 % n_rows // 4)
    grad = torch.ones((m, c), device=DEV)
    got = B.fg_lookup_backward(grad, B.fg_index_sort(index, n_rows), scale)
    named = torch.zeros(n_rows, dtype=torch.bool, device=DEV)
    named[index.long()] = True
    assert bool((got[~named] == 0).all()) and not bool(torch.isfinite(got[named]).any())
    index[::3] = -1
    got = B.fg_lookup(grad, index, scale)
    assert bool((got[index < 0] == 0).all()) and not bool(torch.isfinite(got[(index >= 0) & (index < m)]).any())


def test_what_is_not_finite_stays_in_its_row():
    rng = np.random.default_rng(6)
    index = some_index(rng, (400,), 20)
    index[:3] = [4, -1, 20]
    grad = values(rng, 400, 10, torch.float32)
    grad[0], grad[1], grad[2] = float("nan"), float("inf"), float("nan")
    got = B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 20))
    assert bool(got[4].isnan().all()) and bool(torch.cat([got[:4], got[5:]]).isfinite().all())
    # weights and rows of entries that name nothing
    rows = values(rng, 20, 10, torch.float32)
    at = dev(np.array([[1, -1], [-1, 20]], dtype=np.int32))
    w = dev(np.array([[2.0, np.nan], [np.inf, 1.0]], dtype=np.float32))
    got = B.fg_combine(rows, at, w)
    assert torch.equal(got[0], rows[1] * 2) and not bool(got[1].any())
    g = values(rng, 2, 10, torch.float32)
    g[1] = float("nan")
    for by in (None, B.fg_index_sort(at, 20)):
        grad_rows, grad_w = B.fg_combine_backward(g, rows, at, w, sort=by)
        assert torch.equal(grad_rows[1], g[0] * 2) and not bool(grad_rows[0].any()) and not bool(grad_rows[2:].any())
        assert bool(grad_w.isfinite().all()) and not bool(grad_w.reshape(-1)[1:].any())


# ---- expert order and back ---------------------------------------------------------------------------------------------

def choices(rng, t, k, experts, drop):
    index = np.argsort(rng.random((t, experts)) - 0.3 * rng.random(experts), axis=1)[:, :k].astype(np.int32)
    index[rng.random((t, k)) < drop] = -1
    return index


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,k,experts,c", [(1, 1, 1, 5), (3, 2, 4, 64), (33, 8, 16, 1000), (2500, 3, 10, 129), (70, 9, 64, 8200), (2100, 17, 20, 6)])
def test_to_experts_and_back(t, k, experts, c, dtype):
    rng = np.random.default_rng(t + k + c)
    for drop in (0.0, 0.3):
        index = choices(rng, t, k, experts, drop)
        x, w = values(rng, t, c, dtype), dev(rng.random((t, k)).astype(np.float32))
        by = B.fg_index_sort(dev(index), experts)
        order, bounds, place = R.sort(index, experts)
        assert np.array_equal(by.place.cpu().numpy(), place) and np.array_equal(by.bounds.cpu().numpy(), bounds)
        sent = torch.full((t * k, c), 7.0, dtype=dtype, device=DEV)
        B.fg_dispatch(x, by.place, sent)
        kept = bounds[-1]
        assert torch.equal(sent[:kept], x[dev(order[:kept] // k)]) and bool((sent[kept:] == 7.0).all())
        rows = values(rng, t * k, c, dtype)
        ref, mass = R.combine(R.wide(rows), place, R.wide(w))
        R.check(B.fg_combine(rows, by.place, w), ref, mass, k, dtype)
        ref, mass = R.combine(R.wide(rows), place, None)                     # the gradient of dispatch
        R.check(B.fg_combine(rows, by.place), ref, mass, k, dtype)
        grad = values(rng, t, c, dtype)
        ref, mass, count = R.row_sums(R.wide(grad), place, R.wide(w), t * k)
        grad_rows, grad_w = B.fg_combine_backward(grad, rows, by.place, w)
        R.check(grad_rows, ref, mass, count[:, None], dtype)
        R.check(grad_w, *R.dots(R.wide(grad), R.wide(rows), place), c, torch.float32)
        kept_rows = torch.full((t * k, c), 7.0, dtype=dtype, device=DEV)
        B.fg_combine_backward(grad, rows, by.place, w, grad_rows=kept_rows)
        assert torch.equal(kept_rows[:kept], grad_rows[:kept]) and bool((kept_rows[kept:] == 7.0).all())
        alone, none = B.fg_combine_backward(grad, rows, by.place)            # without weights
        assert none is None
        ref, mass, count = R.row_sums(R.wide(grad), place, None, t * k)
        R.check(alone, ref, mass, count[:, None], dtype)


# ---- neighbours --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,c", [(300, 7, 3), (1000, 16, 64), (700, 40, 33), (260, 128, 10)])
def test_messages_from_neighbours(n, k, c, dtype):
    """A graph, its messages and both gradients, as a training step runs them; splits smaller than k leave -1 in the index"""
    rng = np.random.default_rng(n)
    x, rs = W.uniform(n, 3, seed=n, sizes=[n - 5, 0, 5])
    idx, d2 = B.fg_binned_select_knn(dev(x), dev(rs), k)
    assert bool((idx < 0).any())
    w = torch.exp(-10.0 * d2)
    rows, grad = values(rng, n, c, dtype), values(rng, n, c, dtype)
    index = idx.cpu().numpy()
    ref, mass = R.combine(R.wide(rows), index, R.wide(w))
    R.check(B.fg_combine(rows, idx, w), ref, mass, k, dtype)
    by = B.fg_index_sort(idx, n, place=False)
    grad_rows, grad_w = B.fg_combine_backward(grad, rows, idx, w, sort=by)
    ref, mass, count = R.row_sums(R.wide(grad), index, R.wide(w), n)
    R.check(grad_rows, ref, mass, count[:, None], dtype)
    R.check(grad_w, *R.dots(R.wide(grad), R.wide(rows), index), c, torch.float32)
    # on to the coordinates, through the framework's own backward
    grad_x = B.fg_knn_backward((-10.0 * w * grad_w).contiguous(), idx, dev(x), dev(rs))
    assert bool(grad_x.isfinite().all()) and bool(grad_x.any())
    alone, none = B.fg_combine_backward(grad, rows, idx, sort=by)
    assert none is None
    ref, mass, count = R.row_sums(R.wide(grad), index, None, n)
    R.check(alone, ref, mass, count[:, None], dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,t,k,c", [(5, 300, 7, 24), (3, 1500, 16, 8), (4, 9000, 8, 200), (2500, 4000, 30, 256), (90, 700, 5, 512), (60, 500, 5, 520), (40000, 90000, 3, 5)])
def test_shared_rows(n, t, k, c, dtype):
    """Rows named by few and by thousands of entries, with lanes of a row that have no piece, and rows too wide for products along the way"""
    rng = np.random.default_rng(n + t)
    index = some_index(rng, (t, k), n, "frequent")
    rows, grad, w = values(rng, n, c, dtype), values(rng, t, c, dtype), dev(rng.random((t, k)).astype(np.float32))
    by = B.fg_index_sort(dev(index), n)
    for weights in (w, None):
        wide = None if weights is None else R.wide(w)
        gw, again = torch.full((t, k), 7.0, device=DEV), torch.full((t, k), 7.0, device=DEV)
        got, gw = B.fg_combine_backward(grad, rows, dev(index), weights, sort=by, grad_weights=gw)
        ref, mass, count = R.row_sums(R.wide(grad), index, wide, n)
        R.check(got, ref, mass, count[:, None], dtype)
        R.check(gw, *R.dots(R.wide(grad), R.wide(rows), index), c, torch.float32)
        # the same call, the same bits
        assert all(torch.equal(a, b) for a, b in zip((got, gw), B.fg_combine_backward(grad, rows, dev(index), weights, sort=by, grad_weights=again)))
        if weights is None:                                                  # without the weights' gradient it is another kernel's
            R.check(B.fg_combine_backward(grad, rows, dev(index), sort=by)[0], ref, mass, count[:, None], dtype)
    ref, mass = R.combine(R.wide(rows), index, R.wide(w))
    R.check(B.fg_combine(rows, dev(index), w), ref, mass, k, dtype)


@pytest.mark.parametrize("n,k,c,dtype", [(3000, 12, 64, torch.float32), (9000, 16, 40, torch.bfloat16), (2000, 9, 260, torch.float32), (9000, 5, 3, torch.float16),
                                         (20000, 3, 1024, torch.bfloat16), (700, 6, 64, torch.float32)])
def test_walk_changes_no_bit(n, k, c, dtype):
    """The bins' order of the points, the order reversed, and any order give what no order gives"""
    rng = np.random.default_rng(n + k)
    x, rs = W.uniform(n, 3, seed=k, sizes=[n - 11, 11])
    binning = B.fg_bin_points(dev(x), dev(rs), k)
    idx, d2 = B.fg_query_binned(binning, dev(rs), k)
    rows, grad, w = values(rng, n, c, dtype), values(rng, n, c, dtype), torch.exp(-d2)
    by = B.fg_index_sort(idx, n)
    plain = (B.fg_combine(rows, idx, w), *B.fg_combine_backward(grad, rows, idx, w, sort=by))
    for walk in (binning.perm, dev(np.arange(n, dtype=np.int32)[::-1]), dev(rng.permutation(n).astype(np.int32))):
        got = (B.fg_combine(rows, idx, w, walk=walk), *B.fg_combine_backward(grad, rows, idx, w, sort=by, walk=walk))
        assert all(torch.equal(a, b) for a, b in zip(got, plain))
    # numbers outside are skipped, nothing is read or written there
    out = torch.full((n, c), 7.0, dtype=dtype, device=DEV)
    walk = binning.perm.clone()
    left = walk[:4].long()
    walk[:4] = dev(np.array([-1, n, 2 ** 31 - 1, -2 ** 31], dtype=np.int32))
    B.fg_combine(rows, idx, w, out=out, walk=walk)
    assert bool((out[left] == 7.0).all())
    out[left] = plain[0][left]
    assert torch.equal(out, plain[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [70001, 262144])
def test_wide_rows(c, dtype):
    """Up to the largest width: many wavefronts a row"""
    rng = np.random.default_rng(c)
    n, t, k = 7, 5, 3
    index, w = some_index(rng, (t, k), n), dev(rng.random((t, k)).astype(np.float32))
    rows, grad = values(rng, n, c, dtype), values(rng, t, c, dtype)
    got = B.fg_lookup(rows, dev(index.reshape(-1)), 0.5)
    ref = R.lookup(R.wide(rows), index.reshape(-1), 0.5)
    R.check(got, ref, abs(ref), 0, dtype)
    ref, mass = R.combine(R.wide(rows), index, R.wide(w))
    R.check(B.fg_combine(rows, dev(index), w), ref, mass, k, dtype)
    by = B.fg_index_sort(dev(index), n)
    sums, mass, count = R.row_sums(R.wide(grad), index, R.wide(w), n)
    dots = R.dots(R.wide(grad), R.wide(rows), index)
    got, gw = B.fg_combine_backward(grad, rows, dev(index), w, sort=by)
    R.check(got, sums, mass, count[:, None], dtype)
    R.check(gw, *dots, c, torch.float32)
    sent = B.fg_dispatch(grad, by.place, torch.zeros((t * k, c), dtype=dtype, device=DEV))
    place = by.place.cpu().numpy()
    for (i, j), p in np.ndenumerate(place):
        assert p < 0 or torch.equal(sent[p], grad[i])
    with pytest.raises(B.FgError):
        B.fg_lookup(torch.zeros((2, 262145), device=DEV), dev(index))


def test_nothing_to_do():
    """No tokens, no rows: outputs that are there are written all the same"""
    none, rows = torch.zeros((0, 3), dtype=torch.int32, device=DEV), torch.ones((6, 8), device=DEV)
    empty, w = torch.zeros((0, 8), device=DEV), torch.zeros((0, 3), device=DEV)
    assert B.fg_combine(rows, none, w).shape == (0, 8) and B.fg_dispatch(empty, none).shape == (0, 8)
    by = B.fg_index_sort(none, 6)
    assert by.place.shape == (0, 3) and by.order.numel() == 0 and not bool(by.bounds.any())
    for sort in (by, None):
        got, gw = B.fg_combine_backward(empty, rows, none, w, sort=sort)
        assert got.shape == (6, 8) and not bool(got.any()) and gw.shape == (0, 3)
    assert not bool(B.fg_lookup_backward(empty, B.fg_index_sort(torch.zeros(0, dtype=torch.int32, device=DEV), 6)).any())
    # no rows to name
    index, grad, w = torch.zeros((4, 3), dtype=torch.int32, device=DEV), torch.ones((4, 8), device=DEV), torch.ones((4, 3), device=DEV)
    by = B.fg_index_sort(index, 0)
    assert bool((by.place == -1).all()) and by.bounds.tolist() == [0] and by.order.tolist() == list(range(12))
    assert not bool(B.fg_combine(empty, index, w).any())
    for sort in (by, None):
        got, gw = B.fg_combine_backward(grad, empty, index, w, sort=sort)
        assert got.shape == (0, 8) and not bool(gw.any())
    assert B.fg_lookup_backward(grad.repeat(3, 1), by).shape == (0, 8)
    torch.cuda.synchronize()


def test_gradients_against_differences():
    """Outputs are linear in rows and in weights: a step of 1 in one of them changes the loss by its gradient, but for rounding"""
    rng = np.random.default_rng(12)
    t, k, n, c = 60, 5, 25, 24
    index = dev(some_index(rng, (t, k), n))
    rows, w, up = values(rng, n, c, torch.float32), dev(rng.random((t, k)).astype(np.float32)), values(rng, t, c, torch.float32)
    by = B.fg_index_sort(index, n)
    grad_rows, grad_w = B.fg_combine_backward(up, rows, index, w, sort=by)

    def loss(r, v):
        return float((B.fg_combine(r, index, v).double() * up.double()).sum())
    at = loss(rows, w)
    # each of the t*c outputs is off by at most (2k + 5) 2^-24 of its sum of absolute terms (below 30), and counts |up| (below 5) times
    room = 2 * t * c * (2 * k + 5) * 2.0 ** -24 * 30 * 5
    for i, j in [(0, 0), (7, 23), (24, 11)]:
        moved = rows.clone()
        moved[i, j] += 1
        assert abs(loss(moved, w) - at - float(grad_rows[i, j])) <= room
    for i, j in [(0, 0), (31, 2), (59, 4)]:
        moved = w.clone()
        moved[i, j] += 1
        assert abs(loss(rows, moved) - at - float(grad_w[i, j])) <= room
    table = values(rng, n, c, torch.float32)
    flat = index.reshape(-1)
    up = values(rng, t * k, c, torch.float32)
    grad = B.fg_lookup_backward(up, B.fg_index_sort(flat, n), 3.0)
    table_loss = lambda a: float((B.fg_lookup(a, flat, 3.0).double() * up.double()).sum())      # noqa: E731
    for i, j in [(0, 0), (13, 7), (24, 23)]:
        moved = table.clone()
        moved[i, j] += 1
        assert abs(table_loss(moved) - table_loss(table) - float(grad[i, j])) <= room


# ---- far offsets, streams, graphs --------------------------------------------------------------------------------------

def test_offsets_beyond_32_bits():
    """Tables of more than 2^32 elements: every operator at their far end"""
    n, c, t, k = (1 << 21) + 100, 2080, 40, 3
    rng = np.random.default_rng(21)
    table = torch.zeros((n, c), dtype=torch.bfloat16, device=DEV)
    index = (n - 1 - rng.permutation(t * k)).astype(np.int32)
    used = values(rng, t * k, c, torch.bfloat16)
    table[dev(index).long()] = used
    assert torch.equal(B.fg_lookup(table, dev(index)), used)
    at, w = dev(index.reshape(t, k)), dev(rng.random((t, k)).astype(np.float32))
    local = np.arange(t * k, dtype=np.int32).reshape(t, k)
    ref, mass = R.combine(R.wide(used), local, R.wide(w))
    R.check(B.fg_combine(table, at, w), ref, mass, k, torch.bfloat16)
    grad = values(rng, t, c, torch.bfloat16)
    ref, mass, count = R.row_sums(R.wide(grad), local, R.wide(w), t * k)
    for by in (B.fg_index_sort(at, n), None):
        out = torch.zeros((n, c), dtype=torch.bfloat16, device=DEV)
        got, gw = B.fg_combine_backward(grad, table, at, w, sort=by, grad_rows=out)
        R.check(got[dev(index).long()], ref, mass, count[:, None], torch.bfloat16)
        assert int(torch.count_nonzero(got[:n - t * k].view(torch.int16))) == 0
        R.check(gw, *R.dots(R.wide(grad), R.wide(used), local), c, torch.float32)
    table.zero_()
    B.fg_dispatch(grad, at, table)
    assert torch.equal(table[at.long()], grad[:, None, :].expand(t, k, c))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [72, 1000, 2049, 4104])
def test_more_than_the_caches_hold(c, dtype):
    """Calls that move 512 MB and more against the same rows in calls of a seventh: where a sum does not go by the number of rows, to the bit"""
    gen = torch.Generator(device=DEV).manual_seed(c)
    size, k = torch.empty((), dtype=dtype).element_size(), 3
    m = (512 << 20) // (c * size) + 77
    t = m // k

    def part(n, i):
        return slice(n * i // 7, n * (i + 1) // 7)
    table = torch.randn((5001, c), generator=gen, device=DEV).to(dtype)
    index = torch.randint(-1, 5002, (m,), generator=gen, device=DEV, dtype=torch.int32)
    got = B.fg_lookup(table, index, 0.7)
    assert all(torch.equal(got[part(m, i)], B.fg_lookup(table, index[part(m, i)], 0.7)) for i in range(7))
    # every row named once, a few by nobody
    rows, grad = torch.randn((m, c), generator=gen, device=DEV).to(dtype), torch.randn((t, c), generator=gen, device=DEV).to(dtype)
    at = torch.randperm(m, generator=gen, device=DEV)[:t * k].to(torch.int32).view(t, k)
    at[::50] = -1
    w = torch.rand((t, k), generator=gen, device=DEV)
    for weights in (w, None):
        got = B.fg_combine(rows, at, weights)
        assert all(torch.equal(got[part(t, i)], B.fg_combine(rows, at[part(t, i)], None if weights is None else weights[part(t, i)])) for i in range(7))
    got, gw = B.fg_combine_backward(grad, rows, at, w)
    again, parts = torch.zeros_like(rows), []
    for i in range(7):
        parts.append(B.fg_combine_backward(grad[part(t, i)], rows, at[part(t, i)], w[part(t, i)], grad_rows=again)[1])
    assert torch.equal(got, again)
    # (products go by the lanes that a token gets, and these by the number of tokens)
    terms = [torch.where(at[:, j:j + 1] >= 0, rows[at[:, j].clamp(0).long()].double() * grad.double(), 0.0) for j in range(k)]
    ref, mass = R.wide(torch.stack([x.sum(1) for x in terms], 1)), R.wide(torch.stack([x.abs().sum(1) for x in terms], 1))
    R.check(gw, ref, mass, c, torch.float32)
    R.check(torch.cat(parts), ref, mass, c, torch.float32)
    # a table of which most rows are named by nobody or a few, one by many
    n, few = m, 3001
    index = torch.randint(-1, n, (few,), generator=gen, device=DEV, dtype=torch.int32)
    index[::9] = n // 2
    grad = torch.randn((few, c), generator=gen, device=DEV).to(dtype)
    named = index >= 0
    count = torch.zeros(n, device=DEV, dtype=torch.float64).index_add_(0, index[named].long(), torch.ones(int(named.sum()), device=DEV, dtype=torch.float64))
    some = torch.nonzero(count)[:, 0]
    to = torch.cumsum(count > 0, 0) - 1
    ref, mass = (torch.zeros((len(some), c), device=DEV, dtype=torch.float64).index_add_(0, to[index[named].long()], x) for x in (grad[named].double(), grad[named].double().abs()))
    got = B.fg_lookup_backward(grad, B.fg_index_sort(index, n))
    assert int(torch.count_nonzero(got.view(torch.int32 if dtype == torch.float32 else torch.int16).any(1))) <= len(some)
    R.check(got[some], R.wide(ref), R.wide(mass), count[some, None].cpu().numpy(), dtype)


def test_on_a_stream_of_its_own():
    rng = np.random.default_rng(1)
    index, x, w = dev(choices(rng, 500, 4, 16, 0.1)), values(rng, 500, 320, torch.bfloat16), dev(rng.random((500, 4)).astype(np.float32))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        by = B.fg_index_sort(index, 16)
        sent = B.fg_dispatch(x, by.place, torch.zeros((2000, 320), dtype=torch.bfloat16, device=DEV))
        out = B.fg_combine(sent, by.place, w)
        grads = B.fg_combine_backward(x, sent, by.place, w)
    side.synchronize()
    by = B.fg_index_sort(index, 16)
    sent2 = B.fg_dispatch(x, by.place, torch.zeros((2000, 320), dtype=torch.bfloat16, device=DEV))
    assert torch.equal(sent, sent2) and torch.equal(out, B.fg_combine(sent2, by.place, w))
    assert all(torch.equal(a, b) for a, b in zip(grads, B.fg_combine_backward(x, sent2, by.place, w)))


@pytest.mark.parametrize("m,n_rows", [(1_200_000, 1_000_000), (300_000, 77)])
def test_a_large_sort_captured_and_replayed(m, n_rows):
    rng = np.random.default_rng(m)
    index = torch.zeros(m, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.fg_index_sort(index, n_rows)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.fg_index_sort(index, n_rows)
    for seed in range(4):
        index.copy_(dev(some_index(rng, (m,), n_rows, "frequent" if seed % 2 else "uniform")))
        graph.replay()
        torch.cuda.synchronize()
        now = B.fg_index_sort(index, n_rows)
        assert torch.equal(got.order, now.order) and torch.equal(got.bounds, now.bounds) and torch.equal(got.place, now.place)
        torch.cuda.synchronize()


def test_two_at_once():
    """The same calls on two streams, with what the allocator gives each, over and over: no result depends on the other's"""
    rng = np.random.default_rng(31)
    n, t, k, c = 3000, 20000, 6, 64
    sets = [(dev(some_index(rng, (t, k), n, "frequent")), values(rng, n, c, torch.float32), values(rng, t, c, torch.float32),
             dev(rng.random((t, k)).astype(np.float32))) for _ in range(2)]

    def step(index, rows, grad, w):
        by = B.fg_index_sort(index, n)
        return (B.fg_combine(rows, index, w), *B.fg_combine_backward(grad, rows, index, w, sort=by), by.order)
    alone = [step(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(step(*sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for again in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(alone[i], again))


@pytest.mark.parametrize("t", [70, 5000])
def test_captured_and_replayed(t):
    """The whole layer, forward and backward, in a graph: replays on new inputs give what eager calls give"""
    rng = np.random.default_rng(t)
    k, experts, c, vocab = 4, 24, 200, 3000
    tokens = torch.zeros(t, dtype=torch.int32, device=DEV)
    index = torch.zeros((t, k), dtype=torch.int32, device=DEV)
    table, w, up = values(rng, vocab, c, torch.bfloat16), torch.zeros((t, k), device=DEV), torch.zeros((t, c), dtype=torch.bfloat16, device=DEV)

    def layer():
        x = B.fg_lookup(table, tokens, 2.0)
        by = B.fg_index_sort(index, experts)
        sent = B.fg_dispatch(x, by.place, torch.zeros((t * k, c), dtype=torch.bfloat16, device=DEV))
        out = B.fg_combine(sent, by.place, w)
        grad_sent, grad_w = B.fg_combine_backward(up, sent, by.place, w)
        grad_x = B.fg_combine(grad_sent, by.place)
        names = B.fg_index_sort(tokens, vocab, place=False)
        return out, grad_w, B.fg_lookup_backward(grad_x, names, 2.0, dtype=torch.float32), by.order, names.bounds

    def fill(seed):
        r = np.random.default_rng(seed)
        tokens.copy_(dev(some_index(r, (t,), vocab, "frequent")))
        index.copy_(dev(choices(r, t, k, experts, 0.1)))
        w.copy_(dev(r.random((t, k)).astype(np.float32)))
        up.copy_(values(r, t, c, torch.bfloat16))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer()
    for seed in range(1, 6):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, layer())), seed
        torch.cuda.synchronize()


def test_the_binding_checks_its_tensors():
    f, i = torch.zeros((6, 8), device=DEV), torch.zeros((6, 2), dtype=torch.int32, device=DEV)
    by = B.fg_index_sort(i, 6)
    w = torch.zeros((6, 2), device=DEV)
    bad = [lambda: B.fg_index_sort(i.long(), 6), lambda: B.fg_index_sort(i.t(), 6),
           lambda: B.fg_lookup(f.double(), i), lambda: B.fg_lookup(f.t(), i), lambda: B.fg_lookup(f, i.long()), lambda: B.fg_lookup(f[0], i),
           lambda: B.fg_lookup(f, i, out=torch.zeros((6, 8), device=DEV)), lambda: B.fg_lookup(f, i, out=torch.zeros((12, 8), device=DEV).half()),
           lambda: B.fg_lookup_backward(f, by), lambda: B.fg_lookup_backward(torch.zeros((12, 8), device=DEV), by, accumulate=True),
           lambda: B.fg_lookup_backward(torch.zeros((12, 8), device=DEV), by, grad_table=torch.zeros((5, 8), device=DEV)),
           lambda: B.fg_dispatch(f, i[:5]), lambda: B.fg_dispatch(f, i.reshape(-1)), lambda: B.fg_dispatch(f, i, torch.zeros((12, 7), device=DEV)),
           lambda: B.fg_combine(f, i, walk=torch.zeros(5, dtype=torch.int32, device=DEV)), lambda: B.fg_combine(f, i, walk=torch.zeros(6, device=DEV)),
           lambda: B.fg_combine_backward(f, f, i, w, sort=by, walk=i), lambda: B.fg_combine(f, i, w[:, :1]), lambda: B.fg_combine(f, i, w.half()), lambda: B.fg_combine(f, i, out=f[:5]),
           lambda: B.fg_combine_backward(f[:5], f, i, w), lambda: B.fg_combine_backward(f.half(), f, i, w),
           lambda: B.fg_combine_backward(f, f, i, w, sort=B.fg_index_sort(i, 7)), lambda: B.fg_combine_backward(f, f, i, w, grad_weights=w.half()),
           lambda: B.fg_combine_backward(f, f, i, w, grad_rows=f[:, :4])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in [lambda: B.fg_index_sort(i, -1), lambda: B.fg_combine(f, torch.zeros((6, 129), dtype=torch.int32, device=DEV)),
                 lambda: B.fg_lookup_backward(torch.zeros((12, 8), device=DEV).half(), by, dtype=torch.bfloat16),
                 lambda: B.fg_lookup_backward(torch.zeros((9000, 8), device=DEV), B.fg_index_sort(torch.zeros(9000, dtype=torch.int32, device=DEV), 6),
                                              workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))]:
        with pytest.raises(B.FgError):
            call()
    torch.cuda.synchronize()
