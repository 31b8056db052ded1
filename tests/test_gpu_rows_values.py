"""Rows by index on the GPU, with values whose results are known to the bit: infinities, and whole numbers whose sums are exact in float32."""
import numpy as np
import pytest
import torch

import rows_oracle as R
from paper_2511_10442_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def check_dots(got, grad, rows, index, c):
    """Products in 64 bits; where they are infinite or no number, so must the answer be."""
    with np.errstate(invalid="ignore"):
        ref, mass = R.dots(R.wide(grad), R.wide(rows), index)
    finite = np.isfinite(ref)
    assert finite.any() and (ref == np.inf).any() and (ref == -np.inf).any() and np.isnan(ref).any()
    assert np.array_equal(R.wide(got)[~finite], ref[~finite], equal_nan=True)
    R.check(torch.where(dev(finite), got, 0.0), np.where(finite, ref, 0.0), np.where(finite, mass, 0.0), c, torch.float32)


# (pieces of a row that are a power of two from 8 on, and others: a row's lanes that have no piece of it)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 3, 8, 24, 40, 64, 96, 200, 256, 260])
@pytest.mark.parametrize("n,t,k", [(2000, 500, 4), (6, 900, 3)])
def test_infinities_in_the_gradient_of_weights(n, t, k, c, dtype):
    """An infinity in a row's last element (or its first) gives infinite products, or none with a gradient of 0 there; other entries' stay as they are"""
    rng = np.random.default_rng(n + c)
    rows = dev(rng.standard_normal((n, c)).astype(np.float32)).to(dtype)
    rows[::3, -1], rows[1::6, 0] = float("inf"), float("-inf")
    grad = dev(rng.standard_normal((t, c)).astype(np.float32)).to(dtype)
    grad[::7, -1] = 0.0
    w = dev(rng.random((t, k)).astype(np.float32))
    index = rng.integers(-1, n, size=(t, k)).astype(np.int32)
    by = B.fg_index_sort(dev(index), n)
    for weights in (w, None):
        gw = torch.full((t, k), 7.0, device=DEV)
        got, gw = B.fg_combine_backward(grad, rows, dev(index), weights, sort=by, grad_weights=gw)
        check_dots(gw, grad, rows, index, c)
        ref, mass, count = R.row_sums(R.wide(grad), index, None if weights is None else R.wide(w), n)
        R.check(got, ref, mass, count[:, None], dtype)
    if n == t * k:                                       # every row named once: with a sorted index and without one
        index = rng.permutation(n).astype(np.int32).reshape(t, k)
        for by in (B.fg_index_sort(dev(index), n), None):
            check_dots(B.fg_combine_backward(grad, rows, dev(index), w, sort=by)[1], grad, rows, index, c)


# ---- whole numbers -----------------------------------------------------------------------------------------------------
# Values from 1 to 3: every sum below has whole partial sums under 2^24, which float32 holds, in whatever order they are made.  No part of one is zero, so that
# none can be lost or counted twice unseen.

def whole(rng, n, c, dtype):
    return dev(rng.integers(1, 4, size=(n, c)).astype(np.float32)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,c", [(500_003, 8), (500_003, 20), (5_000_011, 4)])
def test_a_row_of_many_entries(m, c, dtype):
    """Chunks, chunks of chunks, and larger chunks where there would be too many of them (5M entries, below 3 * 5_000_011 < 2^24)"""
    rng = np.random.default_rng(m + c)
    index = np.full(m, 3, dtype=np.int32)
    index[rng.integers(0, m, size=100)] = rng.integers(-1, 7, size=100)
    grad = whole(rng, m, c, dtype)
    got = B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 7), dtype=torch.float32)
    ref = torch.zeros((8, c), dtype=torch.float64, device=DEV).index_add_(0, dev(np.where(index < 0, 7, index)).long(), grad.double())[:7]
    assert torch.equal(got.double(), ref)
    there = whole(rng, 7, c, torch.float32)
    was = there.double()
    B.fg_lookup_backward(grad, B.fg_index_sort(dev(index), 7), 0.5, grad_table=there, accumulate=True)
    assert torch.equal(there.double(), (was + 0.5 * ref).float().double())


@pytest.mark.parametrize("n,t,k,c", [(5, 100_000, 5, 64), (3, 1_250_000, 4, 4), (40, 30_000, 7, 24), (7, 20_000, 5, 1000)])
def test_shared_rows_of_many_entries(n, t, k, c):
    """Sums of at most 2^24 / 3 / 3 entries' products and every entry's product with its row"""
    rng = np.random.default_rng(n + t)
    index = rng.integers(0, n, size=(t, k)).astype(np.int32)
    index[rng.random((t, k)) < 0.6] = 1
    index[rng.random((t, k)) < 0.01] = -1
    rows, grad = whole(rng, n, c, torch.float32), whole(rng, t, c, torch.float32)
    w = whole(rng, t, k, torch.float32) if t * k * 9 < 1 << 24 else None
    gw = torch.full((t, k), 7.0, device=DEV)
    got, gw = B.fg_combine_backward(grad, rows, dev(index), w, sort=B.fg_index_sort(dev(index), n), grad_weights=gw)
    at = dev(np.where(index < 0, n, index)).long()
    ref = torch.zeros((n + 1, c), dtype=torch.float64, device=DEV)
    padded = torch.cat([rows, torch.zeros((1, c), device=DEV)]).double()
    for j in range(k):
        ref.index_add_(0, at[:, j], grad.double() if w is None else grad.double() * w[:, j:j + 1].double())
        assert torch.equal(gw[:, j].double(), (padded[at[:, j]] * grad.double()).sum(1))
    assert torch.equal(got.double(), ref[:n])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [70001, 262144])
def test_the_widest_rows(c, dtype):
    """Products over a whole row (9 * 262144 < 2^24); sums of rows stay below 128, which every type holds"""
    rng = np.random.default_rng(c)
    n, t, k = 7, 5, 3
    index = rng.permutation(np.resize(np.arange(-1, n), t * k)).reshape(t, k).astype(np.int32)
    rows, grad, w = whole(rng, n, c, dtype), whole(rng, t, c, dtype), whole(rng, t, k, torch.float32)
    at = dev(index)
    named = (at >= 0)[:, :, None]
    of = torch.where(named, rows[at.clamp(min=0).long()].double(), 0.0)
    assert torch.equal(B.fg_combine(rows, at, w).double(), (of * w[:, :, None].double()).sum(1))
    dots = (of * grad[:, None, :].double()).sum(2)
    ref = torch.zeros((n, c), dtype=torch.float64, device=DEV)
    for i, j in zip(*np.nonzero(index >= 0)):
        ref[index[i, j]] += grad[i].double() * w[i, j].double()
    got, gw = B.fg_combine_backward(grad, rows, at, w, sort=B.fg_index_sort(at, n))
    assert torch.equal(got.double(), ref) and torch.equal(gw.double(), dots)
    # every row named once
    rows, place = whole(rng, t * k, c, dtype), dev(rng.permutation(t * k).reshape(t, k).astype(np.int32))
    got, gw = B.fg_combine_backward(grad, rows, place, w)
    of = rows[place.long()].double()
    assert torch.equal(gw.double(), (of * grad[:, None, :].double()).sum(2))
    assert torch.equal(got[place.long()].double(), grad[:, None, :].double() * w[:, :, None].double())
    # a table's gradient
    flat = at.reshape(-1)
    up = whole(rng, t * k, c, dtype)
    ref = torch.zeros((n + 1, c), dtype=torch.float64, device=DEV).index_add_(0, torch.where(flat < 0, n, flat).long(), up.double())[:n]
    assert torch.equal(B.fg_lookup_backward(up, B.fg_index_sort(flat, n)).double(), ref)
