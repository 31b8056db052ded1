"""Rows by index on the GPU, with values that are not finite."""
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
