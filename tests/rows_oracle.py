"""Rows by index in 64 bits, entry by entry (numpy on the CPU), and how far float32 sums may be off."""
import numpy as np
import torch

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a step, relative
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half a step of the smallest values


def wide(t):
    return t.detach().double().cpu().numpy()


def names(index, n_rows):
    return (index >= 0) & (index < n_rows)


def sort(index, n_rows):
    flat = index.reshape(-1).astype(np.int64)
    key = np.where(names(flat, n_rows), flat, n_rows)
    order = np.array(sorted(range(flat.size), key=lambda i: (key[i], i)), dtype=np.int64) if flat.size < 5000 else np.lexsort((np.arange(flat.size), key))
    counts = np.bincount(key, minlength=n_rows + 1)
    bounds = np.concatenate([[0], np.cumsum(counts[:n_rows])])
    place = np.empty(flat.size, dtype=np.int64)
    place[order] = np.arange(flat.size)
    place[key == n_rows] = -1
    return order, bounds, place.reshape(index.shape)


def lookup(table, index, scale):
    ok = names(index, len(table))
    out = np.zeros((index.size, table.shape[1]))
    out[ok] = float(np.float32(scale)) * table[index[ok]]
    return out


def row_sums(grad, index, weights, n_rows, scale=1.0):
    """(sums, sums of absolute terms, terms of each row); entry e stands for row e // (entries / rows of grad)."""
    flat = index.reshape(-1)
    fan = flat.size // max(1, len(grad))
    out, mass, count = np.zeros((n_rows, grad.shape[1])), np.zeros((n_rows, grad.shape[1])), np.zeros(n_rows)
    w = np.ones(flat.size) if weights is None else weights.reshape(-1)
    ok = np.flatnonzero(names(flat, n_rows))
    for at in np.array_split(ok, max(1, ok.size * grad.shape[1] // 2_000_000)):
        term = w[at, None] * grad[at // fan]
        np.add.at(out, flat[at], term)
        np.add.at(mass, flat[at], abs(term))
        np.add.at(count, flat[at], 1)
    return float(np.float32(scale)) * out, abs(scale) * mass, count


def combine(rows, index, weights):
    out, mass = np.zeros((len(index), rows.shape[1])), np.zeros((len(index), rows.shape[1]))
    for j in range(index.shape[1]):
        t = np.flatnonzero(names(index[:, j], len(rows)))
        term = rows[index[t, j]] * (1.0 if weights is None else weights[t, j, None])
        out[t] += term
        mass[t] += abs(term)
    return out, mass


def dots(grad, rows, index):
    out, mass = np.zeros(index.shape), np.zeros(index.shape)
    for j in range(index.shape[1]):
        t = np.flatnonzero(names(index[:, j], len(rows)))
        term = rows[index[t, j]] * grad[t]
        out[t, j] = term.sum(1)
        mass[t, j] = abs(term).sum(1)
    return out, mass


def check(got, ref, mass, terms, dtype):
    """A sum of n float32 terms in any order, each a product rounded once or not at all: n - 1 additions and n + 1 products (a scale comes on
    top) are off by at most (2 n + 1) 2^-24 of the sum of absolute terms, to first order (2 n + 4 with room for the second); the result's rounding adds half a step of its type."""
    got = wide(got)
    assert got.shape == ref.shape
    tol = (2 * terms + 4) * 2.0 ** -24 * mass + STEP[dtype] * abs(ref) * 1.01 + LEAST[dtype]
    bad = ~(abs(got - ref) <= tol)
    assert not bad.any(), "%d of %d off, the first at %s: %r, not %r (may be off by %.3g)" % (
        bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], ref[bad][0], np.broadcast_to(tol, bad.shape)[bad][0])
