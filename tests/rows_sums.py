"""Sums over many rows, held to what they have to be: exactly, or within the rounding of the chains in which the
kernels add.

A bound that allows for any order of k additions, k u sum|values|, grows as k^2 and the sum itself as sqrt(k): with
enough rows such a bound lets a sum of zeros pass.  Here sums whose values can be chosen take whole numbers whose
absolute values add up to less than 2^24: every partial sum is a whole number that fp32 holds, so that a sum
has one value in any order.  dweight, whose values are no whole numbers, is held to the chain that its kernels have."""
from __future__ import annotations

import torch

from rows64 import DT, U, _stats


def whole(rows, d, seed, most=7):
    """Whole numbers of up to `most`, less where so many rows would pass 2^24 (as int8)."""
    most = min(most, (2 ** 24 - 1) // max(1, rows))
    assert most >= 1, rows
    return torch.randint(-most, most + 1, (rows, d), dtype=torch.int8, generator=torch.Generator().manual_seed(seed))


def embedding_sums(ids, dy, vocab, scale, n_pos, dtype):
    """dtable and dpos of whole numbers dy, scale a power of two: exact, then rounded once to the storage type."""
    d = dy.shape[-1]
    ok = (ids >= 0) & (ids < vocab)
    whole_ids, whole_dy = (ids, dy) if ok.all() else (ids[ok], dy[ok])
    dtable = torch.zeros(vocab, d, dtype=torch.float64).index_add_(0, whole_ids, whole_dy.double())
    dpos = dy.view(-1, n_pos, d).double().sum(0).to(DT[dtype]) if n_pos else None
    return (scale * dtable).to(DT[dtype]), dpos


def additions(rows, d):
    """How many additions one after the other a column of dweight takes at most.

    Up to 256 workgroups of 512 threads share the rows, and a row takes at most as many lanes as it has vectors of 4
    values, rounded up to a power of two from 4 to 512: a workgroup takes 512 / lanes rows at once, and a lane adds
    one row a round (few rows are one workgroup's, of at most four rounds).  Then up to four levels join the rows of a wave, up to
    eight additions the waves of a workgroup, up to four a lane's share of 256 workgroups, four levels and four additions
    those."""
    lanes = 4
    while lanes < 512 and 4 * lanes < d:
        lanes *= 2
    at_once = 512 // lanes
    return max(4, -(-rows // (256 * at_once)) + 1) + 4 + 8 + 4 + 4 + 4


def dweight(z, dy, eps):
    """sum_r dy xh in 64 bits and its bound: xh off as tests/rows64.py works out, and the roundings of the chain."""
    _, _, xh, _, ex = _stats(z, eps)
    v = dy * xh
    return v.sum(0), (dy.abs() * ex).sum(0) + (additions(*z.shape) + 2) * U * v.abs().sum(0)
