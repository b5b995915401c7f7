"""The loss over a vocabulary and distillation from a teacher's top logits with their gradients, in 64 bits on the CPU, and
how far the kernels' arithmetic may be from them.

u = 2^-24 is half a step of fp32, 2^-11 of fp16.  Operands of the products:
  bf16 storage: exact (an fp16 plane holds values down to 2^-31 of its row's largest, below that
                off by at most 2^-40 of it); G as one fp16 plane, off by 2^-11 of itself and 2^-39 of the largest
  fp32 storage: pairs (hi, lo), off by 2^-22 of the value and 2^-40 of its row's largest; the product leaves lo lo out, 2^-22;
                G off by 2^-22 of itself and 2^-39 of the largest
A product of 16 k is added to its sum at once: it is taken to round at most 16 times, and a sum of K products in P planes
P (K / 16 + 16) times (P = 3 for pairs).  exp2 and log2 are off by at most 2 u of their results.
"""
from __future__ import annotations

import math

import torch

from rows64 import U, d64

PAIR = 2.0 ** -22


def chain(k: int, planes: int) -> int:
    return (3 if planes == 2 else 1) * (-(-k // 16) + 16)


def _size(a):
    """|a| and how far its laid-out values may be from it, by row."""
    return a.abs(), a.abs().amax(-1, keepdim=True) if a.shape[-1] else a.abs()


def logits(x, table, bias, scale, planes):
    """l and the error of its products: sums of |x||w| for their rounding, operands' own errors, and the
    three roundings after them (scale and units of log 2, bias)."""
    b = torch.zeros(table.shape[0], dtype=torch.float64) if bias is None else bias
    l = scale * (x @ table.t() + b)
    ax, mx = _size(x)
    aw, mw = _size(table)
    cross = ax @ aw.t()
    floor = 2.0 ** -40 * (mx * aw.sum(-1) + ax.sum(-1, keepdim=True) * mw.t())
    err = (chain(x.shape[1], planes) * U + (3 * PAIR if planes == 2 else 0)) * cross + floor
    # (an entry whose bias is -inf has no error)
    fine = torch.isfinite(l)
    l0 = torch.where(fine, l, 0.0)
    e = abs(scale) * err + 8 * U * (l0.abs() + abs(scale) * torch.where(torch.isfinite(b), b, 0.0).abs())
    return l, torch.where(fine, e, 0.0)


def _named(ids, vocab, teacher=None):
    ok = (ids >= 0) & (ids < vocab)
    return ok if teacher is None else ok & (teacher != -math.inf)


def teacher_p(ids, teacher, vocab, scale):
    """p, log p (0 where left out), which are named, and p's relative error: the exponents' rounding and the sum."""
    ok = _named(ids, vocab, teacher)
    a = torch.where(ok, teacher * scale, -math.inf)
    any_ = ok.any(-1, keepdim=True)
    z = torch.where(any_, torch.logsumexp(a, -1, keepdim=True), 0.0)
    logp = torch.where(ok, a - z, 0.0)
    p = torch.where(ok, torch.exp(logp), 0.0)
    size = torch.where(ok, a.abs(), 0.0).amax(-1, keepdim=True)
    rel = (6 * size + ids.shape[-1] / 64 + 20) * U
    return p, logp, ok, rel


def dot_error(x, w, d):
    """of an fp32 dot product by 64 lanes."""
    return (d // 64 + 16) * U * (x.abs() * w.abs()).sum(-1)


def loss(x, table, bias, scale, ids, teacher, planes):
    """(loss, lse, logq), their errors.  Cross entropy: ids [n, 1], teacher None."""
    vocab = table.shape[0]
    l, le = logits(x, table, bias, scale, planes)
    n = x.shape[0]
    b = torch.zeros(vocab, dtype=torch.float64) if bias is None else bias
    z = torch.logsumexp(l, 1)
    # the sum of exponentials: a part of at most 64 at a time, parts joined; maxima up to |l|
    size = torch.where(torch.isfinite(l), l, 0.0).abs().amax(1)
    ze = le.amax(1) + (160 + vocab / 128) * U + 8 * U * (size + z.abs())
    ids = ids.reshape(n, -1)
    if teacher is None:
        ok = _named(ids, vocab)
        p, logp, rel = ok.double(), torch.zeros_like(ids, dtype=torch.float64), torch.zeros(n, 1, dtype=torch.float64)
    else:
        p, logp, ok, rel = teacher_p(ids, teacher.reshape(n, -1), vocab, scale)
    at = torch.where(ok, ids, 0)
    w = table[at]
    s = scale * ((x[:, None] * w).sum(-1) + b[at])
    se = abs(scale) * dot_error(x[:, None], w, x.shape[1]) + 4 * U * (s.abs() + abs(scale) * b[at].abs())
    q = torch.where(ok, s - z[:, None], 0.0)
    qe = torch.where(ok, se + ze[:, None] + 2 * U * (q.abs() + z[:, None].abs()), 0.0)
    out = torch.where(ok & (p > 0), p * (logp - q), 0.0)
    part = ok.any(1)
    oute = (p * (qe + 4 * U * logp.abs() + rel) + (rel + 4 * U) * out.abs()).sum(1) + 20 * U * out.abs().sum(1)
    zero = torch.zeros((), dtype=torch.float64)
    return ((torch.where(part, out.sum(1), zero), torch.where(part, z, zero), q),
            (torch.where(part, oute, zero), torch.where(part, ze, zero), qe))


def gradients(x, table, bias, scale, ids, teacher, logq, lse, dloss, planes):
    """(dx, dtable, dbias), their errors before the last rounding; logq [n, top] (cross entropy: minus the loss) and lse
    as they are given to the backward."""
    n, vocab = x.shape[0], table.shape[0]
    ids = ids.reshape(n, -1)
    if teacher is None:
        ok = _named(ids, vocab)
        p, rel = ok.double(), torch.zeros(n, 1, dtype=torch.float64)
    else:
        p, _, ok, rel = teacher_p(ids, teacher.reshape(n, -1), vocab, scale)
    part = ok.any(1) & (dloss != 0)
    x = torch.where(part[:, None], x, 0.0)  # tokens that take no part, whatever they hold
    dl = torch.where(part, dloss, 0.0) * scale
    l, le = logits(x, table, bias, scale, planes)
    q = torch.exp(torch.where(part[:, None], l - lse[:, None], -math.inf))
    qe = q * (le + 8 * U * (torch.where(torch.isfinite(l), l, 0.0).abs() + lse.abs()[:, None]) + 4 * U)
    taught = torch.zeros(n, vocab, dtype=torch.float64)
    taughte = torch.zeros_like(taught)
    at = torch.where(ok, ids, 0)
    taught.scatter_add_(1, at, torch.where(ok, p, 0.0))
    taughte.scatter_add_(1, at, torch.where(ok, p * (rel + 2 * U), 0.0))
    # at the taught ids q comes from logq
    here = torch.zeros(n, vocab, dtype=torch.bool).scatter_(1, at, ok) if ids.shape[1] == 1 else torch.zeros(n, vocab).scatter_add_(
        1, at, ok.float()) > 0
    given = torch.zeros(n, vocab, dtype=torch.float64)
    for k in range(ids.shape[1]):
        rows = ok[:, k] & part
        given[rows, at[rows, k]] = logq.reshape(n, -1)[rows, k]
    sum_q, sum_qe = q.clone(), qe.clone()  # what dbias sums: q as the products give it
    q = torch.where(here & part[:, None], torch.exp(given), q)
    qe = torch.where(here & part[:, None], 4 * U * q * (1 + given.abs()), qe)
    g = dl[:, None] * (q - taught)
    ge = dl.abs()[:, None] * (qe + taughte + 4 * U * (q - taught).abs())
    # as planes: scaled by its rows of x and table
    mx, mw = x.abs().amax(1, keepdim=True), table.abs().amax(1)
    # (a row of zeros is scaled as the largest: of the table by itself, of x times its dloss)
    most = (dl.abs()[:, None] * mx).amax().clamp(min=1e-300)
    sx = torch.where(mx > 0, mx, most / dl.abs()[:, None].clamp(min=1e-300))
    sw = torch.where(mw > 0, mw, mw.max().clamp(min=1e-300))
    f = most * mw.max().clamp(min=1e-300)
    room = (sx * sw[None]).clamp(min=1e-300)
    ge = ge + (2.0 ** -11 if planes == 1 else PAIR) * g.abs() + 2.0 ** -36 * f / room * part[:, None]
    ax, aw = x.abs(), table.abs()
    own = 2 * PAIR if planes == 2 else 0.0
    dx, dw = g @ table, g.t() @ x
    dxe = ge @ aw + (chain(vocab, planes) * U + own) * (g.abs() @ aw) + 2.0 ** -40 * (g.abs() @ mw)[:, None]
    dwe = ge.t() @ ax + (chain(n, planes) * U + own) * (g.abs().t() @ ax) + 2.0 ** -40 * (g.abs().t() @ mx)
    db = (dl[:, None] * (sum_q - taught)).sum(0)
    dbe = (dl.abs()[:, None] * (sum_qe + taughte + 4 * U * (sum_q + taught))).sum(0) + (n / 128 + 70) * U * (
        dl.abs()[:, None] * sum_q).sum(0) + 2.0 ** -39 * dl.abs().max().clamp(min=0) * (here.sum(0) + 1) + 2 * U * db.abs()
    return (dx, dw, db), (dxe, dwe, dbe)


__all__ = ["loss", "gradients", "logits", "teacher_p", "d64", "U"]
