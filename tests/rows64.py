"""The layer norm and the embedding with their gradients, in 64 bits on the CPU, and how far fp32
arithmetic may be from them.

u = 2^-24 is half a step of fp32.  A sum over a row of d values in which a lane adds at most
8 + d / 32 (and never more than 64) one after the other and at most ten levels join the lanes is off by
at most N u sum|values|, N = 10 + min(64, 8 + d / 32).
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}  # half a step of the storage type, relative
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def chain(d: int) -> int:
    return 10 + min(64, 8 + -(-d // 32))


def _stats(z, eps):
    """mean, rstd, xh and the errors of rstd (relative) and of xh.

    The first mean m0 is off by N u mean|z|; the second step takes mean(z - m0), whose own error is N u of the mean
    deviation (at most one standard deviation, xh = 1) and of |m0 - mean|, (N u)^2 mean|z|.  z - m0 and the step's
    subtraction round twice, 2 u |z - mean|.  The variance is that around m0 less the square of
    the step: N + 4 u of itself and 3 N u of (N u mean|z|)^2; rstd half of that and 4 u for the root and the quotient."""
    N = chain(z.shape[-1])
    mean = z.mean(-1, keepdim=True)
    rstd = 1 / ((z - mean).square().mean(-1, keepdim=True) + eps).sqrt()
    xh = (z - mean) * rstd
    shift = N * U * z.abs().mean(-1, keepdim=True)
    er = (N / 2 + 6) * U + 1.5 * N * U * (shift * rstd).square()
    ex = (2 * U + er) * xh.abs() + N * U * (1 + shift * rstd) + 2 * U * shift * rstd
    return mean, rstd, xh, er, ex + 2 * U * xh.abs()


def d64(t):
    return None if t is None else t.detach().cpu().double()


def layer_norm(x, residual, weight, bias, eps):
    """y, z, and the error of y's fp32 arithmetic (before it is rounded to the storage type): that of xh, with
    z = x + residual off by u |z| and with it the mean, and u for the product and for the sum."""
    z = x if residual is None else x + residual
    _, rstd, xh, _, ex = _stats(z, eps)
    if residual is not None:
        ex = ex + U * rstd * (z.abs() + z.abs().mean(-1, keepdim=True)) + U * xh.abs() * rstd * z.abs().amax(-1, keepdim=True)
    w = torch.ones((), dtype=torch.float64) if weight is None else weight
    b = torch.zeros((), dtype=torch.float64) if bias is None else bias
    y = xh * w + b
    return y, z, ex * w.abs() + U * ((xh * w).abs() + y.abs())


def layer_norm_backward(z, weight, dy, dsum, eps):
    """dx, dweight, dbias and the errors of their fp32 arithmetic.

    With g = dy w, dx = rstd (g - a - xh c) + dsum, a = mean g, c = mean(g xh): a is off by (N + 1) u mean|g|, c by
    (N + 2) u mean|g xh| and mean(|g| ex); each product and sum rounds once.  dweight and
    dbias sum rows in any order, at most `rows` additions."""
    rows, d = z.shape
    N = chain(d)
    _, rstd, xh, er, ex = _stats(z, eps)
    g = dy if weight is None else dy * weight
    a, c = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    ln = rstd * (g - a - xh * c)
    dx = ln if dsum is None else ln + dsum
    ga, gx = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True)
    ec = (N + 2) * U * gx + (g.abs() * ex).mean(-1, keepdim=True)
    err = rstd * (4 * U * (g.abs() + a.abs() + (xh * c).abs()) + (N + 1) * U * ga + xh.abs() * ec + ex * (c.abs() + ec))
    err = err + (er + 2 * U) * ln.abs() + U * dx.abs()
    dw, db = (dy * xh).sum(0), dy.sum(0)
    ew = (dy.abs() * ex).sum(0) + (rows + 2) * U * (dy * xh).abs().sum(0)
    eb = rows * U * dy.abs().sum(0)
    return (dx, dw, db), (err, ew, eb)


def embedding(ids, table, scale, pos):
    """y: one product with one sum, rounded once (and once more to 16 bits)."""
    vocab, d = table.shape
    ids = ids.cpu().long()
    ok = (ids >= 0) & (ids < vocab)
    y = torch.zeros(*ids.shape, d, dtype=torch.float64)
    y[ok] = scale * table[ids[ok]]
    if pos is not None:
        y = (y.view(-1, pos.shape[0], d) + pos).view(y.shape)
    return y


def embedding_backward(ids, dy, vocab, scale, n_pos):
    """(dtable, dpos), (their fp32 errors): a sum of k values in any order is off by at most
    k u sum|values|, the product with the scale by u more."""
    ids = ids.cpu().long().view(-1)
    d = dy.shape[-1]
    dy = dy.reshape(-1, d)
    ok = (ids >= 0) & (ids < vocab)
    dtable = torch.zeros(vocab, d, dtype=torch.float64).index_add_(0, ids[ok], dy[ok])
    size = torch.zeros(vocab, d, dtype=torch.float64).index_add_(0, ids[ok], dy[ok].abs())
    count = torch.bincount(ids[ok], minlength=vocab).double()[:, None]
    out, err = [scale * dtable], [abs(scale) * (count + 1) * U * size]
    if n_pos:
        by = dy.view(-1, n_pos, d)
        out.append(by.sum(0))
        err.append(by.shape[0] * U * by.abs().sum(0))
    else:
        out.append(None)
        err.append(None)
    return out, err


def near(name, got, want, err, dtype):
    """got within the fp32 error and half a step of its storage type (fp32: the error holds it)."""
    got = d64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    tol = err + (HALF["bf16"] * (want.abs() + err) if dtype == "bf16" else U * want.abs())
    off = (got - want).abs()
    bad = ~(off <= tol)
    print(f"  {name}: largest part of the bound {float((off / tol.clamp(min=1e-300)).max()) if off.numel() else 0:.3f}", flush=True)
    assert not bad.any(), (name, int(bad.sum()), float((off - tol).max()), [tuple(i.tolist()) for i in bad.nonzero()[:4]])
