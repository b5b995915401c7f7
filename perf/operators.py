"""Performance cases of the operators around the attention: the embedding at an encoder's input and
the layer norm of its residual stream, with their gradients.

Kinds of pass:

  ln       z = x + residual, y = layer norm of z (with z kept where the backward or the next block reads it)
  ln_bwd   its gradients: dx (which is the residual's too), dweight, dbias
  emb      y[t] = scale table[ids[t]] + pos[t mod n]
  emb_bwd  its gradients: dtable (every row), dpos

Sizes are those of workloads.py (12 heads of 64 at 512 tokens and batch 32; two heads of 64 at 4096
tokens and batch 16; 2 x 32768 tokens) and odd ones of the same ranges; vocabularies of subwords (30000) and bytes (256).
Token ids follow a power law, as words do; sequences of a batch are ragged: behind a sequence's end come
padding tokens, either an id outside the vocabulary or an id of their own.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5
_POWER = 3  # id = vocab u^3 of uniform u: the most frequent of 30000 takes 3% of the tokens


def listed():
    return [
        # one token of a serving loop through a post-norm block: latency
        _ln("ln_1x768", rows=1, d=768, residual=True),
        # the residual stream of a batch of 32 x 512 tokens, 16 bits, the sum kept for the backward
        _ln("ln_16384x768_bf16", rows=16384, d=768, dtype="bf16", residual=True, keep=True),
        # a ragged batch packed without padding, at an odd width
        _ln("ln_2999x1001", rows=2999, d=1001),
        # one sequence trained alone
        _ln("ln_bwd_512x768", rows=512, d=768, backward=True),
        # two heads of 64 at 16 x 4096 tokens: many short rows
        _ln("ln_bwd_65536x128", rows=65536, d=128, backward=True),
        # the longest context, 2 x 32768 tokens of 12 heads, with the gradient that passes the norm by
        _ln("ln_bwd_65536x768_bf16", rows=65536, d=768, dtype="bf16", residual=True, keep=True, backward=True),
        # one token of a serving loop: latency
        _emb("emb_1x768", batch=1, n=1, d=768, index="i64"),
        # a batch of 32 x 512 tokens with positions, 16 bits
        _emb("emb_16384x768_bf16", batch=32, n=512, d=768, dtype="bf16", pos=True, pad="ignored"),
        # one sequence trained alone: the whole table's gradient is written for 512 tokens
        _emb("emb_bwd_512x768", batch=1, n=512, d=768, pos=True, backward=True),
        # a batch of 32 x 512 tokens, padding tokens with an id of their own (one long run among short ones)
        _emb("emb_bwd_16384x768", batch=32, n=512, d=768, pos=True, pad="token", backward=True),
        # bytes of 16 x 4096 tokens, two heads of 64: a few hundred rows take all tokens
        _emb("emb_bwd_65536x128_bytes", batch=16, n=4096, d=128, vocab=256, dtype="bf16", pad="ignored", index="i32", backward=True),
        # the longest context, 2 x 32768 tokens
        _emb("emb_bwd_65536x768_bf16", batch=2, n=32768, d=768, dtype="bf16", scale=27.7, backward=True),
    ]


def _ln(name, rows, d, dtype="f32", residual=False, keep=False, backward=False):
    c = {"kind": "ln_bwd" if backward else "ln", "rows": rows, "d": d, "dtype": dtype, "residual": residual, "keep": keep}
    return c if name is None else {"name": name, **c}


def _emb(name, batch, n, d, vocab=30000, dtype="f32", pos=False, pad="none", index="i64", scale=1.0, backward=False):
    c = {"kind": "emb_bwd" if backward else "emb", "batch": batch, "n": n, "d": d, "vocab": vocab, "dtype": dtype, "pos": pos,
         "pad": pad, "index": index, "scale": scale}
    return c if name is None else {"name": name, **c}


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ln", "ln_bwd", "emb", "emb_bwd"])
    dtype = rng.choice(["f32", "bf16"])
    d = _log_int(rng, 32, 4096)
    if rng.random() < 0.5:  # whole heads
        d = 64 * max(1, d // 64)
    # values of one tensor at most: half of the largest listed case's where they have twice the bytes
    most = (65536 * 768) // (2 if dtype == "f32" else 1)
    if kind in ("ln", "ln_bwd"):
        rows = _log_int(rng, 1, min(65536, most // d))
        residual = rng.random() < 0.6
        return _ln(None, rows, d, dtype, residual, residual and rng.random() < 0.7, kind == "ln_bwd")
    vocab = _log_int(rng, 64, min(60000, most // d))
    tokens = _log_int(rng, 1, min(65536, most // d))
    n = _log_int(rng, 1, tokens)
    return _emb(None, max(1, tokens // n), n, d, vocab, dtype, rng.random() < 0.5, rng.choice(["none", "ignored", "token"]),
                rng.choice(["i64", "i32"]), rng.choice([1.0, round(math.sqrt(d), 2)]), kind == "emb_bwd")


# ------------------------------------------------------------------ inputs

def _device():
    return torch.device("cuda", torch.cuda.current_device()) if torch.cuda.is_available() else torch.device("cpu")


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt, d = _DT[case["dtype"]], case["d"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    s = {"case": case}
    if case["kind"] in ("ln", "ln_bwd"):
        rows = case["rows"]
        # the residual stream: rows of different size, some columns far from zero
        column = 1 + 4 * (torch.rand(d, generator=g, device=dev) < 0.01)
        s["x"] = ((normal(rows, d) * column + 0.5 * normal(d)) * (0.2 + 2 * torch.rand(rows, 1, generator=g, device=dev))).to(dt)
        s["weight"], s["bias"] = 1 + 0.2 * normal(d), 0.1 * normal(d)
        if case["kind"] == "ln":
            s["residual"] = normal(rows, d).to(dt) if case["residual"] else None
        else:
            s["dy"] = normal(rows, d).to(dt)
            s["dsum"] = normal(rows, d).to(dt) if case["residual"] and case["keep"] else None
        return s
    batch, n, vocab = case["batch"], case["n"], case["vocab"]
    u = torch.rand(batch, n, generator=g, device=dev, dtype=torch.float64)
    ids = (vocab * u ** _POWER).long().clamp(max=vocab - 1)
    # a power law over shuffled ids: frequent tokens lie anywhere in the table
    ids = torch.randperm(vocab, generator=g, device=dev)[ids]
    if case["pad"] != "none":
        length = (n * (0.4 + 0.6 * torch.rand(batch, 1, generator=g, device=dev))).long() + 1
        behind = torch.arange(n, device=dev) >= length
        ids = torch.where(behind, torch.full_like(ids, -1 if case["pad"] == "ignored" else 0), ids)
    s["ids"] = ids.to(torch.int32 if case["index"] == "i32" else torch.int64)
    if case["kind"] == "emb":
        s["table"] = normal(vocab, d).to(dt)
        s["pos"] = (0.3 * normal(n, d)).to(dt) if case["pos"] else None
    else:
        s["dy"] = normal(batch, n, d).to(dt)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        import paper_2111_09714_amd as Y

        if kind == "ln":
            if s["residual"] is None:
                return Y.layer_norm(s["x"], s["weight"], s["bias"], _EPS)
            y, z = Y.layer_norm(s["x"], s["weight"], s["bias"], _EPS, residual=s["residual"], keep_sum=c["keep"])
            return (y, z) if c["keep"] else y
        if kind == "ln_bwd":
            return Y.layer_norm_backward(s["x"], s["weight"], s["dy"], _EPS, dsum=s["dsum"])
        if kind == "emb":
            return Y.embedding(s["ids"], s["table"], c["scale"], pos=s["pos"])
        dtable, dpos = Y.embedding_backward(s["ids"], s["dy"], c["vocab"], c["scale"], n_pos=c["n"] if c["pos"] else 0)
        return (dtable, dpos) if c["pos"] else dtable
    dt = _DT[c["dtype"]]
    if kind == "ln":
        z = s["x"].float()
        if s["residual"] is not None:
            z = z + s["residual"].float()
        mean = z.mean(-1, keepdim=True)
        xm = z - mean
        y = xm * torch.rsqrt((xm * xm).mean(-1, keepdim=True) + _EPS) * s["weight"] + s["bias"]
        return (y.to(dt), z.to(dt)) if c["keep"] else y.to(dt)
    if kind == "ln_bwd":
        z, dy = s["x"].float(), s["dy"].float()
        xm = z - z.mean(-1, keepdim=True)
        rstd = torch.rsqrt((xm * xm).mean(-1, keepdim=True) + _EPS)
        xh = xm * rstd
        g = dy * s["weight"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return dx.to(dt), (dy * xh).sum(0), dy.sum(0)
    ids, vocab, n = s["ids"].long(), c["vocab"], c["n"]
    valid = (ids >= 0) & (ids < vocab)
    if kind == "emb":
        y = torch.where(valid[..., None], s["table"][ids.clamp(0, vocab - 1)].float() * c["scale"], 0.0)
        return (y if s["pos"] is None else y + s["pos"].float()).to(dt)
    # (tokens without a row add zeros to rows spread over the table)
    dy = s["dy"].float()
    spread = torch.arange(ids.numel(), device=ids.device).view_as(ids) % vocab
    rows = (torch.where(valid[..., None], dy, 0.0) * c["scale"]).view(-1, c["d"])
    dtable = torch.zeros(vocab, c["d"], device=dy.device).index_add_(0, torch.where(valid, ids, spread).view(-1), rows).to(dt)
    return (dtable, dy.sum(0).to(dt)) if c["pos"] else dtable


# ------------------------------------------------------------------ work

def _distinct(tokens, vocab):
    """Expected number of different ids among `tokens` drawn ones."""
    edges = np.power(np.arange(vocab + 1) / vocab, 1 / _POWER)
    return float(np.sum(1 - np.power(1 - np.diff(edges), tokens)))


def work(case):
    """Bytes: inputs read once (of a table, the rows that the tokens name), outputs written once.
    Operations: those of the formulas, a value each."""
    e, d = (2 if case["dtype"] == "bf16" else 4), case["d"]
    if case["kind"] == "ln":
        v = case["rows"] * d
        return {"bytes": e * v * (2 + case["residual"] + case["keep"]) + 8 * d, "flops": v * (8 + case["residual"])}
    if case["kind"] == "ln_bwd":
        v = case["rows"] * d
        dsum = case["residual"] and case["keep"]
        return {"bytes": e * v * (3 + dsum) + 12 * d, "flops": v * (18 + dsum)}
    tokens = case["batch"] * case["n"]
    ids = tokens * (4 if case["index"] == "i32" else 8)
    pos = case["n"] * d if case["pos"] else 0
    if case["kind"] == "emb":
        return {"bytes": ids + e * (d * (_distinct(tokens, case["vocab"]) + tokens) + pos), "flops": tokens * d * (1 + case["pos"])}
    return {"bytes": ids + e * (d * (tokens + case["vocab"]) + pos), "flops": tokens * d * (1 + case["pos"])}


# ------------------------------------------------------------------ exact values

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ln":
        z = s["x"].double()
        if s["residual"] is not None:
            z += s["residual"].double()
        std = (z.var(-1, unbiased=False, keepdim=True) + _EPS).sqrt()
        y = torch.addcmul(s["bias"].double(), (z - z.mean(-1, keepdim=True)) / std, s["weight"].double())
        return (y, z) if case["keep"] else y
    if case["kind"] == "ln_bwd":
        # the Jacobian of a row's norm, applied from its two projections
        z, dy = s["x"].double(), s["dy"].double()
        std = (z.var(-1, unbiased=False, keepdim=True) + _EPS).sqrt()
        h = (z - z.mean(-1, keepdim=True)) / std
        w = s["weight"].double()
        along = torch.matmul((h * dy), w[:, None]) / case["d"]
        level = torch.matmul(dy, w[:, None]) / case["d"]
        dx = (dy * w - level - h * along) / std
        if s["dsum"] is not None:
            dx += s["dsum"].double()
        return dx, torch.einsum("rc,rc->c", dy, h), torch.ones(1, case["rows"], dtype=torch.float64, device=dy.device).matmul(dy)[0]
    ids, vocab, d, n = s["ids"].long().view(-1), case["vocab"], case["d"], case["n"]
    named = torch.nonzero((ids >= 0) & (ids < vocab))[:, 0]
    if case["kind"] == "emb":
        y = torch.zeros(ids.numel(), d, dtype=torch.float64, device=ids.device)
        y[named] = case["scale"] * s["table"].double()[ids[named]]
        y = y.view(case["batch"], n, d)
        if s["pos"] is not None:
            y += s["pos"].double()[None]
        return y
    dy = s["dy"].double()
    dtable = torch.zeros(vocab, d, dtype=torch.float64, device=ids.device)
    dtable.index_put_((ids[named],), dy.view(-1, d)[named], accumulate=True)
    dtable *= case["scale"]
    return (dtable, torch.einsum("bnd->nd", dy)) if case["pos"] else dtable
