"""The calls of one encoder layer together, as a training program makes them: token ids and positions to rows, layer
norm, queries, keys and values, YOSO attention, the residual with its layer norm, and all gradients back
to the tables.  Compared with the same chain in 64 bits on the GPU's own hash codes (as the chain of the normalised
attention is), and replayed as a graph, bit for bit."""
import numpy as np
import pytest

import oracle
import rows64
from parity import check_all

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402

EPS = 1e-5
B, N, H, VOCAB, M, TAU, SCALE = 3, 130, 3, 400, 16, 6, 4.0
D = 64 * H


def make():
    g = torch.Generator().manual_seed(41)
    n = lambda *s: torch.randn(*s, generator=g)
    ids = (VOCAB * torch.rand(B, N, generator=g) ** 3).long().clamp(max=VOCAB - 1)
    ids[1, 100:], ids[2, 60:] = -1, -1  # ragged sequences: padding names no row
    p = {"ids": ids, "table": 0.3 * n(VOCAB, D), "pos": 0.3 * n(N, D), "R": n(64, M * TAU), "dy": n(B, N, D)}
    for i in (0, 1):
        p[f"w{i}"], p[f"b{i}"] = 1 + 0.2 * n(D), 0.1 * n(D)
    for s in "qkv":
        p["W" + s] = n(D, D) / D ** 0.5
    return p


def split(x):
    return x.view(B, N, H, 64).transpose(1, 2).reshape(B * H, N, 64).contiguous()


def merge(x):
    return x.view(B, H, N, 64).transpose(1, 2).reshape(B, N, D).contiguous()


def step(p):
    e = Y.embedding(p["ids"], p["table"], SCALE, p["pos"])
    x0 = Y.layer_norm(e, p["w0"], p["b0"], EPS)
    q, k, v = (split(x0.view(-1, D) @ p["W" + s]) for s in "qkv")
    qh, kh = torch.empty_like(q), torch.empty_like(k)
    Y.yoso_l2_normalize(q, qh)
    Y.yoso_l2_normalize(k, kh)
    qc, kc = Y.hash_qk(qh, kh, p["R"], M, TAU)
    a = merge(Y.forward(qc, kc, v, M, TAU))
    y, z = Y.layer_norm(a, p["w1"], p["b1"], EPS, residual=x0)
    dz, dw1, db1 = Y.layer_norm_backward(z, p["w1"], p["dy"], EPS)
    dqh, dkh, dv = Y.backward(qc, kc, qh, kh, v, split(dz), M, TAU)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    Y.yoso_l2_normalize_backward(q, dqh, dq)
    Y.yoso_l2_normalize_backward(k, dkh, dk)
    dx0 = dz.clone()
    grads = {}
    for s, t in (("q", dq), ("k", dk), ("v", dv)):
        t = merge(t).view(-1, D)
        grads["W" + s] = x0.view(-1, D).t() @ t
        dx0 += (t @ p["W" + s].t()).view(B, N, D)
    de, dw0, db0 = Y.layer_norm_backward(e, p["w0"], dx0, EPS)
    dtable, dpos = Y.embedding_backward(p["ids"], de, VOCAB, SCALE, n_pos=N)
    return qc, kc, {"y": y, "dtable": dtable, "dpos": dpos, "dw0": dw0, "db0": db0, "dw1": dw1, "db1": db1, **grads}


def reference(p, qc, kc):
    p = {k: (v if k == "ids" else v.double()) for k, v in p.items()}
    codes = lambda c: np.ascontiguousarray(c.cpu().numpy().view(np.uint16).transpose(0, 2, 1))
    gq, gk = codes(qc), codes(kc)
    t64 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64))
    e = rows64.embedding(p["ids"], p["table"], SCALE, p["pos"])
    x0 = rows64.layer_norm(e.view(-1, D), None, p["w0"], p["b0"], EPS)[0]
    q, k, v = (split(x0 @ p["W" + s]) for s in "qkv")
    qh, kh = (oracle.l2_normalize(x.view(-1, 64).numpy()).reshape(x.shape) for x in (q, k))
    for x, gc in ((qh, gq), (kh, gk)):
        ref, margin = oracle.hash_codes(x, p["R"].numpy(), M, TAU, with_margin=True)
        assert not ((ref != gc) & (margin > 1e-4)).any()
    a = merge(t64(oracle.forward(gq, gk, v.numpy(), M, TAU))).view(-1, D)
    y, z, _ = rows64.layer_norm(a, x0, p["w1"], p["b1"], EPS)
    (dz, dw1, db1), _ = rows64.layer_norm_backward(z, p["w1"], p["dy"].view(-1, D), None, EPS)
    dqh, dkh, dv = oracle.backward(gq, gk, qh, kh, v.numpy(), split(dz.view(B, N, D)).numpy(), M, TAU)
    back = lambda x, g: t64(oracle.l2_normalize_backward(x.view(-1, 64).numpy(), np.asarray(g).reshape(-1, 64))).view(x.shape)
    dx0, grads = dz.clone(), {}
    for s, t in (("q", back(q, dqh)), ("k", back(k, dkh)), ("v", t64(dv))):
        t = merge(t).view(-1, D)
        grads["W" + s] = x0.t() @ t
        dx0 += t @ p["W" + s].t()
    (de, dw0, db0), _ = rows64.layer_norm_backward(e.view(-1, D), p["w0"], dx0, None, EPS)
    (dtable, dpos), _ = rows64.embedding_backward(p["ids"], de, VOCAB, SCALE, N)
    return {"y": y.view(B, N, D), "dtable": dtable, "dpos": dpos, "dw0": dw0, "db0": db0, "dw1": dw1, "db1": db1, **grads}


def test_layer_forward_and_backward():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    p = make()
    qc, kc, got = step({k: v.cuda() for k, v in p.items()})
    want = reference(p, qc, kc)
    host = lambda t: t.double().cpu().numpy().reshape(1, -1, t.shape[-1])
    check_all("encoder layer f32", [(k, host(got[k]), host(want[k])) for k in want], 1e-4)
    absent = torch.ones(VOCAB, dtype=torch.bool)
    absent[p["ids"][p["ids"] >= 0]] = False
    assert not got["dtable"].cpu()[absent].any()


def test_layer_as_a_graph():
    p = {k: v.cuda() for k, v in make().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(p)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(p)[2]
    g = torch.Generator().manual_seed(1)
    for rep in range(3):
        p["dy"].copy_(torch.randn(B, N, D, generator=g))
        want = step(p)[2]
        torch.cuda.synchronize()
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want), rep
