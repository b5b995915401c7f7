"""An encoder's ends together, as a training program makes them with one table at both: token ids to rows, layer norm, the loss
of masked tokens, and every gradient back to the table, from the loss and from the lookup.  And a student that learns from a teacher's
top logits through the same rows.  Compared with the same chain in 64 bits, and replayed as a graph."""
import pytest

import loss64
import rows64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402

B, N, D, VOCAB, TOP, EPS = 3, 70, 96, 400, 6, 1e-5


def make():
    g = torch.Generator().manual_seed(23)
    r = lambda *s: torch.randn(*s, generator=g)
    ids = (VOCAB * torch.rand(B, N, generator=g) ** 3).long().clamp(max=VOCAB - 1)
    ids[1, 50:] = -1  # padding names no row
    targets = torch.where((torch.rand(B, N, generator=g) < 0.3) & (ids >= 0), ids, -1)
    return {"ids": ids, "targets": targets, "table": 0.3 * r(VOCAB, D), "pos": 0.3 * r(N, D), "w": 1 + 0.2 * r(D), "b": 0.1 * r(D), "bias": 0.2 * r(VOCAB),
            "top": torch.randint(0, VOCAB, (B, N, TOP), generator=g), "teacher": 2 * r(B, N, TOP), "dloss": 0.5 + torch.rand(B, N, generator=g)}


def step(p, distil):
    e = Y.embedding(p["ids"], p["table"], 1.0, p["pos"])
    x = Y.layer_norm(e, p["w"], p["b"], EPS)
    if distil:
        loss, lse, logq = Y.distillation(x, p["table"], p["top"], p["teacher"], 2.0, p["bias"])
        dx, dtable, dbias = Y.distillation_backward(x, p["table"], p["top"], p["teacher"], logq, lse, p["dloss"], 2.0, p["bias"])
    else:
        loss, lse = Y.cross_entropy(x, p["table"], p["targets"], 0.5, p["bias"])
        dx, dtable, dbias = Y.cross_entropy_backward(x, p["table"], p["targets"], loss, lse, p["dloss"], 0.5, p["bias"])
    de, dw, db = Y.layer_norm_backward(e, p["w"], dx, EPS)
    dt, dpos = Y.embedding_backward(p["ids"], de, VOCAB, 1.0, n_pos=N)
    return {"loss": loss, "dtable": dtable + dt, "dpos": dpos, "dw": dw, "db": db, "dbias": dbias}


def reference(p, distil):
    p = {k: v.double() if v.is_floating_point() else v for k, v in p.items()}
    e = rows64.embedding(p["ids"], p["table"], 1.0, p["pos"]).view(-1, D)
    x = rows64.layer_norm(e, None, p["w"], p["b"], EPS)[0]
    ids, teacher = (p["top"].view(-1, TOP), p["teacher"].view(-1, TOP)) if distil else (p["targets"].view(-1, 1), None)
    (loss, lse, logq), _ = loss64.loss(x, p["table"], p["bias"], 0.5, ids, teacher, 2)
    (dx, dtable, dbias), _ = loss64.gradients(x, p["table"], p["bias"], 0.5, ids, teacher, logq if distil else -loss[:, None], lse, p["dloss"].view(-1), 2)
    (de, dw, db), _ = rows64.layer_norm_backward(e, p["w"], dx, None, EPS)
    (dt, dpos), _ = rows64.embedding_backward(p["ids"], de, VOCAB, 1.0, N)
    return {"loss": loss.view(B, N), "dtable": dtable + dt, "dpos": dpos, "dw": dw, "db": db, "dbias": dbias}


@pytest.mark.parametrize("distil", [False, True])
def test_one_table_at_both_ends(distil):
    p = make()
    got, want = step({k: v.cuda() for k, v in p.items()}, distil), reference(p, distil)
    for k, v in want.items():
        off = float((got[k].double().cpu() - v).norm() / v.norm())
        print(k, off, flush=True)
        # fp32 throughout: products of 96 and 400 values, layer norm's statistics: some 100 roundings of 2^-24 each way at the worst
        assert off <= 1e-5, k


@pytest.mark.parametrize("distil", [False, True])
def test_one_table_at_both_ends_as_a_graph(distil):
    p = {k: v.cuda() for k, v in make().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(p, distil)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(p, distil)
    for rep in range(3):
        p["dloss"].copy_(torch.rand(B, N, generator=torch.Generator().manual_seed(rep)) + 0.1)
        want = step(p, distil)
        torch.cuda.synchronize()
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want), rep
