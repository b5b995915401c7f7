"""Refusals of the losses over a vocabulary: bad arguments come back as errors before any HIP call.  No call here reaches
a kernel; the device pointers are fake (never dereferenced).  And their 64-bit reference against differences."""
import ctypes
import os

import pytest

import loss64
import paper_2111_09714_amd as Y
from paper_2111_09714_amd import build as ybuild

FAKE = 0x10000  # 16-byte aligned, never dereferenced
BIG = 1 << 60
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(Y.lib_path()):
        ybuild.build()
    return Y.lib()


def _ce(L, x=FAKE, table=FAKE, bias=FAKE, ids=FAKE, index=1, dtype=0, tokens=10, vocab=100, d=64, scale=1.0, loss=FAKE, lse=2 * FAKE, ws=FAKE,
        wsb=BIG):
    return L.yoso_cross_entropy(x, table, bias, ids, index, dtype, tokens, vocab, d, scale, loss, lse, ws, wsb, None)


def _ceb(L, x=FAKE, table=FAKE, bias=FAKE, ids=FAKE, index=1, loss=FAKE, lse=FAKE, dloss=FAKE, dtype=0, tokens=10, vocab=100, d=64, scale=1.0,
         dx=FAKE, dtable=2 * FAKE, dbias=FAKE, ws=FAKE, wsb=BIG):
    return L.yoso_cross_entropy_backward(x, table, bias, ids, index, loss, lse, dloss, dtype, tokens, vocab, d, scale, dx, dtable, dbias, ws,
                                         wsb, None)


def _kd(L, x=FAKE, table=FAKE, bias=FAKE, ids=FAKE, index=1, teacher=FAKE, dtype=0, tokens=10, top=4, vocab=100, d=64, scale=1.0, loss=FAKE,
        lse=2 * FAKE, logq=3 * FAKE, ws=FAKE, wsb=BIG):
    return L.yoso_distillation(x, table, bias, ids, index, teacher, dtype, tokens, top, vocab, d, scale, loss, lse, logq, ws, wsb, None)


def _kdb(L, x=FAKE, table=FAKE, bias=FAKE, ids=FAKE, index=1, teacher=FAKE, logq=FAKE, lse=FAKE, dloss=FAKE, dtype=0, tokens=10, top=4, vocab=100,
         d=64, scale=1.0, dx=FAKE, dtable=2 * FAKE, dbias=FAKE, ws=FAKE, wsb=BIG):
    return L.yoso_distillation_backward(x, table, bias, ids, index, teacher, logq, lse, dloss, dtype, tokens, top, vocab, d, scale, dx, dtable,
                                        dbias, ws, wsb, None)


ANY = [(dict(dtype=2), 4), (dict(dtype=-1), 4), (dict(index=2), 4), (dict(index=-1), 4), (dict(d=0), 2), (dict(d=-64), 2), (dict(d=8193), 2),
       (dict(vocab=0), 2), (dict(vocab=(1 << 20) + 1), 2), (dict(tokens=-1), 2), (dict(tokens=(1 << 22) + 1), 2), (dict(scale=NAN), 9),
       (dict(scale=INF), 9), (dict(scale=0.0), 9), (dict(x=None), 1), (dict(x=FAKE + 4), 5), (dict(table=None), 1), (dict(table=FAKE + 8), 5),
       (dict(bias=FAKE + 2), 5), (dict(ids=None), 1), (dict(ids=FAKE + 4), 5), (dict(index=0, ids=FAKE + 2), 5), (dict(d=63, x=FAKE + 2), 5),
       (dict(d=63, dtype=1, table=FAKE + 1), 5), (dict(lse=None), 1), (dict(lse=FAKE + 2), 5), (dict(ws=None), 6), (dict(ws=FAKE + 8), 5),
       (dict(wsb=16), 6)]
FWD = [(dict(loss=None), 1), (dict(loss=FAKE + 1), 5), (dict(loss=FAKE, lse=FAKE), 9)]
BWD = [(dict(dloss=None), 1), (dict(dloss=FAKE + 2), 5), (dict(dx=None), 1), (dict(dx=FAKE + 4), 5), (dict(dtable=None), 1),
       (dict(dtable=FAKE + 2), 5), (dict(dbias=FAKE + 1), 5), (dict(d=63, dx=FAKE + 2), 5), (dict(dx=FAKE, dtable=FAKE), 9)]
TOP = [(dict(top=0), 2), (dict(top=-1), 2), (dict(top=1025), 2), (dict(top=(1 << 32) + 4), 2), (dict(teacher=None), 1), (dict(teacher=FAKE + 2), 5),
       (dict(logq=None), 1), (dict(logq=FAKE + 2), 5), (dict(scale=-1.0), 9), (dict(scale=1e-45), 9), (dict(scale=1e39), 9)]


@pytest.mark.parametrize("kw,status", ANY + FWD)
def test_cross_entropy_rejects(L, kw, status):
    assert _ce(L, **kw) == status
    assert L.yoso_last_error()


@pytest.mark.parametrize("kw,status", ANY + BWD + [(dict(loss=None), 1), (dict(loss=FAKE + 1), 5)])
def test_cross_entropy_backward_rejects(L, kw, status):
    assert _ceb(L, **kw) == status
    assert L.yoso_last_error()


@pytest.mark.parametrize("kw,status", ANY + FWD + TOP + [(dict(logq=FAKE), 9), (dict(logq=2 * FAKE), 9)])
def test_distillation_rejects(L, kw, status):
    assert _kd(L, **kw) == status
    assert L.yoso_last_error()


@pytest.mark.parametrize("kw,status", ANY + BWD + TOP)
def test_distillation_backward_rejects(L, kw, status):
    assert _kdb(L, **kw) == status
    assert L.yoso_last_error()


def test_workspace(L):
    f, b = Y.yoso_cross_entropy_workspace_bytes, Y.yoso_cross_entropy_backward_workspace_bytes
    k = lambda n, vocab, d, dt: Y.yoso_distillation_workspace_bytes(n, 4, vocab, d, dt)
    for size, call in ((f, _ce), (b, _ceb), (k, _kd), (b, _kdb)):
        for n in (1, 64, 65, 5000):
            need = size(n, 3000, 96, Y.F32)
            assert need > 0
            assert call(L, tokens=n, vocab=3000, d=96, wsb=need - 1) == 6
    # few tokens, and bf16 rows of whole steps, are read where they lie
    assert f(64, 30000, 768, Y.F32) <= (1 << 20) + 256 and f(512, 30000, 768, Y.BF16) <= 1 << 21
    # G is at most 1 GiB (or 256 entries), beside copies of x and table, fp32 parts of dx and dtable and sums of db
    for n, vocab, d, dt, e in ((65536, 30000, 768, Y.BF16, 2), (65536, 30000, 768, Y.F32, 4), (1 << 22, 1 << 16, 64, Y.F32, 4)):
        g = max(1 << 30, 256 * e * n)
        rows = (n + 255) // 256 * 256
        assert b(n, vocab, d, dt) <= g + (rows + vocab + 256) * (d + 127) // 128 * 128 * e + rows * (d + 127) // 128 * 128 * 4 + (3 << 26) + g // 16 + 64 * (n + vocab)
    assert Y.yoso_distillation_workspace_bytes(5000, 64, 3000, 96, Y.F32) <= f(5000, 3000, 96, Y.F32) + 5000 * 272
    bad = ctypes.c_size_t(-1).value
    for args in ((10, 0, 10, 64, 0), (10, 1025, 10, 64, 0), (-1, 1, 10, 64, 0), (10, 1, 10, 64, 5)):
        assert L.yoso_distillation_workspace_bytes(*args) == bad
    for fn, raw in ((f, L.yoso_cross_entropy_workspace_bytes), (b, L.yoso_cross_entropy_backward_workspace_bytes)):
        for args in ((-1, 10, 64, 0), (10, 0, 64, 0), (10, 10, 0, 0), (10, 10, 8193, 0), (10, 10, 64, 5), ((1 << 22) + 1, 10, 64, 0)):
            assert raw(*args) == bad
            with pytest.raises(Y.YosoError):
                fn(*args)


def test_no_tokens_need_no_pointers(L):
    assert _ce(L, x=None, table=None, bias=None, ids=None, loss=None, lse=None, ws=None, wsb=0, tokens=0) == 0
    assert _kd(L, x=None, table=None, bias=None, ids=None, teacher=None, loss=None, lse=None, logq=None, ws=None, wsb=0, tokens=0) == 0
    # (the backward still writes dtable)
    assert _ceb(L, tokens=0, table=None) == 1 and _ceb(L, tokens=0, dtable=None) == 1 and _kdb(L, tokens=0, dtable=None) == 1


def test_binding_refuses_types_and_shapes():
    """What the C ABI cannot see is refused before the call; a host tensor is refused last."""
    torch = pytest.importorskip("torch")
    f32 = torch.float32
    x, table, bias = torch.zeros(2, 3, 32), torch.zeros(9, 32), torch.zeros(9)
    ids, top = torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3, 4, dtype=torch.int64)
    row, lst = torch.zeros(2, 3), torch.zeros(2, 3, 4)
    calls = {
        "ce": (lambda a: Y.yoso_cross_entropy(a["x"], a["table"], a["ids"], 1.0, a["loss"], a["lse"], None, a["bias"]), ids),
        "ceb": (lambda a: Y.yoso_cross_entropy_backward(a["x"], a["table"], a["ids"], a["loss"], a["lse"], a["dloss"], 1.0, a["dx"], a["dtable"], None,
                                                        a["dbias"], a["bias"]), ids),
        "kd": (lambda a: Y.yoso_distillation(a["x"], a["table"], a["ids"], a["teacher"], 1.0, a["loss"], a["lse"], a["logq"], None, a["bias"]), top),
        "kdb": (lambda a: Y.yoso_distillation_backward(a["x"], a["table"], a["ids"], a["teacher"], a["logq"], a["lse"], a["dloss"], 1.0, a["dx"],
                                                       a["dtable"], None, a["dbias"], a["bias"]), top)}
    reads = {"ce": "x table bias ids loss lse", "ceb": "x table bias ids loss lse dloss dx dtable dbias", "kd": "x table bias ids teacher loss lse logq",
             "kdb": "x table bias ids teacher logq lse dloss dx dtable dbias"}
    for name, (call, named) in calls.items():
        good = dict(x=x, table=table, bias=bias, ids=named, loss=row, lse=row, dloss=row, teacher=lst, logq=lst, dx=x, dtable=table, dbias=bias)
        with pytest.raises(ValueError):
            call(good)  # on the host
        for arg in reads[name].split():
            t = good[arg]
            for wrong in (t[..., :-1], t[:1].contiguous() if arg != "x" else t[..., :31], t.unsqueeze(0) if arg not in ("x", "ids") else t[..., :1]):
                if wrong.shape == t.shape:
                    continue
                with pytest.raises(ValueError):
                    call(good | {arg: wrong})
            with pytest.raises((TypeError, ValueError)):
                call(good | {arg: t.to(torch.int16 if arg == "ids" else torch.float64)})
            if arg not in ("ids", "x"):
                with pytest.raises(TypeError):
                    call(good | {arg: t.bfloat16()})
            with pytest.raises(ValueError):
                call(good | {arg: torch.stack((t, t), -1)[..., 0]})  # not contiguous
    with pytest.raises(Y.YosoError):
        Y.yoso_cross_entropy_workspace_bytes(4, 9, (1 << 32) + 64, Y.F32)


@pytest.mark.parametrize("top", [0, 5])
def test_reference_gradients_are_those_of_the_reference_loss(top):
    """Central differences of the 64-bit loss along random directions: off by h^2 third derivatives (h = 2^-14, of order 1
    to 100 here) and by 2^-52 / h, so by less than 1e-6 of the sums' size."""
    torch = pytest.importorskip("torch")
    g = torch.Generator().manual_seed(7 + top)
    n, vocab, d, scale = 20, 30, 12, 0.7
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x, w, b, dl = r(n, d), 0.5 * r(vocab, d), 0.3 * r(vocab), r(n)
    ids = torch.randint(-3, vocab + 2, (n, max(1, top)), generator=g)
    teacher = r(n, top) if top else None
    if top:
        teacher[0] = -float("inf")  # no entry left: takes no part
        teacher[1, :2] = -float("inf")
        ids[2, 1] = ids[2, 0]
    value = lambda x, w, b: (loss64.loss(x, w, b, scale, ids, teacher, 2)[0][0] * dl).sum()
    (l, lse, logq), _ = loss64.loss(x, w, b, scale, ids, teacher, 2)
    grads, _ = loss64.gradients(x, w, b, scale, ids, teacher, logq if top else -l[:, None], lse, dl, 2)
    h = 2.0 ** -14
    for i, (t, gt) in enumerate(zip((x, w, b), grads)):
        for _ in range(3):
            u = r(*t.shape)
            args = [x, w, b]
            args[i] = t + h * u
            up = value(*args)
            args[i] = t - h * u
            want = (up - value(*args)) / (2 * h)
            assert abs(float(want - (gt * u).sum())) < 1e-6 * float((gt * u).abs().sum() + 1)
