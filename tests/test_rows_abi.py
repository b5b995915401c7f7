"""Refusals of the layer norm and the embedding: bad arguments come back as errors before any HIP call.  No call here
reaches a kernel; the device pointers are fake (never dereferenced)."""
import ctypes
import os

import pytest

import paper_2111_09714_amd as Y
from paper_2111_09714_amd import build as ybuild

FAKE = 0x10000  # 16-byte aligned, never dereferenced
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(Y.lib_path()):
        ybuild.build()
    return Y.lib()


def _ln(L, x=FAKE, residual=FAKE, weight=FAKE, bias=FAKE, dtype=0, rows=10, d=768, eps=1e-5, sum=2 * FAKE, y=FAKE):
    return L.yoso_layer_norm(x, residual, weight, bias, dtype, rows, d, eps, sum, y, None)


def _lnb(L, z=FAKE, weight=FAKE, dy=FAKE, dsum=FAKE, dtype=0, rows=10, d=768, eps=1e-5, dx=FAKE, dw=FAKE, db=2 * FAKE, ws=FAKE, wsb=BIG):
    return L.yoso_layer_norm_backward(z, weight, dy, dsum, dtype, rows, d, eps, dx, dw, db, ws, wsb, None)


def _emb(L, ids=FAKE, index=1, table=FAKE, pos=FAKE, dtype=0, tokens=12, n_pos=4, vocab=100, d=64, scale=1.0, y=FAKE):
    return L.yoso_embedding(ids, index, table, pos, dtype, tokens, n_pos, vocab, d, scale, y, None)


def _embb(L, ids=FAKE, index=1, dy=FAKE, dtype=0, tokens=12, n_pos=4, vocab=100, d=64, scale=1.0, dtable=FAKE, dpos=FAKE, ws=FAKE, wsb=BIG):
    return L.yoso_embedding_backward(ids, index, dy, dtype, tokens, n_pos, vocab, d, scale, dtable, dpos, ws, wsb, None)


ROWS = [(dict(dtype=2), 4), (dict(dtype=-1), 4), (dict(d=0), 2), (dict(d=-64), 2), (dict(d=8193), 2), (dict(rows=-1), 2),
        (dict(rows=(1 << 40) + 1), 2), (dict(eps=0.0), 9), (dict(eps=-1e-5), 9), (dict(eps=NAN), 9), (dict(eps=INF), 9),
        (dict(eps=1e-40), 9)]


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(x=None), 1), (dict(y=None), 1), (dict(x=FAKE + 4), 5), (dict(y=FAKE + 8), 5), (dict(residual=FAKE + 2), 5),
    (dict(weight=FAKE + 2), 5), (dict(bias=FAKE + 1), 5), (dict(d=767, x=FAKE + 2), 5),
    (dict(d=770, dtype=1, y=FAKE + 1), 5), (dict(d=6, dtype=1, residual=FAKE + 1), 5), (dict(sum=FAKE + 1), 5), (dict(sum=FAKE, y=FAKE), 9)])
def test_layer_norm_rejects(L, kw, status):
    assert _ln(L, **kw) == status
    assert L.yoso_last_error()


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(z=None), 1), (dict(dy=None), 1), (dict(dx=None), 1), (dict(dw=None), 1), (dict(db=None), 1), (dict(z=FAKE + 8), 5),
    (dict(dy=FAKE + 4), 5), (dict(dx=FAKE + 4), 5), (dict(dsum=FAKE + 4), 5), (dict(weight=FAKE + 2), 5), (dict(dw=FAKE + 2), 5),
    (dict(db=FAKE + 1), 5), (dict(d=767, dx=FAKE + 2), 5), (dict(d=770, dtype=1, z=FAKE + 1), 5), (dict(dw=FAKE, db=FAKE), 9)])
def test_layer_norm_backward_rejects(L, kw, status):
    assert _lnb(L, **kw) == status
    assert L.yoso_last_error()


def test_layer_norm_backward_workspace(L):
    need = Y.yoso_layer_norm_backward_workspace_bytes(100000, 768, Y.F32)
    assert need > 0
    assert _lnb(L, rows=100000, ws=None, wsb=0) == 6
    assert _lnb(L, rows=100000, wsb=need - 1) == 6
    assert _lnb(L, rows=100000, ws=FAKE + 4, wsb=need) == 5
    bad = ctypes.c_size_t(-1).value
    for args in ((-1, 64, 0), (1, 0, 0), (1, 20000, 0), (1, 64, 7)):
        assert L.yoso_layer_norm_backward_workspace_bytes(*args) == bad
        assert L.yoso_last_error()
        with pytest.raises(Y.YosoError):
            Y.yoso_layer_norm_backward_workspace_bytes(*args)


EMB = [(dict(dtype=2), 4), (dict(index=2), 4), (dict(index=-1), 4), (dict(d=0), 2), (dict(d=8193), 2), (dict(vocab=0), 2),
       (dict(vocab=(1 << 20) + 1), 2), (dict(tokens=-1), 2), (dict(tokens=(1 << 27) + 1, n_pos=1), 2), (dict(n_pos=-1), 2), (dict(n_pos=5), 2),
       (dict(n_pos=24), 2), (dict(n_pos=1 << 28), 2), (dict(scale=NAN), 9), (dict(scale=INF), 9), (dict(ids=None), 1), (dict(ids=FAKE + 4), 5), (dict(index=0, ids=FAKE + 2), 5),
       (dict(n_pos=0), 2)]  # positions given, but none counted


@pytest.mark.parametrize("kw,status", EMB + [
    (dict(table=None), 1), (dict(table=FAKE + 4), 5), (dict(pos=None), 1), (dict(pos=FAKE + 4), 5), (dict(y=None), 1), (dict(y=FAKE + 2), 5),
    (dict(d=63, table=FAKE + 2), 5), (dict(d=63, dtype=1, pos=FAKE + 1), 5)])
def test_embedding_rejects(L, kw, status):
    assert _emb(L, **kw) == status
    assert L.yoso_last_error()


@pytest.mark.parametrize("kw,status", EMB + [
    (dict(dy=None), 1), (dict(dy=FAKE + 4), 5), (dict(dtable=None), 1), (dict(dtable=FAKE + 4), 5), (dict(dpos=None), 1), (dict(dpos=FAKE + 2), 5),
    (dict(d=63, dtable=FAKE + 2), 5)])
def test_embedding_backward_rejects(L, kw, status):
    assert _embb(L, **kw) == status
    assert L.yoso_last_error()


def test_embedding_backward_workspace(L):
    need = Y.yoso_embedding_backward_workspace_bytes(5000, 0, 100, 64, Y.F32)
    assert need > 0
    assert _embb(L, tokens=5000, n_pos=0, dpos=None, ws=None, wsb=0) == 6
    assert _embb(L, tokens=5000, n_pos=0, dpos=None, wsb=need - 1) == 6
    assert _embb(L, tokens=5000, n_pos=0, dpos=None, ws=FAKE + 4, wsb=need) == 5
    # a chunk's rows are at most as many as its entries, whatever the vocabulary
    for vocab in (300, 30000, 1 << 20):
        assert Y.yoso_embedding_backward_workspace_bytes(65536, 0, vocab, 768, Y.BF16) < 65536 * (12 + 4 * 768) + (1 << 20)
    assert Y.yoso_embedding_backward_workspace_bytes(512, 0, 30000, 768, Y.F32) == 0
    bad = ctypes.c_size_t(-1).value
    for args in ((-1, 0, 10, 64, 0), (10, 3, 10, 64, 0), (10, 0, 0, 64, 0), (10, 0, 10, 0, 0), (10, 0, 10, 64, 5)):
        assert L.yoso_embedding_backward_workspace_bytes(*args) == bad
        with pytest.raises(Y.YosoError):
            Y.yoso_embedding_backward_workspace_bytes(*args)


def test_no_rows_no_tokens_need_no_pointers(L):
    assert _ln(L, x=None, residual=None, weight=None, bias=None, sum=None, y=None, rows=0) == 0
    assert _lnb(L, z=None, weight=None, dy=None, dsum=None, dx=None, dw=None, db=None, ws=None, wsb=0, rows=0) == 0
    assert _emb(L, ids=None, table=None, pos=None, y=None, tokens=0, n_pos=0) == 0


def test_status_string():
    assert Y.yoso_status_str(9) and Y.STATUS[9] == "YOSO_ERR_VALUE"


def test_binding_refuses_types_and_shapes():
    """What the C ABI cannot see is refused before the call; a host tensor is refused last, so every
    other mistake shows on the CPU."""
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(6, 32), torch.zeros(32)
    h, wh = x.bfloat16(), w.bfloat16()
    for bad in (dict(weight=wh), dict(bias=wh), dict(residual=h), dict(sum=h), dict(y=h)):
        a = dict(weight=w, bias=w, y=x, residual=x, sum=x) | bad
        with pytest.raises(TypeError):
            Y.yoso_layer_norm(x, a["weight"], a["bias"], 1e-5, a["y"], a["residual"], a["sum"])
    for bad in (dict(weight=w[:31]), dict(bias=x), dict(residual=x[:5]), dict(sum=x[:, :31]), dict(y=x[:5])):
        a = dict(weight=w, bias=w, y=x, residual=x, sum=x) | bad
        with pytest.raises(ValueError):
            Y.yoso_layer_norm(x, a["weight"], a["bias"], 1e-5, a["y"], a["residual"], a["sum"])
    for bad in (dict(weight=wh), dict(dy=h), dict(dx=h), dict(dsum=h), dict(dw=wh), dict(db=wh)):
        a = dict(weight=w, dy=x, dx=x, dsum=x, dw=w, db=w) | bad
        with pytest.raises(TypeError):
            Y.yoso_layer_norm_backward(x, a["weight"], a["dy"], 1e-5, a["dx"], a["dw"], a["db"], None, a["dsum"])
    ids, table, y = torch.zeros(2, 3, dtype=torch.int64), torch.zeros(9, 32), torch.zeros(2, 3, 32)
    with pytest.raises(TypeError):
        Y.yoso_embedding(ids, table, 1.0, y.bfloat16())
    with pytest.raises(TypeError):
        Y.yoso_embedding(ids, table, 1.0, y, table.bfloat16())
    for bad in (y[:1], torch.zeros(2, 3, 31), torch.zeros(6, 32)):
        with pytest.raises(ValueError):
            Y.yoso_embedding(ids, table, 1.0, bad)
    with pytest.raises(ValueError):
        Y.yoso_embedding(ids, table[0], 1.0, y)
    with pytest.raises(ValueError):
        Y.yoso_embedding(ids, table, 1.0, y, torch.zeros(3, 31))
    with pytest.raises(TypeError):
        Y.yoso_embedding_backward(ids, y, 1.0, table.bfloat16(), None)
    with pytest.raises(ValueError):
        Y.yoso_embedding_backward(ids, y[:1], 1.0, table, None)
    for kind in (torch.int16, torch.float32, torch.bool):
        with pytest.raises((TypeError, ValueError)):
            Y.yoso_embedding(ids.to(kind), table, 1.0, y)
    for call in (lambda: Y.yoso_layer_norm(x, w, w, 1e-5, x), lambda: Y.yoso_layer_norm_backward(x, w, x, 1e-5, x),
                 lambda: Y.yoso_embedding(ids, table, 1.0, y), lambda: Y.yoso_embedding_backward(ids, y, 1.0, table, None)):
        with pytest.raises(ValueError):
            call()
