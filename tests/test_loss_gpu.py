"""Cross entropy over a vocabulary and distillation from a teacher's top logits, with their gradients, against plain sums in 64
bits (tests/loss64.py, which derives the bounds)."""
import math

import pytest

import loss64
from rows64 import DT, near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402


def make(n, vocab, d, dtype, top=0, bias=True, seed=0, index=torch.int64, share=0.7, size=1.0):
    g = torch.Generator().manual_seed(1000 * seed + 7 * n + vocab + d)
    r = lambda *s: torch.randn(*s, generator=g)
    s = {"x": (r(n, d) * size).to(DT[dtype]), "table": (r(vocab, d) * (0.3 + torch.rand(vocab, 1, generator=g)) / (size * d ** 0.5)).to(DT[dtype]),
         "bias": 0.5 * r(vocab) if bias else None, "dloss": 0.5 + torch.rand(n, generator=g)}
    k = max(1, top)
    ids = torch.randint(0, vocab, (n, k), generator=g)
    out = torch.rand(n, 1, generator=g) >= share
    ids = torch.where(out, torch.tensor([-1, vocab, -100, 2 ** 31 - 1])[torch.randint(0, 4, (n, k), generator=g)], ids)
    s["ids"] = ids.to(index)
    s["teacher"] = 3 * r(n, k) if top else None
    return s


def cuda(s):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in s.items()}


def planes(dtype):
    return 1 if dtype == "bf16" else 2


def forward(c, scale):
    if c["teacher"] is None:
        loss, lse = Y.cross_entropy(c["x"], c["table"], c["ids"][:, 0].contiguous(), scale, c["bias"])
        return loss, lse, -loss[:, None]
    return Y.distillation(c["x"], c["table"], c["ids"], c["teacher"], 1 / scale, c["bias"])


def backward(c, scale, logq, lse):
    if c["teacher"] is None:
        return Y.cross_entropy_backward(c["x"], c["table"], c["ids"][:, 0].contiguous(), -logq[:, 0], lse, c["dloss"], scale, c["bias"])
    return Y.distillation_backward(c["x"], c["table"], c["ids"], c["teacher"], logq, lse, c["dloss"], 1 / scale, c["bias"])


def as64(s):
    return {k: (v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v) for k, v in s.items()}


def check(s, dtype, scale=1.0):
    e = as64(s)
    ids = s["ids"].long()
    c = cuda(s)
    print(f"n {s['x'].shape[0]} vocab {s['table'].shape[0]} d {s['x'].shape[1]} {dtype} top {ids.shape[1]}", flush=True)
    got = forward(c, scale)
    torch.cuda.synchronize()
    want, err = loss64.loss(e["x"], e["table"], e["bias"], scale, ids, e["teacher"], planes(dtype))
    for name, a, b, t in zip(("loss", "lse", "logq"), got, want, err):
        if name != "logq" or s["teacher"] is not None:
            near(name, a, b, t, "f32")
    # what the forward left, as the reference rounds it
    logq = (want[2] if s["teacher"] is not None else -want[0][:, None]).float()
    lse = want[1].float()
    grads = backward(c, scale, logq.cuda(), lse.cuda())
    torch.cuda.synchronize()
    wantg, errg = loss64.gradients(e["x"], e["table"], e["bias"], scale, ids, e["teacher"], logq.double(), lse.double(), e["dloss"], planes(dtype))
    near("dx", grads[0], wantg[0], errg[0], dtype)
    near("dtable", grads[1], wantg[1], errg[1], dtype)
    if s["bias"] is not None:
        near("dbias", grads[2], wantg[2], errg[2], "f32")
    else:
        assert grads[2] is None


SHAPES = [(1, 1, 1), (1, 40, 64), (2, 1100, 1024), (9, 9000, 260), (31, 700, 257), (20, 8300, 1020), (32, 300, 1001), (33, 300, 1024), (20, 90, 1025), (3, 17, 33), (16, 257, 96), (17, 500, 128), (40, 300, 200), (64, 1000, 100), (65, 256, 64), (70, 129, 32),
          (100, 1, 40), (127, 2000, 96), (128, 255, 160), (129, 512, 128), (300, 77, 65), (500, 1003, 300), (1025, 300, 64), (2100, 130, 31),
          (16, 260, 2048), (9, 700, 1100), (16, 40, 2049), (1, 33, 1501)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d", SHAPES)
def test_cross_entropy(n, vocab, d, dtype):
    check(make(n, vocab, d, dtype, bias=(n + d) % 2 == 0, index=torch.int32 if n % 2 else torch.int64), dtype, 1.0 if n % 3 else 0.37)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,top", [(1, 40, 64, 1), (5, 300, 33, 7), (1, 500, 300, 1024), (16, 20, 72, 64), (32, 600, 700, 32), (32, 600, 70, 33), (64, 500, 96, 64), (65, 500, 96, 3), (130, 90, 128, 20), (300, 1100, 50, 65),
                                           (700, 3, 64, 8), (1100, 260, 256, 33), (40, 50, 64, 300), (90, 900, 96, 1000), (3000, 150, 300, 64), (5000, 1500, 70, 63), (2000, 40, 2080, 5),
                                           (16, 30, 2048, 64), (7, 200, 1500, 9), (4000, 97, 65, 40)])
def test_distillation(n, vocab, d, top, dtype):
    check(make(n, vocab, d, dtype, top=top, bias=n % 2 == 0, index=torch.int32 if n % 2 else torch.int64), dtype, 0.5)


# more tokens than one workgroup lists, than the loss takes a workgroup each; bf16 rows laid out; whole and half tiles
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,top", [(9001, 300, 32, 0), (8193, 70, 40, 9), (4500, 50000, 32, 0), (2000, 257, 1100, 0), (200, 100, 2080, 3)])
def test_more_tokens_and_columns(n, vocab, d, top, dtype):
    # (the reference takes n x vocab values: a sample of the larger ones)
    s = make(n, vocab, d, dtype, top=top, share=0.02 if n * vocab > 10 ** 8 else 0.9)
    if n * vocab <= 10 ** 8:
        return check(s, dtype)
    part = ((s["ids"] >= 0) & (s["ids"] < vocab)).any(1).nonzero()[:, 0]
    few = {k: (v[part] if k in ("x", "ids", "dloss") else v) for k, v in s.items()}
    c, e = cuda(s), as64(few)
    loss, lse, _ = forward(c, 1.0)
    want, err = loss64.loss(e["x"], e["table"], e["bias"], 1.0, few["ids"].long(), None, planes(dtype))
    near("loss", loss[part.cuda()], want[0], err[0], "f32")
    near("lse", lse[part.cuda()], want[1], err[1], "f32")
    rest = torch.ones(n, dtype=torch.bool)
    rest[part] = False
    assert not loss.cpu()[rest].any() and not lse.cpu()[rest].any()
    logq, z = -want[0][:, None].float(), torch.full((n,), math.nan)
    all_loss, all_lse = z.clone(), z.clone()
    all_loss[part], all_lse[part] = want[0].float(), want[1].float()
    grads = backward(c, 1.0, -all_loss[:, None].cuda(), all_lse.cuda())
    wantg, errg = loss64.gradients(e["x"], e["table"], e["bias"], 1.0, few["ids"].long(), None, logq.double(), lse.cpu()[part].double() * 0 + want[1].float().double(),
                                   e["dloss"], planes(dtype))
    near("dx", grads[0][part.cuda()], wantg[0], errg[0], dtype)
    near("dtable", grads[1], wantg[1], errg[1], dtype)
    near("dbias", grads[2], wantg[2], errg[2], "f32")
    assert not grads[0].cpu()[rest].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("n", [20, 300])
def test_tokens_that_take_no_part(n, top, dtype):
    """NaN and infinities in rows of x without a target (and in the backward in those with dloss 0) reach nothing; a teacher's
    logit of -inf is left out, and so is a row that has no other; a bias of -inf takes an entry out."""
    vocab, d = 180, 64
    s = make(n, vocab, d, dtype, top=top, share=0.6, seed=3)
    s["bias"][7] = -math.inf
    s["ids"][s["ids"] == 7] = 8
    s["ids"][0] = 5
    s["dloss"][0] = 1.0
    if top:
        s["teacher"][torch.rand(n, top, generator=torch.Generator().manual_seed(1)) < 0.3] = -math.inf
        s["teacher"][4] = -math.inf
        s["teacher"][0, 0] = 1.0
    part = loss64._named(s["ids"].long(), vocab, s["teacher"]).any(1)
    clean = {k: v for k, v in s.items()}
    check(clean, dtype, 0.5)
    dirty = dict(s, x=s["x"].clone())
    dirty["x"][~part] = torch.tensor([math.nan, math.inf, -math.inf, 1.0]).repeat(d // 4).to(DT[dtype])
    a, b = forward(cuda(clean), 0.5), forward(cuda(dirty), 0.5)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    if top:
        assert not a[2].cpu()[~loss64._named(s["ids"].long(), vocab, s["teacher"])].any()
    assert not a[0].cpu()[~part].any() and not a[1].cpu()[~part].any()
    # rows with dloss 0 too
    clean["dloss"] = dirty["dloss"] = torch.where(torch.arange(n) % 5 == 1, 0.0, s["dloss"])
    dirty["x"][(clean["dloss"] == 0)] = math.nan
    ga = backward(cuda(clean), 0.5, a[2], a[1])
    gb = backward(cuda(dirty), 0.5, a[2], a[1])
    assert all(torch.equal(x, y) for x, y in zip(ga, gb))
    out = ~part | (clean["dloss"] == 0)
    assert not ga[0].cpu()[out].any() and not ga[1].cpu()[7].any()
    assert all(torch.isfinite(t).all() for t in ga)
    # a NaN in a row with a target: that token's loss alone
    dirty = dict(s, x=s["x"].clone())
    dirty["x"][0, 3] = math.nan
    c = forward(cuda(dirty), 0.5)
    assert torch.isnan(c[0][0]) and torch.equal(c[0][1:], a[0][1:]) and torch.equal(c[1][1:], a[1][1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,top", [(20, 6), (40, 6), (300, 6), (300, 70)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_teachers_logit_that_is_no_number(n, top, dtype, bad):
    """Of token 9 alone: its loss, dx, and the taught ids' rows of dtable and dbias are NaN, every other value is as without it."""
    vocab, d = 400, 64
    s = make(n, vocab, d, dtype, top=top, share=0.6, seed=5)
    s["ids"][9] = torch.arange(top) * 3
    s["dloss"][9] = 1.0
    a = forward(cuda(s), 0.5)
    ga = backward(cuda(s), 0.5, a[2], a[1])
    dirty = dict(s, teacher=s["teacher"].clone())
    dirty["teacher"][9, 2] = bad
    b = forward(cuda(dirty), 0.5)
    gb = backward(cuda(dirty), 0.5, a[2], a[1])
    other = torch.arange(n) != 9
    assert torch.isnan(b[0][9]) and torch.equal(a[0].cpu()[other], b[0].cpu()[other])
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert torch.isnan(gb[0][9]).all() and torch.equal(ga[0].cpu()[other], gb[0].cpu()[other])
    rest = ~torch.isin(torch.arange(vocab), s["ids"][9])
    for x, y in zip(ga[1:], gb[1:]):
        assert torch.isnan(y.cpu()[~rest]).all() and torch.equal(x.cpu()[rest], y.cpu()[rest])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 3])
def test_no_token_takes_part_and_no_tokens(top, dtype):
    s = cuda(make(100, 90, 48, dtype, top=top, share=0.0))
    loss, lse, logq = forward(s, 1.0)
    assert not loss.any() and not lse.any()
    for t in backward(s, 1.0, logq, lse):
        assert not t.any()
    e = {k: (v[:0] if k in ("x", "ids", "dloss", "teacher") and v is not None else v) for k, v in s.items()}
    loss, lse, logq = forward(e, 1.0)
    dx, dw, db = backward(e, 1.0, logq, lse)
    assert dx.shape == (0, 48) and not dw.any() and not db.any()


def test_rows_at_any_element_and_odd_shapes():
    """Rows that are no whole vectors start at any element; tokens in more dimensions; one token without any."""
    s = make(24, 61, 37, "bf16", top=4)
    want = forward(cuda(s), 0.5)
    x = torch.empty(24 * 37 + 3, dtype=torch.bfloat16, device="cuda")[3:].view(2, 12, 37).copy_(s["x"].view(2, 12, 37))
    w = torch.empty(61 * 37 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(61, 37).copy_(s["table"])
    ids, teacher = s["ids"].cuda().view(2, 12, 4), s["teacher"].cuda().view(2, 12, 4)
    got = Y.distillation(x, w, ids, teacher, 2.0, s["bias"].cuda())
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))
    g = Y.distillation_backward(x, w, ids, teacher, got[2], got[1], s["dloss"].cuda().view(2, 12), 2.0, s["bias"].cuda())
    ref = backward(cuda(s), 0.5, want[2], want[1])
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(g, ref))
    one = Y.distillation(x[0, 0], w, ids[0, 0], teacher[0, 0], 2.0, s["bias"].cuda())
    assert one[0].shape == () and one[2].shape == (4,)
    assert abs(float(one[0]) - float(want[0][0])) <= 1e-5 * (1 + abs(float(want[0][0])))


def test_pieces_of_the_vocabulary():
    """G of 2100 x 300000 fp32 takes three pieces; compared with sums in 64 bits on the GPU, blocks of the vocabulary at a time.

    Logits up to about 14, off by 2^-24 of that each way, put 2e-6 on a probability, operands 2^-22 and parts of sums 60 roundings: 1e-5
    of each sum's size.  G's planes: the lower half's smallest step is 2^-24, half of it 2^-25 of Gs, whose largest is at most 2^14:
    2^-39 2^e max(sw) / (sx_t sw_v) of G with 2^e <= 2 max(dloss sx).  sx 2^14 <= max|x_t| < sx 2^15, sw alike, so at most
    2^-36 max(dloss max|x|) max|table| / (max|x_t| max|table_v|), times |x_t| over n tokens or |table_v| over the vocabulary."""
    n, vocab, d, top = 2100, 300000, 8, 5
    s = cuda(make(n, vocab, d, "f32", top=top, share=0.9))
    loss, lse, logq = forward(s, 1.0)
    dx, dw, db = backward(s, 1.0, logq, lse)
    x, w, b = s["x"].double(), s["table"].double(), s["bias"].double()
    ok = (s["ids"] >= 0) & (s["ids"] < vocab)
    p = torch.softmax(s["teacher"].double().masked_fill(~ok, -1e300), 1) * ok
    dl = torch.where(ok.any(1), s["dloss"].double(), 0.0)
    wx, sx, z, ww, sw, wb, sb = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(n, dtype=torch.float64, device="cuda"), [], [], [], []
    for v in range(0, vocab, 50000):
        r = slice(v, v + 50000)
        l = x @ w[r].t().contiguous() + b[r]
        z += torch.exp(l).sum(1)
        q = torch.exp(l - lse.double()[:, None])
        here = ok & (s["ids"] >= v) & (s["ids"] < v + 50000)
        t = torch.zeros_like(q).scatter_add_(1, torch.where(here, s["ids"] - v, 0), p * here)
        g, size = dl[:, None] * (q - t), dl[:, None] * (q + t)
        wx += g @ w[r]
        sx += size @ w[r].abs()
        ww.append(g.t().contiguous() @ x)
        sw.append(size.t().contiguous() @ x.abs())
        wb.append(g.sum(0))
        sb.append(size.sum(0))
    part = ok.any(1)
    assert float((lse.double() - torch.log(z))[part].abs().max()) <= 2e-6 * 14
    mx, mw = x.abs().amax(1, keepdim=True), w.abs().amax(1, keepdim=True)
    floor = 2.0 ** -36 * float((dl[:, None] * mx).max()) * float(mw.max())
    for name, got, want, size, least in (("dx", dx, wx, sx, floor * vocab / mx), ("dtable", dw, torch.cat(ww), torch.cat(sw), floor * n / mw),
                                         ("dbias", db, torch.cat(wb), torch.cat(sb), 2.0 ** -39 * float(dl.max()) * n * top)):
        off = ((got.double() - want).abs() - (1e-5 * size + least)).max()
        assert float(off) <= 0, (name, float(off))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_calls_and_another_stream(dtype):
    """The same bits every time, on whichever stream, beside other work."""
    s = cuda(make(700, 900, 96, dtype, top=7))
    ref = forward(s, 0.5)
    refg = backward(s, 0.5, ref[2], ref[1])
    other = cuda(make(700, 900, 96, dtype, seed=5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            a = forward(s, 0.5)
            g = backward(s, 0.5, a[2], a[1])
        o = forward(other, 1.0)
        backward(other, 1.0, o[2], o[1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + g, ref + refg))


@pytest.mark.parametrize("dtype,n", [("f32", 40), ("bf16", 700), ("f32", 9000)])
def test_as_a_graph(dtype, n):
    """Forward and backward captured once and replayed with other inputs, eager calls in between."""
    s = cuda(make(n, 500, 64, dtype, top=5))
    out = {}

    def step():
        loss, lse, logq = forward(s, 0.5)
        return (loss, lse, logq, *backward(s, 0.5, logq, lse))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for rep in range(3):
        for k, v in cuda(make(n, 500, 64, dtype, top=5, seed=rep + 10, share=0.3 + 0.3 * rep)).items():
            s[k].copy_(v)
        want = step()
        torch.cuda.synchronize()
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), rep


def test_cross_entropy_is_distillation_from_a_certain_teacher():
    """One id with any logit has probability 1: the same loss, log q and gradients as cross entropy up to the last bits.

    lse: the two calls join a row's parts (5 tiles of 128 entries and two halves of each) in their own orders, at most 12 joins of six
    roundings of 2^-24 of the sum, and round values up to 8 four times: 7e-6.  The target's logit is the tile's there and a dot
    product here: chain(64) + 17 roundings of its sum of |x||w|."""
    s = cuda(make(400, 600, 64, "f32"))
    loss, lse, _ = forward(s, 1.0)
    s["teacher"] = torch.randn(400, 1, device="cuda")
    l2, lse2, logq = forward(s, 1.0)
    ids = s["ids"][:, 0].clamp(0, 599)
    near_lse = 7e-6
    near_loss = near_lse + (loss64.chain(64, 2) + 17 + 12) * loss64.U * (s["x"] * s["table"][ids]).abs().sum(1).double()
    assert float((lse - lse2).abs().max()) <= near_lse
    assert ((loss - l2).double().abs() <= near_loss).all() and torch.allclose(l2, -logq[:, 0], rtol=1e-6, atol=1e-6)
    a = Y.cross_entropy_backward(s["x"], s["table"], s["ids"][:, 0].contiguous(), loss, lse, s["dloss"], 1.0, s["bias"])
    b = Y.distillation_backward(s["x"], s["table"], s["ids"], s["teacher"], -loss[:, None].contiguous(), lse, s["dloss"], 1.0, s["bias"])
    for x, y in zip(a, b):
        assert float((x - y).abs().max()) <= 2.0 ** -20 * float(x.abs().max())


def test_scales_of_rows():
    """Rows of x and of the table 2^12 apart, in either direction, tokens' weights 2^10: within the bounds."""
    s = make(200, 300, 64, "f32", share=1.0)
    g = torch.Generator().manual_seed(2)
    k = torch.randint(-6, 7, (200, 1), generator=g).float()
    s["x"] *= 2.0 ** k / 2.0 ** 6
    s["table"] *= 2.0 ** torch.randint(-6, 7, (300, 1), generator=g).float()
    s["dloss"] *= 2.0 ** torch.randint(-5, 6, (200,), generator=g).float()
    check(s, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 3])
def test_rows_of_zeros(top, dtype):
    """Rows of zeros in x and in the table have gradients as exact as the others', beside rows as small as 2^-20."""
    s = make(300, 200, 96, dtype, top=top, share=0.9, seed=9)
    s["x"] *= 2.0 ** -20
    s["table"] *= 2.0 ** -20
    s["x"][::7] = 0
    s["table"][::5] = 0
    s["x"][3], s["table"][11] = -0.0, -0.0
    check(s, dtype, 2.0 ** 40 if not top else 2.0 ** 39)  # (logits of 2^40, from the bias)
    if top:
        s["teacher"] *= 2.0 ** -39
    check(dict(s, bias=None), dtype, 2.0 ** 40 if not top else 2.0 ** 39)
    s["x"][:] = 0
    check(s, dtype)
    s["table"][:] = 0
    check(s, dtype)


@pytest.mark.parametrize("n,vocab,d,dtype,top", [((1 << 22) - 3, 20, 3, "f32", 0), (1 << 22, 9, 2, "bf16", 3), (70, (1 << 20) - 1, 5, "f32", 0),
                                                 (100, 1 << 20, 8, "bf16", 2), (12, 1 << 20, 8, "f32", 1), (80, 40, 8192, "f32", 0)])
def test_largest_sizes(n, vocab, d, dtype, top):
    """The limits of each size: offsets past 2^32 bytes in G and in x's planes, 2^20 entries, 8192 columns.  Compared with sums in 64
    bits on the GPU.  u = 2^-24: logits are off by 400 u (chain(8192) is 1600, of products that add up to about 1), sums of K products by
    chain(K / parts) + parts, at most 3 (2^22 / 16 / 512 + 16) + 512 = 2100 u of the sum of sizes; fp16 planes of G 2^-11 of each value (bf16)."""
    s = cuda(make(n, vocab, d, dtype, top=top, share=0.8, index=torch.int32))
    loss, lse, logq = forward(s, 1.0)
    dx, dw, db = backward(s, 1.0, logq, lse)
    torch.cuda.synchronize()
    x, w, b, ids = s["x"].double(), s["table"].double(), s["bias"].double(), s["ids"].long()
    ok = (ids >= 0) & (ids < vocab)
    part = ok.any(1)
    p = torch.softmax(s["teacher"].double().masked_fill(~ok, -1e300), 1) * ok if top else ok.double()
    dl = torch.where(part, s["dloss"].double(), 0.0)
    u, half = 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 0.0
    g_off = 2.0 ** -11 if dtype == "bf16" else 1e-5
    ww, sw = torch.zeros_like(w), torch.zeros_like(w)
    wb, sb = torch.zeros_like(b), torch.zeros_like(b)
    step = max(1, (1 << 24) // vocab)
    least = 2.0 ** -36 * float((dl * x.abs().amax(1)).max()) * float(w.abs().max())
    for a in range(0, n, step):
        r = slice(a, a + step)
        l = x[r] @ w.t().contiguous() + b
        z = torch.logsumexp(l, 1)
        at = torch.where(ok[r], ids[r], 0)
        q = l.gather(1, at) - z[:, None]
        want = torch.where(ok[r] & (p[r] > 0), p[r] * (torch.log(p[r].clamp(min=1e-300)) - q), 0.0).sum(1)
        size = 1 + l.abs().amax(1)
        assert ((loss[r] - want).abs() <= 1700 * u * size).all()
        assert ((lse[r] - torch.where(part[r], z, 0.0)).abs() <= 1700 * u * size).all()
        prob = torch.exp(l - z[:, None])
        taught = torch.zeros_like(prob).scatter_add_(1, at, p[r] * ok[r])
        g, gs = dl[r, None] * (prob - taught), dl[r, None] * (prob + taught) * (1700 * u * size[:, None] + g_off + 2100 * u)
        e = (gs + 2100 * u * g.abs()) @ w.abs() + least * vocab / x[r].abs().amax(1, keepdim=True) + half * (g @ w).abs()
        assert ((dx[r] - g @ w).abs() <= e).all()
        ww += g.t().contiguous() @ x[r]
        sw += gs.t().contiguous() @ x[r].abs()
        wb += g.sum(0)
        sb += (dl[r, None] * (prob + taught) * (1700 * u * size[:, None] + 100 * u)).sum(0)
    assert ((dw - ww).abs() <= sw + half * ww.abs() + least * n / w.abs().amax(1, keepdim=True)).all()
    assert ((db - wb).abs() <= sb + u * wb.abs() + 2.0 ** -39 * n).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d", [(5, 900, 128), (64, 3000, 96), (200, 900, 128), (700, 2000, 64)])
def test_losses_near_zero(n, vocab, d, dtype):
    """Tokens whose target has nearly all probability: loss = log(1 + rest), rest = sum exp(l - l_y) of the other entries.  The logits of the
    token are all off by less than `le`, so rest by 2 le of itself and 4 u for the exponentials; 1 + rest rounds at up to 40 + vocab / 128
    sums (a part at a time) and joins, each by u, and the logarithm by 4 u: not by a step of lse."""
    s = make(n, vocab, d, dtype, bias=False, share=1.0, seed=4)
    s["table"] = (s["table"].float() * 3).to(DT[dtype])
    y = s["ids"][:, 0]
    w = s["table"].float()[y]
    s["x"] = (s["x"].float() * 0.1 + w * (torch.linspace(8, 24, n)[:, None] / w.square().sum(1, keepdim=True))).to(DT[dtype])
    e = as64(s)
    l, le = loss64.logits(e["x"], e["table"], None, 1.0, planes(dtype))
    z = torch.logsumexp(l, 1)
    at = l.gather(1, y[:, None])[:, 0]
    rest = torch.exp(l - at[:, None]).scatter_(1, y[:, None], 0.0).sum(1)
    assert float(rest.min()) < 1e-4
    loss, lse, _ = forward(cuda(s), 1.0)
    want = torch.log1p(rest)
    bound = rest * (2 * le.amax(1) + 4 * loss64.U) + (44 + vocab / 128) * loss64.U * (1 + rest)
    off = (loss.double().cpu() - want).abs()
    print(float((off / bound).max()), flush=True)
    assert (off <= bound).all()
