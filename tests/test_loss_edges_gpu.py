"""The losses over a vocabulary where single rows are out of the ordinary: rows of x that are no numbers, tokens that are sure of what they
are taught, entries taken out under a negative scale.  Against sums in 64 bits (tests/loss64.py) or against the same call without the row."""
import math

import pytest

import loss64
from rows64 import DT, near
from test_loss_gpu import as64, backward, cuda, forward, make, planes

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,top", [(20, 64, 0), (20, 1100, 0), (20, 1100, 6), (40, 64, 0), (40, 64, 70), (300, 96, 0), (300, 96, 6)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_row_of_x_that_is_no_number(n, d, top, dtype, bad):
    """Token 9 takes part: its loss and dx are NaN and so are dtable and dbias, which sum over it; every other token's loss and dx have
    the bits that they have without it."""
    s = make(n, 400, d, dtype, top=top, share=0.6, seed=6)
    s["ids"][9] = torch.arange(max(1, top)) * 3
    s["dloss"][9] = 0.5
    a = forward(cuda(s), 0.5)
    ga = backward(cuda(s), 0.5, a[2], a[1])
    dirty = dict(s, x=s["x"].clone())
    dirty["x"][9, d // 2] = bad
    b = forward(cuda(dirty), 0.5)
    gb = backward(cuda(dirty), 0.5, b[2], b[1])
    other = torch.arange(n) != 9
    assert torch.isnan(b[0][9]) and torch.equal(a[0].cpu()[other], b[0].cpu()[other]) and torch.equal(a[1].cpu()[other], b[1].cpu()[other])
    assert torch.isnan(gb[0][9]).all() and torch.equal(ga[0].cpu()[other], gb[0].cpu()[other])
    assert torch.isnan(gb[1]).all() and torch.isnan(gb[2]).all()


def sure(n, vocab, d, dtype, top, logits=None, less=None, seed=4):
    """Tokens whose first id y has nearly all probability, the teacher's too: its logit from the first to the last of `logits`, or such that
    1 - q goes (evenly in its logarithm) from the first to the last of `less`."""
    s = make(n, vocab, d, dtype, top=top, bias=False, share=1.0, seed=seed)
    # (for `less` rows of one length: of a short one none can be sure)
    s["table"] = (s["table"].float() * 3 if less is None else 3 * torch.nn.functional.normalize(s["table"].float(), dim=1)).to(DT[dtype])
    y = s["ids"][:, 0].long()
    w = s["table"].float()
    point = w[y] / w[y].square().sum(1, keepdim=True)
    noise = s["x"].float() * 0.1
    if less is None:
        at = torch.linspace(*logits, n)
    else:
        want = torch.logspace(*(math.log10(v) for v in less), n, dtype=torch.float64)
        a, b = noise.double() @ w.double().t(), point.double() @ w.double().t()
        lo, hi = torch.zeros(n, dtype=torch.float64), torch.full((n,), 100.0, dtype=torch.float64)
        for _ in range(40):
            mid = (lo + hi) / 2
            c = -torch.expm1(torch.log_softmax(a + mid[:, None] * b, 1).gather(1, y[:, None])[:, 0])
            lo, hi = torch.where(c > want, mid, lo), torch.where(c > want, hi, mid)
        at = hi.float()
    s["x"] = (noise + at[:, None] * point).to(DT[dtype])
    if top:
        s["teacher"] = torch.where(torch.arange(top) == 0, 3.0, -60 - torch.rand(n, top, generator=torch.Generator().manual_seed(seed)))
        # (an id twice would share its probability)
        s["ids"][:, 1:] = (s["ids"][:, :1] + 1 + torch.arange(top - 1) * max(1, (vocab - 1) // top)) % vocab
    return s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,top", [(5, 900, 128, 1), (20, 900, 128, 70), (64, 3000, 96, 5), (300, 2000, 96, 1), (300, 2000, 96, 5), (300, 2000, 96, 70),
                                           (700, 2000, 500, 64), (4100, 300, 64, 1)])
def test_log_q_near_zero(n, vocab, d, top, dtype):
    """As cross entropy's losses near zero: log q = -log(1 + rest), rest = sum exp(l - l_y) of the other entries, off by rest (2 le + 4 u) for
    the logits' errors and the exponentials and by u (44 + vocab / 128) (1 + rest) for the sums of 1 + rest and the logarithm, never above 0.
    The teacher's probability of y is 1 in fp32 (the others' e^-60).  So the loss is -log q, and G at y, expm1(log q), as far off as log q."""
    s = sure(n, vocab, d, dtype, top, logits=(8, 24))
    e = as64(s)
    y = s["ids"][:, 0]
    l, le = loss64.logits(e["x"], e["table"], None, 1.0, planes(dtype))
    at = l.gather(1, y[:, None])[:, 0]
    rest = torch.exp(l - at[:, None]).scatter_(1, y[:, None], 0.0).sum(1)
    assert float(rest.min()) < 1e-4
    loss, lse, logq = forward(cuda(s), 1.0)
    bound = rest * (2 * le.amax(1) + 4 * loss64.U) + (44 + vocab / 128) * loss64.U * (1 + rest)
    mine = logq[:, 0].double().cpu()
    off = (mine + torch.log1p(rest)).abs()
    print(float((off / bound).max()), int((mine > 0).sum()), flush=True)
    assert (mine <= 0).all() and (off <= bound).all()
    assert ((loss.double().cpu() + mine).abs() <= 1e-6 * (1 + mine.abs()) * mine.abs() + 1e-20).all()
    grads = backward(cuda(s), 1.0, logq, lse)
    exact = l.gather(1, s["ids"].long()) - torch.logsumexp(l, 1, keepdim=True)
    want, err = loss64.gradients(e["x"], e["table"], None, 1.0, s["ids"].long(), e["teacher"], exact, lse.double().cpu(), e["dloss"], planes(dtype))
    more = e["dloss"] * bound
    w = e["table"].abs()
    near("dx", grads[0], want[0], err[0] + more[:, None] * w[y], dtype)
    near("dtable", grads[1], want[1], err[1] + torch.zeros_like(w).index_add_(0, y, more[:, None] * e["x"].abs()), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,top,less", [(300, 4000, 96, 0, (1e-6, 1e-3)), (300, 4000, 96, 1, (1e-6, 1e-3)), (512, 8000, 64, 0, (1e-6, 1e-3)),
                                                (90, 5000, 200, 4, (1e-6, 1e-3)), (300, 20000, 40, 0, (2e-7, 2e-6)), (300, 20000, 40, 3, (2e-7, 2e-6))])
def test_gradients_of_tokens_that_are_sure(n, vocab, d, top, less, dtype):
    """1 - q of the taught id small for all tokens: dx and dtable keep their digits, although every G is small.

    G's planes: the largest |G sx sw| of all tokens and entries, c' dloss sx sw, is at most 2^14 of a plane, c' = c + 2^-12 with c the largest of
    the tokens' 1 - q (to 1%).  One plane's smallest step is 2^-24, half of it 2^-25: 2^-39 c' of what the bound of loss64 takes for the largest
    (there with c = 1).  Of a pair the lower plane carries 2^12 times what the upper one leaves: 2^-51 c'."""
    s = sure(n, vocab, d, dtype, top, less=less)
    e = as64(s)
    ids = s["ids"].long()
    (loss, lse, logq), _ = loss64.loss(e["x"], e["table"], None, 1.0, ids, e["teacher"], planes(dtype))
    c = -torch.expm1(logq[:, 0])
    print("1 - q from", float(c.min()), "to", float(c.max()), flush=True)
    assert 0.5 < float(c.min()) / less[0] < 2 and 0.5 < float(c.max()) / less[1] < 2
    logq, lse = (logq if top else -loss[:, None]).float(), lse.float()
    grads = backward(cuda(s), 1.0, logq.cuda(), lse.cuda())
    want, err = loss64.gradients(e["x"], e["table"], None, 1.0, ids, e["teacher"], logq.double(), lse.double(), e["dloss"], planes(dtype))
    # loss64's floor of G and what it makes of the errors, in the present one's place
    ax, aw = e["x"].abs(), e["table"].abs()
    mx, mw = ax.amax(1, keepdim=True), aw.amax(1)
    room = 2.0 ** -36 * (e["dloss"][:, None] * mx).amax() * mw.max() / (mx * mw[None])
    less = 1 - (1.01 * float(c.max()) + 2.0 ** -12) * (2.0 ** -12 if dtype == "f32" else 1.0)
    err = (err[0] - less * (room @ aw), err[1] - less * (room.t() @ ax))
    for name, got, b, t in zip(("dx", "dtable"), grads, want, err):
        off = (got.double().cpu() - b).norm(dim=1) / b.norm(dim=1)
        print(f"  {name}: rows off by {float(off.median()):.2g} (median), {float(off.max()):.2g}; bound {float((t.norm(dim=1) / b.norm(dim=1)).max()):.2g}",
              flush=True)
        near(name, got, b, t, dtype)


def test_gradients_of_sure_tokens_beside_others():
    """fp32, every other token far from sure: the sure ones' dx and the rows of dtable that are improbable for all keep their digits."""
    n, vocab, d = 300, 4000, 96
    s = sure(n, vocab, d, "f32", 0, less=(1e-6, 1e-3))
    s["x"][::2] = torch.randn(150, d, generator=torch.Generator().manual_seed(3))
    s["bias"] = torch.where(torch.arange(vocab) % 3 == 1, -16.0, 0.0)
    s["bias"][s["ids"][:, 0]] = 0
    e = as64(s)
    ids = s["ids"].long()
    (loss, lse, _), _ = loss64.loss(e["x"], e["table"], e["bias"], 1.0, ids, None, 2)
    logq, lse = -loss[:, None].float(), lse.float()
    grads = backward(cuda(s), 1.0, logq.cuda(), lse.cuda())
    want, err = loss64.gradients(e["x"], e["table"], e["bias"], 1.0, ids, None, logq.double(), lse.double(), e["dloss"], 2)
    ax, aw = e["x"].abs(), e["table"].abs()
    mx, mw = ax.amax(1, keepdim=True), aw.amax(1)
    room = 2.0 ** -36 * (e["dloss"][:, None] * mx).amax() * mw.max() / (mx * mw[None])
    less = 1 - 2.0 ** -12
    near("dx", grads[0], want[0], err[0] - less * (room @ aw), "f32")
    near("dtable", grads[1], want[1], err[1] - less * (room.t() @ ax), "f32")
    near("dbias", grads[2], want[2], err[2], "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 20, 50, 300])
def test_entries_taken_out_under_a_negative_scale(n, dtype):
    """A bias of -inf takes its row of the table out whatever the sign of the scale (so does +inf under a negative one, by the formula)."""
    s = make(n, 180, 64, dtype, share=1.0, seed=8)
    out = torch.zeros(180, dtype=torch.bool)
    out[torch.tensor([3, 7, 100, 179])] = True
    s["ids"] = torch.where(out[s["ids"]], 5, s["ids"])
    e = as64(s)
    s["bias"][out] = -math.inf
    e["bias"][out] = math.inf
    ids = s["ids"].long()
    got = forward(cuda(s), -0.5)
    want, err = loss64.loss(e["x"], e["table"], e["bias"], -0.5, ids, None, planes(dtype))
    near("loss", got[0], want[0], err[0], "f32")
    near("lse", got[1], want[1], err[1], "f32")
    logq, lse = -want[0][:, None].float(), want[1].float()
    grads = backward(cuda(s), -0.5, logq.cuda(), lse.cuda())
    e["bias"][out] = 0.0  # (and the entries away: their G is 0)
    keep = torch.where(out, -1, torch.cumsum(~out, 0) - 1)
    wantg, errg = loss64.gradients(e["x"], e["table"][~out], e["bias"][~out], -0.5, keep[ids], None, logq.double(), lse.double(), e["dloss"], planes(dtype))
    near("dx", grads[0], wantg[0], errg[0], dtype)
    near("dtable", grads[1][~out.cuda()], wantg[1], errg[1], dtype)
    near("dbias", grads[2][~out.cuda()], wantg[2], errg[2], "f32")
    assert not grads[1].cpu()[out].any() and not grads[2].cpu()[out].any()


@pytest.mark.parametrize("n,vocab,d,top", [(1, 700, 64, 0), (16, 2000, 96, 0), (16, 2000, 96, 64), (16, 2000, 96, 65), (9, 30, 2048, 3), (32, 300, 200, 4), (300, 500, 72, 5)])
def test_the_backwards_own_workspace(n, vocab, d, top):
    """With as many bytes as the call says it takes: the same gradients, and nothing behind them is written."""
    s = cuda(make(n, vocab, d, "f32", top=top, share=0.9))
    _, lse, logq = forward(s, 0.5)
    want = backward(s, 0.5, logq, lse)
    need = Y.yoso_distillation_backward_workspace_bytes(n, max(1, top), vocab, d, Y.F32)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    got = [torch.full_like(t, math.nan) for t in want]
    if top:
        Y.yoso_distillation_backward(s["x"], s["table"], s["ids"], s["teacher"], logq, lse, s["dloss"], 2.0, got[0], got[1], ws[:need], got[2], s["bias"])
    else:
        Y.yoso_cross_entropy_backward(s["x"], s["table"], s["ids"][:, 0].contiguous(), -logq[:, 0], lse, s["dloss"], 0.5, got[0], got[1], ws[:need], got[2],
                                      s["bias"])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (ws[need:] == 0x5A).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [4, 66])
@pytest.mark.parametrize("teacher", ["twice", "half", "other"])
def test_sure_tokens_with_ids_listed_twice(teacher, top, dtype):
    """Students that are sure of y, which is listed twice (with another id twice): a teacher whose two entries of y add up to 1, one that gives
    y one half of its probability, and one that is sure of the other id.  G is finite and as exact as any."""
    n, vocab, d = 200, 3000, 80
    s = sure(n, vocab, d, dtype, top, less=(1e-6, 1e-4))
    s["ids"][:, 1] = s["ids"][:, 0]
    s["ids"][:, 3] = s["ids"][:, 2]
    at = {"twice": [0.0, 0.0, -60.0, -60.0], "half": [0.0, -60.0, 0.0, -60.0], "other": [-60.0, -60.0, 0.0, 0.0]}[teacher]
    s["teacher"] = torch.full((n, top), -60.0)
    s["teacher"][:, :4] = torch.tensor(at)
    e = as64(s)
    ids = s["ids"].long()
    (_, lse, logq), _ = loss64.loss(e["x"], e["table"], None, 1.0, ids, e["teacher"], planes(dtype))
    logq, lse = logq.float(), lse.float()
    grads = backward(cuda(s), 1.0, logq.cuda(), lse.cuda())
    want, err = loss64.gradients(e["x"], e["table"], None, 1.0, ids, e["teacher"], logq.double(), lse.double(), e["dloss"], planes(dtype))
    for name, got, b, t in zip(("dx", "dtable"), grads, want, err):
        assert torch.isfinite(got).all()
        off = (got.double().cpu() - b).norm(dim=1) / b.norm(dim=1)
        print(f"  {name}: rows off by {float(off.median()):.2g} (median), {float(off.max()):.2g}", flush=True)
        near(name, got, b, t, dtype)
