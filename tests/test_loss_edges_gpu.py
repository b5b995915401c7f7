"""The losses over a vocabulary where single rows are out of the ordinary."""
import math

import pytest

from test_loss_gpu import backward, cuda, forward, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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
