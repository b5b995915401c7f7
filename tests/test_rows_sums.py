"""The bounds of tests/rows_sums.py see a part of a sum that is lost: the mistakes are planted in the 64-bit sums, on the CPU."""
import pytest

torch = pytest.importorskip("torch")
import rows_sums  # noqa: E402
from rows64 import DT, U  # noqa: E402

EPS = 1e-5


@pytest.mark.parametrize("rows,d", [(70001, 40), (20000, 128), (2500, 1001)])
def test_a_lost_partial_row_shows(rows, d):
    """One of 256 workgroups, or one round of it, left out of dweight and dbias."""
    g = torch.Generator().manual_seed(rows)
    z, dy = torch.randn(rows, d, generator=g, dtype=torch.float64), rows_sums.whole(rows, d, 1).double()
    want, err = rows_sums.dweight(z, dy, EPS)
    tol = err + U * want.abs()
    step = -(-rows // 256)
    for lost in (slice(0, rows, 256), slice(7 * step, 8 * step), slice(rows - step, rows)):
        off = rows_sums.dweight(z[lost], dy[lost], EPS)[0].abs()
        assert (off > tol).float().mean() > 0.9
        assert (dy[lost].sum(0) != 0).float().mean() > 0.8
    assert (want.abs() > tol).float().mean() > 0.9  # (and no sum at all)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,d,n_pos", [(300000, 300, 16, 4), (100000, 10, 24, 1)])
def test_a_lost_chunk_shows(tokens, vocab, d, n_pos, dtype):
    g = torch.Generator().manual_seed(2)
    ids = torch.randint(-2, vocab + 2, (tokens,), generator=g)
    dy = rows_sums.whole(tokens, d, 3)
    want, pos = rows_sums.embedding_sums(ids, dy, vocab, 0.5, n_pos, dtype)
    assert want.dtype == DT[dtype] and torch.equal(want.double(), want.double().round(decimals=1) if dtype == "f32" else want.double())
    for lost in (slice(0, 512), slice(tokens - tokens // 130, tokens)):
        part = dy.clone()
        part[lost] = 0
        a, b = rows_sums.embedding_sums(ids, part, vocab, 0.5, n_pos, dtype)
        hit = torch.zeros(vocab, dtype=torch.bool)
        named = ids[lost]
        hit[named[(named >= 0) & (named < vocab)]] = True
        assert (a != want)[hit].any(1).float().mean() > 0.5
        assert not torch.equal(b, pos)


def test_whole_numbers_stay_exact():
    for rows in (1, 512, 300000, 600000, 8_500_000):
        v = rows_sums.whole(rows, 2, 4)
        assert int(v.abs().max()) * rows < 2 ** 24 and v.min() < 0 < v.max() or rows == 1
    with pytest.raises(AssertionError):
        rows_sums.whole(1 << 24, 1, 4)


def test_additions():
    # 512 / 16 rows a round at d = 40 (no more than 16 lanes), 256 workgroups: 9 rounds for 70001 rows
    assert rows_sums.additions(70001, 40) == 9 + 1 + 24
    assert rows_sums.additions(3, 8192) == 4 + 24
    assert rows_sums.additions(2560, 8192) == 10 + 1 + 24
