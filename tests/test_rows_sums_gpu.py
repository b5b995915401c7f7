"""Sums over many rows in the embedding's gradient and the layer norm's parameter gradients: many chunks, blocks and workgroups,
whole numbers summed exactly (tests/rows_sums.py), and rows of several waves over many rounds."""
import pytest

import rows64
import rows_sums
from rows64 import DT, d64, near
from test_embedding_gpu import make_ids

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402

EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    Y.lib()
    yield
    torch.cuda.empty_cache()


def check(tokens, vocab, d, dtype, kind, n_pos=0, scale=0.5, index="i64"):
    ids = make_ids(kind, tokens, vocab, tokens)
    dy = rows_sums.whole(tokens, d, tokens + d)
    want = rows_sums.embedding_sums(ids, dy, vocab, scale, n_pos, dtype)
    got = Y.embedding_backward(ids.to(torch.int32 if index == "i32" else torch.int64).cuda(), dy.cuda().to(DT[dtype]), vocab, scale, n_pos)
    for name, a, b in zip(("dtable", "dpos"), got, want):
        if b is not None:
            wrong = (a.cpu() != b)
            assert not wrong.any(), (name, int(wrong.sum()), [tuple(i.tolist()) for i in wrong.nonzero()[:4]])


# Rows of at least 512 bytes of fp32 sums go in chunks of 512 entries from 2^18 tokens on, of 1024 from 2^19 on: neighbouring
# buckets packed into one (30000 ids), buckets of several chunks (all kinds but even ids), buckets of one id (500 ids).
@pytest.mark.parametrize("tokens,vocab,d,dtype,kind", [
    (262144, 30000, 128, "f32", "uniform"), (300000, 30000, 128, "f32", "power"), (300000, 5000, 256, "bf16", "uniform"),
    (300000, 5000, 256, "bf16", "two"), (300001, 500, 128, "f32", "uniform"), (300000, 500, 131, "f32", "one"),
    (524288, 30000, 256, "bf16", "uniform"), (600000, 30000, 256, "bf16", "power"), (600000, 5000, 128, "f32", "two"),
    (600000, 5000, 128, "f32", "one"), (600011, 500, 128, "f32", "uniform"), (600000, 500, 256, "bf16", "two"),
    (600000, 300000, 128, "f32", "uniform"), (600000, 300000, 128, "f32", "power"), (600000, 700000, 128, "f32", "once")])
def test_long_chunks(tokens, vocab, d, dtype, kind):
    check(tokens, vocab, d, dtype, kind)


@pytest.mark.parametrize("kind", ["uniform", "power", "one", "two"])
@pytest.mark.parametrize("tokens,vocab,d,dtype", [(70000, 2, 130, "f32"), (200001, 3000, 8, "f32"), (600000, 5000, 8, "f32"),
                                                  (300000, 1 << 18, 8, "bf16"), (2_100_003, 1000, 16, "f32")])
def test_many_tokens(tokens, vocab, d, dtype, kind):
    check(tokens, vocab, d, dtype, kind, scale=-2.0)


def test_more_tokens_than_blocks_of_counts():
    # past 128 blocks of 65535 tokens there are more blocks
    check(8_500_000, 90, 2, "f32", "two", n_pos=100, index="i32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,n", [(300000, 1), (200000, 3), (20000, 17), (8, 40000), (7, 40001), (2, 131072), (1, 300000)])
def test_positions(batch, n, dtype):
    check(batch * n, 50, 24, dtype, "two", n_pos=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(70001, 40), (200003, 16), (20001, 128), (9000, 1001), (5000, 2047), (3001, 4096),
                                    (600, 5003), (2600, 8191), (2600, 8192)])
def test_parameter_gradients_of_many_rows(rows, d, dtype):
    """More rows than the workgroups take in one round, rows of one wave and of up to eight; the forward too."""
    g = torch.Generator().manual_seed(rows)
    n = lambda *s: torch.randn(*s, generator=g)
    x, dy = (0.5 + n(rows, d)).to(DT[dtype]).cuda(), rows_sums.whole(rows, d, d).cuda().to(DT[dtype])
    w, b = (1 + 0.3 * n(d)).cuda(), (0.2 * n(d)).cuda()
    x64, dy64 = x.double(), dy.double()
    y = Y.layer_norm(x, w, b, EPS)
    want, _, err = rows64.layer_norm(x64, None, w.double(), b.double(), EPS)
    near("y", y, want.cpu(), err.cpu(), dtype)
    dx, dw, db = Y.layer_norm_backward(x, w, dy, EPS)
    (want, _, _), (err, _, _) = rows64.layer_norm_backward(x64, w.double(), dy64, None, EPS)
    near("dx", dx, want.cpu(), err.cpu(), dtype)
    want, err = rows_sums.dweight(x64, dy64, EPS)
    near("dweight", dw, want.cpu(), err.cpu(), "f32")
    assert torch.equal(db.double(), dy64.sum(0))
