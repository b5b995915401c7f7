"""Launches of 2^32 threads and more, which would run a part of themselves without an error, are refused on the host; the
largest that fit are right to the last head."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402

BF16, I16 = torch.bfloat16, torch.int16


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    Y.lib()
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def empty(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def signs(*shape):
    x = torch.empty(*shape, dtype=BF16, device="cuda")
    return x.bernoulli_(0.5, generator=torch.Generator("cuda").manual_seed(1)).mul_(2).sub_(1)


def refused(call):
    with pytest.raises(Y.YosoError) as e:
        call()
    assert e.value.status == 7 and "hipErrorInvalidConfiguration" in str(e.value)


# a workgroup of 256 threads to a head of one row: 2^24 heads are one too many
@pytest.mark.parametrize("bh", [(1 << 24) - 1, 1 << 24])
def test_forward_of_single_rows(bh):
    v, y = signs(bh, 1, 64), torch.zeros(bh, 1, 64, dtype=BF16, device="cuda")
    codes = torch.zeros(bh, 1, 8, dtype=I16, device="cuda")
    if bh == 1 << 24:
        return refused(lambda: Y.yoso_forward(codes, codes, v, 8, 4, y))
    Y.yoso_forward(codes, codes, v, 8, 4, y)  # every code collides: y is v
    assert torch.equal(y, v)


@pytest.mark.parametrize("bh", [(1 << 24) - 1, 1 << 24])
def test_expectation_of_single_rows(bh):
    q, v = signs(bh, 1, 64).mul_(0.125), signs(bh, 1, 64)
    y = torch.zeros_like(v)
    if bh == 1 << 24:
        return refused(lambda: Y.yoso_expectation_forward(q, q, v, 4, y))
    Y.yoso_expectation_forward(q, q, v, 4, y)  # cosine 1: y is v
    assert torch.equal(y, v)


def test_tables_of_many_heads():
    # 32 feature slices of 512 threads a head
    bh = 1 << 18
    q, k = empty(bh, 1025, 4, dtype=I16), empty(bh, 1, 4, dtype=I16)
    refused(lambda: Y.yoso_forward(q, k, empty(bh, 1, 64), 4, 12, empty(bh, 1025, 64)))


def test_star_pairs_of_many_heads():
    # two sides of 504 derived hashes of 256 threads a head
    bh, m, tau = 16700, 56, 9
    t = [torch.ones(bh, 1, 64, dtype=BF16, device="cuda") for _ in range(4)]
    c = torch.zeros(bh, 1, m, dtype=I16, device="cuda")
    ws = empty(Y.yoso_workspace_bytes(Y.OP_BACKWARD_STAR, bh, 1, 1, 64, m, tau, Y.BF16), dtype=torch.uint8)
    refused(lambda: Y.yoso_backward_star(c, c, *t, m, tau, *[torch.empty_like(t[0]) for _ in range(3)], ws))
