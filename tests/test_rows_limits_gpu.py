"""Positions by the ten million: more groups of lanes than one side of a grid has threads for (2^32)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2111_09714_amd as Y  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    Y.lib()
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def slices(n, step=1 << 22):
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


def test_positions_without_tokens():
    # a wave to a position, four to a workgroup of 256: n 64 threads
    n, d = (1 << 26) + 3, 264
    dpos = torch.full((n, d), 7.0, dtype=torch.bfloat16, device="cuda")
    dtable = torch.full((5, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ids, dy = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(1, Y.yoso_embedding_backward_workspace_bytes(0, n, 5, d, Y.BF16)), dtype=torch.uint8, device="cuda")
    Y.yoso_embedding_backward(ids, dy, 1.0, dtable, ws, dpos)
    assert not dtable.any() and not any(dpos[s].any() for s in slices(n))


def test_a_position_to_a_token():
    # a wave to a position again, eight to a workgroup of 512; no token names a row, one sequence: dpos is dy
    n, d = (1 << 26) + 3, 514
    dy = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    for i, s in enumerate(slices(n)):
        dy[s] = torch.randn(len(range(*s.indices(n))), d, dtype=torch.bfloat16, device="cuda",
                            generator=torch.Generator("cuda").manual_seed(i))
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    dtable, dpos = Y.embedding_backward(ids, dy, 300, n_pos=n)
    assert not dtable.any()
    assert all(torch.equal(dpos[s], dy[s]) for s in slices(n))
