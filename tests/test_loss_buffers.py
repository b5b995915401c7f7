"""Buffers of the losses' backward, refused before any HIP call (fake pointers, never dereferenced): one for dbias and another output,
a workspace that is too small."""
import ctypes

import pytest

import paper_2111_09714_amd as Y
from test_loss_abi import FAKE, L, _ceb, _kdb  # noqa: F401  (L is the library's fixture)


@pytest.mark.parametrize("call", [_ceb, _kdb])
@pytest.mark.parametrize("tokens", [1, 10, 100])
def test_dbias_is_a_buffer_of_its_own(L, call, tokens):  # noqa: F811
    for dbias, other in ((FAKE, "dx"), (2 * FAKE, "dtable")):
        assert call(L, tokens=tokens, dx=FAKE, dtable=2 * FAKE, dbias=dbias) == 9
        assert other in L.yoso_last_error().decode() and "dbias" in L.yoso_last_error().decode()


def test_workspace_of_the_backward(L):  # noqa: F811
    """Few tokens take fp32 parts of dx alone (one per 16 entries, at most 512), no copy of the table; what one size function gives for
    any top is enough for every top."""
    size, most = Y.yoso_distillation_backward_workspace_bytes, Y.yoso_cross_entropy_backward_workspace_bytes
    for n, top, vocab, d, dt in ((1, 1, 3000, 96, 0), (2, 1, 3000, 96, 1), (16, 1, 30000, 768, 0), (16, 64, 3000, 96, 0), (16, 65, 3000, 96, 0), (1, 1024, 50, 64, 1),
                                 (17, 1, 300, 96, 0), (32, 32, 300, 96, 0), (32, 33, 300, 96, 0), (500, 7, 3000, 96, 1), (16, 1, 40, 2048, 0), (1, 1, 1, 1, 0)):
        need = size(n, top, vocab, d, dt)
        assert 0 < need <= most(n, vocab, d, dt)
        assert _kdb(L, tokens=n, top=top, vocab=vocab, d=d, dtype=dt, wsb=need - 1, dbias=3 * FAKE) == 6
        if top == 1:
            assert _ceb(L, tokens=n, vocab=vocab, d=d, dtype=dt, wsb=need - 1, dbias=3 * FAKE) == 6
        if n <= 16 and n * top <= 1024 and d <= 2048:
            assert need == min(512, -(-vocab // 16)) * 16 * d * 4
    bad = ctypes.c_size_t(-1).value
    for args in ((10, 0, 10, 64, 0), (10, 1025, 10, 64, 0), (-1, 1, 10, 64, 0), (10, 1, 10, 64, 5), (10, 1, 0, 64, 0), (10, 1, 10, 8193, 0)):
        assert L.yoso_distillation_backward_workspace_bytes(*args) == bad
        with pytest.raises(Y.YosoError):
            Y.yoso_distillation_backward_workspace_bytes(*args)
