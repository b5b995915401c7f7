"""The losses' backward refuses one buffer for dbias and another output before any HIP call (fake pointers, never dereferenced)."""
import pytest

from test_loss_abi import FAKE, L, _ceb, _kdb  # noqa: F401  (L is the library's fixture)


@pytest.mark.parametrize("call", [_ceb, _kdb])
@pytest.mark.parametrize("tokens", [1, 10, 100])
def test_dbias_is_a_buffer_of_its_own(L, call, tokens):  # noqa: F811
    for dbias, other in ((FAKE, "dx"), (2 * FAKE, "dtable")):
        assert call(L, tokens=tokens, dx=FAKE, dtable=2 * FAKE, dbias=dbias) == 9
        assert other in L.yoso_last_error().decode() and "dbias" in L.yoso_last_error().decode()
