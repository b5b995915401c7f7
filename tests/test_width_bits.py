"""Rows wider than the C ABI's 32-bit d are refused by the binding: ctypes would keep the lower bits, and a row of 2^32 + 64 values
pass for one of 64.  Tensors without memory (meta), no GPU."""
import os

import pytest

import paper_2111_09714_amd as Y
from paper_2111_09714_amd import build as ybuild

torch = pytest.importorskip("torch")

WIDE = (1 << 32) + 64


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(Y.lib_path()):
        ybuild.build()


def t(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="meta")


CALLS = {
    "layer_norm": lambda: Y.yoso_layer_norm(t(2, WIDE), None, None, 1e-5, t(2, WIDE)),
    "layer_norm of one row": lambda: Y.layer_norm(t(WIDE), None, None),
    "layer_norm_backward": lambda: Y.yoso_layer_norm_backward(t(2, WIDE), None, t(2, WIDE), 1e-5, t(2, WIDE)),
    "embedding": lambda: Y.yoso_embedding(t(3, dtype=torch.int64), t(9, WIDE), 1.0, t(3, WIDE)),
    "embedding_backward": lambda: Y.yoso_embedding_backward(t(3, dtype=torch.int64), t(3, WIDE), 1.0, t(9, WIDE), None),
    "layer norm's workspace": lambda: Y.yoso_layer_norm_backward_workspace_bytes(10, WIDE, Y.F32),
    "embedding's workspace": lambda: Y.yoso_embedding_backward_workspace_bytes(1000, 0, 10, WIDE, Y.F32),
    "workspace": lambda: Y.yoso_workspace_bytes(Y.OP_BACKWARD, 1, 8, 8, WIDE, 4, 4, Y.F32),
    "l2_normalize": lambda: Y.yoso_l2_normalize(t(2, WIDE), t(2, WIDE)),
    "l2_normalize_backward": lambda: Y.yoso_l2_normalize_backward(t(2, WIDE), t(2, WIDE), t(2, WIDE)),
    "hash": lambda: Y.yoso_hash(t(1, 2, WIDE), t(WIDE, 16), 4, 4, t(1, 2, 4, dtype=torch.int16)),
    "fast_hash": lambda: Y.yoso_fast_hash(t(1, 2, WIDE), t(1, 3, dtype=torch.int64), 4, 4, t(1, 2, 4, dtype=torch.int16)),
    "forward": lambda: Y.yoso_forward(*[t(1, 2, 4, dtype=torch.int16)] * 2, t(1, 2, WIDE), 4, 4, t(1, 2, WIDE)),
    "backward": lambda: Y.yoso_backward(*[t(1, 2, 4, dtype=torch.int16)] * 2, *[t(1, 2, WIDE)] * 4, 4, 4, *[t(1, 2, WIDE)] * 3, None),
    "backward_star": lambda: Y.yoso_backward_star(*[t(1, 2, 4, dtype=torch.int16)] * 2, *[t(1, 2, WIDE)] * 4, 4, 4, *[t(1, 2, WIDE)] * 3, None),
    "backward_noalloc": lambda: Y.yoso_backward_noalloc(*[t(1, 2, 4, dtype=torch.int16)] * 2, *[t(1, 2, WIDE)] * 4, 4, 4, *[t(1, 2, WIDE)] * 3),
    "expectation_forward": lambda: Y.yoso_expectation_forward(*[t(1, 2, WIDE)] * 3, 4, t(1, 2, WIDE)),
    "expectation_backward": lambda: Y.yoso_expectation_backward(*[t(1, 2, WIDE)] * 4, 4, *[t(1, 2, WIDE)] * 3),
}


@pytest.mark.parametrize("call", CALLS)
def test_a_width_past_32_bits_is_refused(call):
    with pytest.raises(Y.YosoError) as e:
        CALLS[call]()
    assert e.value.status == 2 and str(WIDE) in str(e.value)


@pytest.mark.parametrize("d", [-WIDE, -(1 << 31) - 1, 1 << 31])
def test_widths_beside_the_limits(d):
    with pytest.raises(Y.YosoError) as e:
        Y.yoso_layer_norm_backward_workspace_bytes(10, d, Y.F32)
    assert e.value.status == 2 and str(d) in str(e.value)
    for d in (-(1 << 31), (1 << 31) - 1):  # (the library's own refusal)
        with pytest.raises(Y.YosoError):
            Y.yoso_layer_norm_backward_workspace_bytes(10, d, Y.F32)
