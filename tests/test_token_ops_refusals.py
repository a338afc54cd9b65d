"""Calls of the lookup and the vocabulary's loss that could not come out right are refused before any GPU work (runs without
one): scales that a float cannot hold, results in the place of what the call still reads."""
import ctypes as C

import pytest

from paper_2402_14212_b200 import binding as mwb
from test_token_ops_abi import INVALID, embed, loss


@pytest.mark.parametrize("scale", [1e39, -1e39, 1e300])
def test_scales_beyond_a_float(scale):
    L, n = mwb.lib(), C.c_size_t()
    assert L.mw_embedding_scratch_bytes(embed(scale=scale), n) == INVALID
    assert L.mw_embedding_forward(embed(scale=scale), 256, 512, 1024, None) == INVALID
    assert L.mw_token_loss_workspace_bytes(loss(scale=scale), 0, n) == INVALID
    assert L.mw_token_loss_forward(loss(scale=scale), 256, 512, 1024, None, 2048, 4096, 256, 1 << 50, None) == INVALID


def test_results_in_the_place_of_what_is_read():
    L, n = mwb.lib(), C.c_size_t()
    assert L.mw_embedding_forward(embed(), 256, 512, 512, None) == INVALID
    assert L.mw_embedding_scratch_bytes(embed(), n) == 0
    assert L.mw_embedding_backward(embed(), 256, 512, 512, 0, 256, n.value, None) == INVALID
    for dtype in (1, 2):
        for rows in (4, 40):
            d = loss(dtype=dtype, rows=rows)
            assert L.mw_token_loss_workspace_bytes(d, 1, n) == 0
            h, w, t, out, total = 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20
            for dh, dw in ((6 << 20, w), (6 << 20, h), (6 << 20, 6 << 20), (w, 6 << 20), (w, None), (None, w), (h, h)):
                assert L.mw_token_loss_gradient(d, h, w, t, None, out, total, dh, dw, 256, n.value, None) == INVALID
