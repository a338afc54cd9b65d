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
