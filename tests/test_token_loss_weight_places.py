"""Where the vocabulary's loss takes its weight from: at any place where it need not be aligned, without a copy."""
import ctypes as C

import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import ALL, BF16, F32, check, make, reference
from test_sequence_ops_host import on_device, recorder  # noqa: F401
from test_token_ops_host import D, N, V, allocations, ids  # noqa: F401


def test_a_float_weight_is_not_copied(recorder, allocations):
    """Float weights are read by loads of any alignment: one that starts off a 16-byte boundary is handed on as it is."""
    base = on_device(torch.randn(V * D + 8))
    w = torch.as_strided(base, (V, D), (D, 1), (-base.data_ptr() // 4) % 4 + 1)
    assert w.data_ptr() % 16 == 4
    for call in (mwb.token_loss, mwb.token_loss_gradient):
        call(on_device(torch.randn(N, D)), w, ids(N))
        assert recorder.calls[-1][1][2] == w.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 20, 128, 129])
def test_the_c_abi_takes_a_weight_off_its_boundary_for_gradients(rows):
    """bf16 rows over a large weight, which an aligned one is read in place for: no other number of rows, columns or tokens
    decides whether a call is valid."""
    vocab, dim, L = 12353, 1088, mwb.lib()
    h, W, t = make(rows, vocab, dim, BF16, seed=rows)
    wide = torch.zeros(vocab, dim + 8, device="cuda", dtype=BF16)
    off = wide[:, 1:dim + 1]
    off.copy_(W)
    assert off.data_ptr() % 16 == 2
    d = mwb.TokenLossDesc(rows, vocab, dim, 2, 0, 8, 0, 0, dim + 8, 0, 0, 1.0)
    need = C.c_size_t()
    assert L.mw_token_loss_workspace_bytes(d, 1, need) == 0
    room = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    loss, total = torch.empty(rows, device="cuda"), torch.empty((), device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(W)
    assert L.mw_token_loss_gradient(d, h.data_ptr(), off.data_ptr(), t.data_ptr(), None, loss.data_ptr(), total.data_ptr(), dh.data_ptr(), dw.data_ptr(),
                                    room.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
    assert L.mw_token_loss_status(room.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    check(mwb.TokenLoss(loss, total, dh, dw), reference(h, W, t), ALL)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 9, 150])
def test_float_weights_off_their_boundary(rows):
    h, W, t = make(rows, 700, 128, F32, seed=rows)
    base = torch.zeros(700 * 128 + 1, device="cuda")
    off = base[1:].view(700, 128)
    off.copy_(W)
    want = reference(h, W, t)
    check(mwb.token_loss(h, off, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, off, t), want, ALL)
