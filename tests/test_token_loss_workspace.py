"""The vocabulary's loss in memory that the caller keeps, and its status: what the binding hands over and refuses, without
a GPU (CPU tensors stand in for CUDA ones, a recorder for the library), and the calls on one."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_sequence_ops_host import on_device, recorder  # noqa: F401
from test_token_ops_host import D, N, V, allocations, ids, refuse  # noqa: F401


def test_a_call_uses_the_memory_it_is_given(recorder, allocations):
    h, w, t = on_device(torch.randn(N, D)), on_device(torch.randn(V, D)), ids(N)
    base = torch.zeros(1 << 16, dtype=torch.uint8)
    room = on_device(base[1:])                                  # (from its first multiple of 256 on)
    for call in (lambda: mwb.token_loss(h, w, t, workspace=room), lambda: mwb.token_loss_gradient(h, w, t, workspace=room)):
        recorder.calls.clear()
        call()
        *_, at, size, _ = recorder.calls[-1][1]
        assert at % 256 == 0 and base.data_ptr() < at <= base.data_ptr() + 256 and at + size <= base.data_ptr() + base.numel()


def test_refusals_of_workspaces(recorder, allocations):
    h, w, t = on_device(torch.randn(N, D)), on_device(torch.randn(V, D)), ids(N)
    for call in (mwb.token_loss, mwb.token_loss_gradient):
        call(h, w, t)                                           # (a layout that has passed is looked at all the same)
        refuse(lambda: call(h, w, t, workspace=on_device(torch.zeros(1 << 16))))
        refuse(lambda: call(h, w, t, workspace=on_device(torch.zeros(1 << 17, dtype=torch.uint8))[::2]))
    refuse(lambda: mwb.token_loss_workspace(torch.randn(N, D), w))
    refuse(lambda: mwb.token_loss_workspace(h, on_device(torch.randn(V))))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [0, 1, 9, 200, 700])
def test_calls_in_kept_memory(rows, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    wide = rand(333, 73)
    for w in (rand(333, 64), wide[:, 5:69], wide[:, :64], rand(1, 64).expand(333, 64)):
        h, t = rand(rows, 64), torch.randint(-1, 333, (rows,), generator=g, device="cuda")
        for gradient, call in ((False, mwb.token_loss), (True, lambda *a, **k: mwb.token_loss_gradient(*a, piece_rows=256, **k))):
            room = mwb.token_loss_workspace(h, w, gradient, 256 if gradient else 0)
            want = call(h, w, t)
            for _ in range(2):
                got = call(h, w, t, workspace=room)
                assert mwb.token_loss_status(room) == 0
                assert all(torch.equal(a, b) for a, b in zip(want, got) if a is not None)
            with pytest.raises(ValueError):
                call(h, w, t, workspace=room[:1024])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mwb.token_loss_gradient(h, w, t, piece_rows=256, stream=side, workspace=room)
    assert mwb.token_loss_status(room, stream=side) == 0 and all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_small_gradient_takes_little_memory():
    """Operands, exponentials and sums of 10 rows of 50x16 are a few hundred KB; a large call has room for shares."""
    import ctypes as C

    def need(rows, vocab, dim, dtype=2):
        n = C.c_size_t()
        assert mwb.lib().mw_token_loss_workspace_bytes(mwb.TokenLossDesc(rows, vocab, dim, dtype, 0, 8, 0, 0, 0, 0, 0, 1.0), 1, n) == 0
        return n.value

    assert need(10, 50, 16) < 1 << 20 and need(10, 50, 16, 1) < 1 << 20
    assert need(4, 50, 16, 1) < 1 << 20 and need(300, 1000, 64) < 16 << 20
    assert need(4096, 32768, 2048) > 4096 * 32768 * 2 + (4096 + 32768) * 2048 * 2 + 54 * 3 * 65536 * 4
