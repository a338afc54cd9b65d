"""A bounded wait of the vocabulary's loss that runs out: the call ends, its status says so, its total is NaN, and of its other
results each number is NaN or what it would have been; the next call in the same memory is right."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import BF16, F32, make

pytestmark = pytest.mark.gpu
TIMEOUT = mwb.STATUS_NAMES.index("MW_ERR_TIMEOUT")
LOGITS, DH, DW = range(3)


@pytest.fixture
def unmet():
    yield lambda product: mwb.token_loss_selftest_unmet_wait(5, product)
    mwb.token_loss_selftest_unmet_wait(0)


def right_or_nan(got, want):
    return bool((got.isnan() | (got == want)).all())


@pytest.mark.parametrize("N,dtype", [(20, BF16), (200, BF16), (300, BF16), (9, F32), (300, F32)])
def test_loss_alone(N, dtype, unmet):
    h, W, t = make(N, 1000, 128, dtype, left_out=0.2)
    room = mwb.token_loss_workspace(h, W)
    want = mwb.token_loss(h, W, t)
    unmet(LOGITS)
    r = mwb.token_loss(h, W, t, workspace=room)
    assert mwb.token_loss_status(room) == TIMEOUT and bool(r.total.isnan()) and right_or_nan(r.loss, want.loss)
    unmet(DH)                                       # (a product that this call does not have)
    r = mwb.token_loss(h, W, t, workspace=room)
    assert mwb.token_loss_status(room) == 0 and torch.equal(r.loss, want.loss) and torch.equal(r.total, want.total)


@pytest.mark.parametrize("N,V,D,dtype,piece", [(9, 1000, 128, F32, 0), (300, 1000, 128, BF16, 0), (20, 12353, 1088, BF16, 0), (700, 600, 65, F32, 256),
                                               (700, 600, 128, BF16, 256), (2100, 200, 100, BF16, 0)])
@pytest.mark.parametrize("product", [LOGITS, DH, DW])
@pytest.mark.parametrize("live", ["all", "in the first piece"])
def test_gradients(live, product, N, V, D, dtype, piece, unmet):
    h, W, t = make(N, V, D, dtype)
    if live != "all":
        t[200:] = -1
    room = mwb.token_loss_workspace(h, W, True, piece)
    want = mwb.token_loss_gradient(h, W, t, piece_rows=piece)
    for _ in range(2):
        unmet(product)
        r = mwb.token_loss_gradient(h, W, t, piece_rows=piece, workspace=room,
                                    dh=torch.full_like(h, 7.0), dweight=torch.full_like(W, 7.0))
        assert mwb.token_loss_status(room) == TIMEOUT and bool(r.total.isnan())
        assert all(right_or_nan(a, b) for a, b in zip((r.loss, r.dh, r.dweight), (want.loss, want.dh, want.dweight)))
        assert bool(r.dweight.isnan().any())
        if product != DW:
            assert bool(r.dh[:1].isnan().all())
        mwb.token_loss_selftest_unmet_wait(0)
        r = mwb.token_loss_gradient(h, W, t, piece_rows=piece, workspace=room)
        assert mwb.token_loss_status(room) == 0 and all(torch.equal(a, b) for a, b in zip(r, want))


def test_limits_out_of_range():
    for limit, product in ((1001, 0), (5, 3), (5, -1)):
        with pytest.raises(mwb.MwError):
            mwb.token_loss_selftest_unmet_wait(limit, product)
