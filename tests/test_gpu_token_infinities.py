"""The vocabulary's loss where logits are infinite or very large: a block of the vocabulary that no row can choose, a target
whose own logit is infinite, powers of two that 32 bits round.  Formulas and tolerances are those of test_gpu_token_loss.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import ALL, BF16, F32, check, make, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,dtype", [(1, F32), (4, F32), (8, F32), (1, BF16), (20, BF16), (200, BF16), (300, BF16)])
@pytest.mark.parametrize("beyond", [1, 65, 128, 300])
@pytest.mark.parametrize("size", [20.0, 150.0, 3000.0])
def test_blocks_that_no_row_can_choose(size, beyond, N, dtype):
    """The vocabulary's last rows are -inf, whole blocks of them or a short last one; the logits of the others lie around
    -size, so far below one that their exponentials cannot be held relative to one."""
    V, D = 256, 64
    g = torch.Generator(device="cuda").manual_seed(N)
    W = -(size / D) * (1 + 0.02 * torch.rand(V + beyond, D, generator=g, device="cuda"))
    W[V:] = float("-inf")
    W, h = W.to(dtype), torch.ones(N, D, device="cuda", dtype=dtype)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    want = reference(h, W[:V].contiguous(), t)
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t), want, ("loss", "total"))


def test_blocks_that_no_row_can_choose_of_a_large_weight():
    """The same where the gradient of few rows reads the weight in place."""
    N, V, D = 20, 12288, 1024
    W = torch.full((V + 100, D), -150.0 / D, device="cuda") * (1 + 0.02 * torch.rand(V + 100, 1, device="cuda"))
    W[V:] = float("-inf")
    W, h, t = W.to(BF16), torch.ones(N, D, device="cuda", dtype=BF16), torch.arange(N, device="cuda") * 600
    check(mwb.token_loss_gradient(h, W, t), reference(h, W[:V].contiguous(), t), ("loss", "total"))


@pytest.mark.parametrize("N,dtype", [(1, F32), (4, F32), (8, F32), (1, BF16), (20, BF16), (200, BF16), (300, BF16)])
def test_an_infinite_logit_of_the_target(N, dtype):
    """inf - inf is no loss of zero: a row of the weight that holds infinities is not a sure prediction of its own token."""
    h, W, t = make(N, 300, 64, dtype, lean=0.0)
    h, t = h.abs() + 0.5, torch.full((N,), 170, device="cuda")
    W[170] = float("inf")
    for r in (mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)):
        assert bool(r.loss.isnan().all()) and bool(r.total.isnan())
    assert not bool(torch.isfinite(r.dh).any())


@pytest.mark.parametrize("N,dtype", [(3, F32), (8, F32), (9, F32), (200, F32), (3, BF16), (300, BF16)])
def test_a_target_whose_logit_overflows(N, dtype):
    """Finite operands whose product is beyond 32 bits: loss and dh of that row alone are not finite."""
    h, W, t = make(N, 300, 64, dtype, lean=0.0)
    h[:, 0], W[:, 0], t[0] = 0.0, 0.0, 170
    t[1:][t[1:] == 170] = 171
    h[0, 0] = 2.0 ** 70
    W[170, 0] = 2.0 ** 70
    for r in (mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)):
        assert bool(r.loss[0].isnan()) and bool(torch.isfinite(r.loss[1:]).all())
    assert not bool(torch.isfinite(r.dh[0]).any()) and bool(torch.isfinite(r.dh[1:]).all())


@pytest.mark.parametrize("N,dtype", [(8, F32), (9, F32), (300, F32), (20, BF16), (300, BF16)])
@pytest.mark.parametrize("size", [10, 18, 20, 22, 24, 30, 44, 100])
def test_logits_far_from_one(size, N, dtype):
    """Logits of 2^size: everything is finite, and rows that are sure of their target have a loss of zero."""
    h, W, t = make(N, 700, 128, dtype, seed=N, lean=8.0)
    h, W = h * 2.0 ** (size // 2), W * 2.0 ** (size - size // 2)
    want = reference(h, W, t)
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t), want, ALL)
