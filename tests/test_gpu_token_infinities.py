"""The vocabulary's loss where logits are infinite: a block of the vocabulary that no row can choose.  Formulas and tolerances are those of test_gpu_token_loss.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import BF16, F32, check, make, reference

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
