"""Up to 8 rows of float operands, which have kernels of their own, and the ninth, which has not: captured calls, rows that are
all left out, values that are not finite, repeated calls.  Formulas and tolerances are those of test_gpu_token_loss.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import ALL, F32, check, make, reference

pytestmark = pytest.mark.gpu
ROWS = pytest.mark.parametrize("N", [1, 4, 5, 8, 9])
SIZES = pytest.mark.parametrize("V,D", [(9001, 520), (4097, 1030), (70, 60000)])


@ROWS
@SIZES
@pytest.mark.parametrize("left_out", [0.0, 1.0])
def test_captured_calls(left_out, V, D, N):
    h, W, t = make(N, V, D, F32, left_out=left_out)
    mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
    for seed in (1, 2):
        for x, y in zip((h, W, t), make(N, V, D, F32, seed=seed, left_out=left_out)):
            x.copy_(y)
        b.dh.fill_(7.0), b.dweight.fill_(7.0)
        graph.replay()
        check(b, reference(h, W, t), ALL)
        c, d = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
        assert torch.equal(a.loss, c.loss) and torch.equal(a.total, c.total) and all(torch.equal(x, y) for x, y in zip(b, d))
        if left_out == 1.0:
            assert all(bool((x == 0).all()) for x in b)


@ROWS
@SIZES
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_in_their_row(bad, V, D, N):
    h, W, t = make(N, V, D, F32)
    clean = mwb.token_loss_gradient(h, W, t)
    h[N - 1, 3] = bad
    r, alone = mwb.token_loss_gradient(h, W, t), mwb.token_loss(h, W, t)
    assert not bool(torch.isfinite(r.loss[N - 1])) and not bool(torch.isfinite(r.dh[N - 1]).any())
    assert not bool(torch.isfinite(alone.loss[N - 1]))
    assert torch.equal(r.loss[:N - 1], clean.loss[:N - 1]) and torch.equal(r.dh[:N - 1], clean.dh[:N - 1])
    assert torch.equal(alone.loss[:N - 1], mwb.token_loss(torch.nan_to_num(h, 0.0, 0.0), W, t).loss[:N - 1])
    # the same row left out: nothing of it is read into anything
    t[N - 1] = -1
    r = mwb.token_loss_gradient(h, W, t)
    check(r, reference(h, W, t), ALL)


@ROWS
@SIZES
def test_repeated_calls_agree_bit_for_bit(V, D, N):
    h, W, t = make(N, V, D, F32, left_out=0.2)
    a, b = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
    for _ in range(3):
        c, d = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
        assert torch.equal(a.loss, c.loss) and torch.equal(a.total, c.total) and all(torch.equal(x, y) for x, y in zip(b, d))
