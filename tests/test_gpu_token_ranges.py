"""The vocabulary's loss of rows that differ by many powers of two: a row's loss and dh keep their digits whatever stands
beside it, in h or among the row weights.

Tolerances are those of test_gpu_token_loss.py, without what they allow a row for the weights of others: dh_i = g_i times the
dh_i of weight one, so its bound is |g_i| times the bound there.  In dweight the rows meet: h_i times 2^x, x by its weight,
is held in half precision (two terms of float operands) with the largest number at 2^13 and more, so each is off by 2^-25 of
that scale, and its dz, relative to its weight at most |p - [j = t]|, times 2^14: 2^-37 max_i(|g_i| max |h_i|) sum_i |p_ij - [j = t_i]|.
Where all rows are of the usual size that operand is the logits', whose rows have their largest number at 2^4 and more: each
is off by 2^-25 of that scale, 2^-29 of its row's largest: 2^-29 sum_i |g_i| max |h_i| |p_ij - [j = t_i]|."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import ALL, BF16, F32, check, make, reference

pytestmark = pytest.mark.gpu


def by_weight(want, w):
    """Values and bounds of dh of weight one, turned into those of the weights w."""
    value, bound = want["dh"]
    return dict(want, dh=(value * w.double()[:, None], bound * w.double().abs()[:, None]))


def meeting(want, h, W, t, w, scale=1.0):
    """dweight's bound with what rows of different sizes lose there."""
    p = torch.softmax(scale * h.double() @ W.double().T, 1)
    d = p.scatter_add(1, t[:, None], -torch.ones(len(t), 1, device="cuda", dtype=torch.float64)).abs()
    value, bound = want["dweight"]
    size = w.double().abs() * h.double().abs().amax(1)
    return dict(want, dweight=(value, bound + abs(scale) * (2.0 ** -37 * size.max() * d.sum(0) + 2.0 ** -29 * size @ d)[:, None]))


@pytest.mark.parametrize("N,dtype", [(5, F32), (9, F32), (100, F32), (300, F32), (9, BF16), (129, BF16), (300, BF16)])
@pytest.mark.parametrize("size", [-40, -20, 12, 20, 32, 60])
def test_one_row_far_larger_or_smaller_than_the_others(size, N, dtype):
    h, W, t = make(N, 700, 128, dtype, seed=N, lean=4.0)
    h[3] *= 2.0 ** size
    want = meeting(reference(h, W, t), h, W, t, torch.full((N,), 1 / N, device="cuda"))
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t), want, ALL)
    check(mwb.token_loss_gradient(h, W, t, piece_rows=256), want, ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [40, 300, 1500])
def test_rows_of_every_size(N, dtype):
    """Rows from 2^-30 to 2^30 beside one another, targets left out among them."""
    h, W, t = make(N, 333, 200, dtype, seed=N, lean=2.0)
    h *= torch.exp2((torch.arange(N, device="cuda") % 61 - 30.0))[:, None]
    t[::7] = -1
    h[::7] = float("nan")
    on = (t >= 0).float()
    want = reference(h, W, t)
    hc, tc = torch.where(on[:, None] > 0, h, torch.zeros_like(h)), t.clamp(min=0)
    want = meeting(want, hc, W, tc, on / on.sum())
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    for piece in (0, 256):
        check(mwb.token_loss_gradient(h, W, t, piece_rows=piece), want, ALL)


@pytest.mark.parametrize("N,dtype", [(8, F32), (9, F32), (100, F32), (300, F32), (9, BF16), (129, BF16), (300, BF16)])
@pytest.mark.parametrize("light", [1e-3, 1e-6, 1e-8, 2.0 ** -40, 2.0 ** -80])
def test_light_rows_keep_their_digits(light, N, dtype):
    h, W, t = make(N, 700, 128, dtype, seed=N, lean=4.0)
    w = torch.rand(N, device="cuda") + 0.5
    w[1::2] *= light
    w[::5] *= -1
    one = reference(h, W, t, weight=torch.ones(N, device="cuda"))
    want = dict(reference(h, W, t, weight=w), dh=by_weight(one, w)["dh"])
    want = meeting(want, h, W, t, w)
    for piece in (0, 256):
        check(mwb.token_loss_gradient(h, W, t, row_weight=w, piece_rows=piece), want, ALL)


@pytest.mark.parametrize("N,dtype", [(8, F32), (9, F32), (300, F32), (129, BF16), (300, BF16), (1500, BF16)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_weight_that_is_not_finite_stays_in_its_row(bad, N, dtype):
    h, W, t = make(N, 700, 128, dtype, seed=N, lean=4.0)
    w = torch.full((N,), 2.0 ** -13, device="cuda")
    w[4] = bad
    one = reference(h, W, t, weight=torch.ones(N, device="cuda"))
    r = mwb.token_loss_gradient(h, W, t, row_weight=w)
    assert not bool(torch.isfinite(r.dh[4]).any()) and not bool(torch.isfinite(r.total))
    rest = torch.arange(N, device="cuda") != 4
    w[4] = 1.0
    want = by_weight(one, w)
    value, bound = (x[rest] for x in want["dh"])
    check(mwb.TokenLoss(r.loss, None, r.dh[rest]), dict(want, dh=(value, bound)), ("loss", "dh"))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_and_rows_of_every_size(dtype):
    """Weights and rows of h go against one another, so that g_i h_i is of one size and every row counts in dweight."""
    N = 700
    h, W, t = make(N, 333, 136, dtype, lean=2.0)
    x = torch.exp2(torch.arange(N, device="cuda") % 41 - 20.0)
    h, w = h * x[:, None].to(dtype), (torch.rand(N, device="cuda") + 0.5) / x
    one = reference(h, W, t, weight=torch.ones(N, device="cuda"))
    want = dict(reference(h, W, t, weight=w), dh=by_weight(one, w)["dh"])
    want = meeting(want, h, W, t, w)
    for piece in (0, 256):
        check(mwb.token_loss_gradient(h, W, t, row_weight=w, piece_rows=piece), want, ALL)


def test_captured_calls_of_even_and_uneven_rows():
    """One graph, replayed on rows of one size and of many, with weights alike and not."""
    N, V, D = 300, 500, 128
    h, W, t = make(N, V, D, BF16)
    w = torch.full((N,), 1 / N, device="cuda")
    call = lambda: mwb.token_loss_gradient(h, W, t, row_weight=w)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for size, weight in ((0, 0), (24, 0), (0, 24), (24, 24), (0, 0)):
        for a, b in zip((h, W, t), make(N, V, D, BF16, seed=size + weight)):
            a.copy_(b)
        h[5] *= 2.0 ** size
        w[6] = 2.0 ** weight / N
        graph.replay()
        got = [x.clone() for x in held]
        assert all(torch.equal(a, b) for a, b in zip(got, call()))


@pytest.mark.parametrize("N,dtype", [(8, F32), (9, F32), (300, F32), (9, BF16), (300, BF16)])
@pytest.mark.parametrize("size", [-118, -105, 105, 118])
def test_operands_near_the_ends_of_the_range(size, N, dtype):
    h, W, t = make(N, 700, 128, dtype, seed=N, lean=4.0)
    h, W = h * 2.0 ** size, W * 2.0 ** -size
    want = reference(h, W, t)
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t), want, ALL)
    h[3] *= 2.0 ** (-size // 2)
    want = meeting(reference(h, W, t), h, W, t, torch.full((N,), 1 / N, device="cuda"))
    check(mwb.token_loss_gradient(h, W, t), want, ALL)


SIZED = [(8, F32, 700, 128), (100, F32, 700, 128), (300, BF16, 700, 128), (20, BF16, 12353, 1088)]


@pytest.mark.parametrize("size,N,dtype,V,D", [(2.0 ** x, *s) for x in (-108, 100) for s in SIZED] + [(2.0 ** -114, *s) for s in SIZED[1:]])
def test_weights_near_the_ends_of_the_range(size, N, dtype, V, D):
    """W lies so that dh of weight one is of the size of 1 / size: what is formed of them does not end where they do."""
    h, W, t = make(N, V, D, dtype, seed=N, lean=4.0)
    h, W = h * size, W * (1 / size)
    w = (torch.rand(N, device="cuda") + 0.5) * size
    one = reference(h, W, t, weight=torch.ones(N, device="cuda"))
    r = mwb.token_loss_gradient(h, W, t, row_weight=w, want=(True, False))
    check(r, by_weight(one, w), ("loss", "dh"))


@pytest.mark.parametrize("N,dtype", [(8, F32), (9, F32), (300, F32), (9, BF16), (300, BF16)])
@pytest.mark.parametrize("size", [-16, -9, -6, -3, 0, 5])
def test_small_columns_of_rows_of_any_size(size, N, dtype):
    """Columns of h 2^-14 below the others, which no sum hides in dweight: what they lose goes by their row's largest."""
    h, W, t = make(N, 333, 128, dtype, seed=N, lean=0.0)
    h *= 2.0 ** size
    h[:, :16] *= 2.0 ** -14
    want = meeting(reference(h, W, t), h, W, t, torch.full((N,), 1 / N, device="cuda"))
    check(mwb.token_loss_gradient(h, W, t), want, ALL)
    g = torch.rand(N, device="cuda") + 0.5
    want = meeting(reference(h, W, t, weight=g), h, W, t, g)
    check(mwb.token_loss_gradient(h, W, t, row_weight=g), want, ALL)
