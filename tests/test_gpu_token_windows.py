"""The vocabulary's loss in windows of wider rows that start and repeat on 16-byte boundaries, with columns that do not end on one:
nothing beyond a row's last column is written, and what stands there is read into nothing.  Formulas and tolerances are
those of test_gpu_token_loss.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_token_loss import ALL, BF16, F32, check, make, reference

pytestmark = pytest.mark.gpu


def window(rows, D, dtype, fill):
    """(a tensor full of `fill`, its window of D columns): rows 32 bytes apart in their starts, 8 columns or more beyond."""
    wide = torch.full((rows, -(-D // 16) * 16 + 32), fill, device="cuda", dtype=dtype)
    return wide, wide[:, 16:16 + D]


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [1, 3, 62, 63, 64, 66, 157, 260, 515])
@pytest.mark.parametrize("N", [4, 20, 300, 700])
def test_columns_beyond_the_last_are_left_alone(N, D, dtype, kind):
    V = 600
    h, W, t = make(N, V, D, dtype, seed=N + D, left_out=0.2)
    want = reference(h, W, t)
    (hw, hv), (ww, wv) = window(N, D, dtype, float("nan")), window(V, D, dtype, float("nan"))
    hv.copy_(h), wv.copy_(W)
    check(mwb.token_loss(hv, wv, t), want, ("loss", "total"))
    for piece in (0, 256):
        (dh, dhv), (dw, dwv) = window(N, D, dtype, 7.0), window(V, D, kind, 7.0)
        check(mwb.token_loss_gradient(hv, wv, t, dh=dhv, dweight=dwv, piece_rows=piece), want, ALL)
        for x in (dh, dw):
            assert bool((x[:, :16] == 7).all() and (x[:, 16 + D:] == 7).all())


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("N", [20, 128])
def test_few_rows_over_a_large_weight(N, kind):
    V, D = 12353, 1024
    h, W, t = make(N, V, D, BF16, seed=N)
    (hw, hv), (ww, wv) = window(N, D, BF16, float("nan")), window(V, D, BF16, float("nan"))
    hv.copy_(h), wv.copy_(W)
    (dh, dhv), (dw, dwv) = window(N, D, BF16, 7.0), window(V, D, kind, 7.0)
    check(mwb.token_loss_gradient(hv, wv, t, dh=dhv, dweight=dwv), reference(h, W, t), ALL)
    for x in (dh, dw):
        assert bool((x[:, :16] == 7).all() and (x[:, 16 + D:] == 7).all())
