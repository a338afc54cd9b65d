"""Sequence-block operators and the orthogonalised update at the sizes of real nets: many rows a thread, many
matrices, many tiles, rows far apart.  Formulas in 64 bits and tolerances are those of the operators' own tests,
except where one is derived here."""
import numpy as np
import pytest

import test_gpu_gated_scan as scan
import test_gpu_residual_norm as norm
from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu

# every way of laying rows over threads (8 and 16 lanes, 1 to 16 warps), each with five rows and more a thread in the
# backward pass, so that the copies' rings wrap; widths that take 16-byte accesses and widths that do not
MANY_ROWS = [(48000, 64), (48000, 57), (24000, 128), (24000, 121), (12000, 256), (12000, 243), (6000, 512), (6000, 507),
             (3000, 1024), (3000, 1021), (1500, 2048), (1500, 2043), (750, 4096), (750, 4091), (400, 8192)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", MANY_ROWS, ids=lambda s: "x".join(map(str, s)))
def test_norm_of_many_rows(size, dtype):
    norm.run_and_check(*size, dtype, seed=size[1])


def project64(U, steps=5, coef=(3.4445, -4.7750, 2.0315)):
    """The iteration in 64 bits on the GPU, for a batch of matrices."""
    import torch
    a, b, c = coef
    X = U.double()
    X = X / torch.linalg.matrix_norm(X)[:, None, None]
    tall = X.shape[1] > X.shape[2]
    X = X.mT if tall else X
    for _ in range(steps):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.mT if tall else X


# more matrices than one launch of the small kernels takes, small and large; one to sixteen rows of tiles, odd ones
# and wide ones.  Tolerances as for smaller ones: a two-term sum is cut into pieces of 256 terms whatever its length,
# and a one-term sum of 4096 terms is truncated 256 times, 1.5e-5, well inside 5e-3.
ORTH = [(40, 48, 130), (64, 64, 65), (140, 150, 70), (1024, 1024, 2), (1100, 2500, 2), (2300, 900, 1), (4096, 4096, 1)]


@pytest.mark.parametrize("prec", ["f32", "bf16_f32acc"])
@pytest.mark.parametrize("shape", ORTH, ids=lambda s: "x".join(map(str, s)))
def test_projection_at_the_sizes_of_nets(shape, prec):
    import torch
    rows, cols, count = shape
    plan = mwb.Orth(rows, cols, count, prec)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    U = torch.randn(count, rows, cols, generator=g, device="cuda")
    U = (U * 10.0 ** torch.randint(-3, 4, (count, 1, 1), generator=g, device="cuda")).to(plan.storage_dtype())
    ws = plan.alloc_workspace()
    X = torch.stack(plan.project(list(U), ws)).double()
    assert plan.status(ws) == 0
    want = project64(U)
    err = torch.linalg.matrix_norm(X - want) / torch.linalg.matrix_norm(want)
    tol = 1e-4 if prec == "f32" else 5e-3 + 2.0 ** -9
    assert float(err.max()) <= tol


@pytest.mark.parametrize("prec", ["f32", "bf16_f32acc"])
@pytest.mark.parametrize("shape", [(40, 48, 130), (140, 150, 70), (1024, 1100, 3)], ids=lambda s: "x".join(map(str, s)))
def test_step_at_the_sizes_of_nets(shape, prec):
    import torch
    rows, cols, count = shape
    plan = mwb.Orth(rows, cols, count, prec)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rand = lambda: torch.randn(count, rows, cols, generator=g, device="cuda")
    W, G, M = (rand() / np.sqrt(cols)).to(plan.storage_dtype()), rand(), rand()
    lr, beta, wd, scale = 0.02, 0.9, 0.1, 0.2 * np.sqrt(max(rows, cols))
    m = beta * M.double() + G.double()
    X = project64(G.double() + beta * m)
    want = (1 - lr * wd) * W.double() - lr * scale * X
    ws = plan.alloc_workspace()
    plan.step(list(W), list(G), list(M), ws, lr, beta, wd, scale)
    assert plan.status(ws) == 0
    assert float((M.double() - m).abs().max()) <= 2.0 ** -22 * float(m.abs().max())
    size = torch.linalg.matrix_norm
    tol = lr * scale * (1e-4 if prec == "f32" else 5e-3) * size(X) + (2.0 ** -23 if prec == "f32" else 2.0 ** -8) * size(want)
    assert bool((size(W.double() - want) <= tol).all())


# rows 2^27 bytes apart, which only the walk addresses, and 2^25 bytes, which the other kernels do; either way the
# tensors' ends lie more than 2^31 bytes from their beginnings
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,apart", [(40, 27), (80, 25), (300, 25)])
def test_recurrence_over_rows_far_apart(T, apart, dtype):
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    D, row = 64, (1 << apart) // (4 if dtype == "f32" else 2)
    v, f, dy, h0, dh, _, _ = scan.make(1, T, D, dtype, seed=T + apart)
    wide = torch.empty((1, T, row), dtype=dt, device="cuda")
    at = lambda i: wide[:, :, row - (i + 1) * D:row - i * D]
    for i, t in enumerate((v, f, dy)):
        at(i).copy_(t)
    y, h_last, st = mwb.gated_scan(at(0), at(1), h0=h0, y=at(3), keep_states=True)
    dv, df, dh0 = mwb.gated_scan_backward(at(0), at(1), at(2), st, dh_last=dh, dv=at(4), df=at(5))
    assert y.data_ptr() == at(3).data_ptr() and dv.data_ptr() == at(4).data_ptr()
    V, F, G = (scan.f64(t) for t in (v, f, dy))
    ref = scan.reference(V, F, "complement", None, None, scan.f64(h0), G, scan.f64(dh))
    got = {k: scan.f64(t) for k, t in dict(y=y, h_last=h_last, dv=dv, df=df, dh0=dh0).items()}
    scan.check(got, ref, V, dtype)
    for i, t in enumerate((v, f, dy)):
        assert torch.equal(at(i), t)


# sequences of 30 to 70 steps with channels for every SM, on both sides of where the walk ends in either pass
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [30, 32, 33, 48, 64, 65])
def test_short_sequences_of_many_channels(T, dtype):
    got, ref, V = scan.run_both(230, T, 264, dtype, "energy", T % 2 == 0, seed=T)
    scan.check(got, ref, V, dtype)


# bf16 weights of few rows, or small ones, take two-term products: the same bits as when two are asked for.  (One-term
# products leave up to 9e-3 of X where only a few singular values share the error.)
@pytest.mark.parametrize("shape", [(1, 1, 20), (1, 6, 70), (2, 13, 70), (13, 2, 70), (3, 207, 30), (26, 123, 30), (64, 64, 8),
                                   (128, 256, 4), (3, 700, 20), (31, 1000, 4), (2000, 5, 6)], ids=lambda s: "x".join(map(str, s)))
def test_bf16_matrices_that_are_small_or_of_few_rows_take_two_terms(shape):
    import torch
    rows, cols, count = shape
    U = [torch.randn(rows, cols, device="cuda").bfloat16() for _ in range(count)]
    got = []
    for terms in (0, 2):
        plan = mwb.Orth(rows, cols, count, "bf16_f32acc", terms=terms)
        ws = plan.alloc_workspace()
        got.append(plan.project(U, ws))
        assert plan.status(ws) == 0
    assert all(torch.equal(p, q) for p, q in zip(*got))


# ... and two-term products are right there: fp32 weights, the tolerance of the other shapes
@pytest.mark.parametrize("shape", [(1, 1, 20), (1, 6, 70), (2, 13, 70), (13, 2, 70), (3, 207, 30), (26, 123, 30), (3, 700, 20),
                                   (31, 1000, 4), (2000, 5, 6)], ids=lambda s: "x".join(map(str, s)))
def test_projection_of_matrices_of_few_rows(shape):
    import torch
    rows, cols, count = shape
    plan = mwb.Orth(rows, cols, count, "f32")
    U = torch.randn(count, rows, cols, device="cuda")
    ws = plan.alloc_workspace()
    X = torch.stack(plan.project(list(U), ws)).double()
    want = project64(U)
    err = torch.linalg.matrix_norm(X - want) / torch.linalg.matrix_norm(want)
    assert plan.status(ws) == 0 and float(err.max()) <= 1e-4
