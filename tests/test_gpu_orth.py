"""mw_orth_* against the iteration in 64 bits.

Tolerances, relative in the Frobenius norm of X.  One step's polynomial moves a relative error e of its
operands by at most (|c0| + 2 |c1| + 3 |c2|) e < 20 e, and the steps contract towards 1 once the singular
values are there.  Operands of two terms carry 2^-22, accumulation over K up to K/16 truncations of 2^-24:
below 2.5e-6 for the sizes here, 5e-5 in all, doubled for ill-conditioned inputs: 1e-4.  Operands of one
term carry half a unit of 11 bits, 2^-12, whose sign is random: 20 x 2^-12 = 5e-3 in all.  bf16 results add
their own rounding, 2^-9.  The update adds lr scale times that to W's own rounding."""
import numpy as np
import pytest

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)
TOL = {1: 5e-3, 2: 1e-4}


def project(U, steps=5, coef=COEF):
    a, b, c = coef
    n = np.linalg.norm(U)
    X = U / n if n > 0 else U.copy()
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    for _ in range(steps):
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.T if tall else X


def tensors(arrays, dtype):
    import torch
    dt = {"f32": torch.float32, "bf16_f32acc": torch.bfloat16}[dtype]
    return [torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda() for a in arrays]


def f64(t):
    return t.double().cpu().numpy()


def rel(a, b):
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


SHAPES = [(1, 1, 2), (1, 9, 1), (7, 3, 2), (33, 65, 3), (64, 64, 2), (128, 128, 1), (70, 130, 2), (200, 96, 3), (128, 256, 3), (250, 128, 2), (128, 300, 1), (129, 200, 1), (513, 520, 14),
          (256, 256, 2), (257, 300, 2), (512, 192, 1), (640, 640, 2), (1000, 260, 1)]


@pytest.mark.parametrize("prec", ["f32", "bf16_f32acc"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_projection_matches_the_iteration(shape, prec):
    rows, cols, count = shape
    rng = np.random.default_rng(rows + cols)
    U = tensors([rng.standard_normal((rows, cols)) * 10.0 ** rng.integers(-3, 4) for _ in range(count)], prec)
    plan = mwb.Orth(rows, cols, count, prec)
    ws = plan.alloc_workspace()
    X = plan.project(U, ws)
    assert plan.status(ws) == 0
    tol = TOL[2] if prec == "f32" else TOL[1] + 2.0 ** -9
    for u, x in zip(U, X):
        assert rel(f64(x), project(f64(u))) <= tol


@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("kind", ["low_rank", "decay", "orthogonal", "one_row", "equal_rows"])
def test_projection_of_special_matrices(kind, terms):
    rng = np.random.default_rng(3)
    m, n = 192, 320
    if kind == "low_rank":
        U = rng.standard_normal((m, 6)) @ rng.standard_normal((6, n))
    elif kind == "decay":
        q, _ = np.linalg.qr(rng.standard_normal((m, m)))
        p, _ = np.linalg.qr(rng.standard_normal((n, m)))
        U = (q * np.exp(-np.linspace(0, 6, m))) @ p.T
    elif kind == "orthogonal":
        U = np.linalg.qr(rng.standard_normal((n, m)))[0].T * 17.0
    elif kind == "one_row":
        U = np.zeros((m, n))
        U[5] = rng.standard_normal(n)
    else:
        U = np.tile(rng.standard_normal((1, n)), (m, 1))
    plan = mwb.Orth(m, n, 1, "f32", terms=terms)
    ws = plan.alloc_workspace()
    u = tensors([U], "f32")
    x = plan.project(u, ws)[0]
    assert rel(f64(x), project(f64(u[0]))) <= TOL[terms]


@pytest.mark.parametrize("prec", ["f32", "bf16_f32acc"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(64, 64, 3), (130, 70, 2), (256, 512, 2), (301, 301, 1)],
                         ids=lambda s: "x".join(map(str, s)))
def test_step_matches_the_formula(shape, prec, nesterov):
    import torch
    rows, cols, count = shape
    rng = np.random.default_rng(11)
    W = tensors([rng.standard_normal((rows, cols)) / np.sqrt(cols) for _ in range(count)], prec)
    G, M = (tensors([rng.standard_normal((rows, cols)) for _ in range(count)], "f32") for _ in range(2))
    lr, beta, wd, scale = 0.02, 0.9, 0.1, 0.2 * np.sqrt(max(rows, cols))
    plan = mwb.Orth(rows, cols, count, prec, nesterov=nesterov)
    ws = plan.alloc_workspace()
    W2, M2 = [torch.empty_like(t) for t in W], [torch.empty_like(t) for t in M]
    plan.step(W, G, M, ws, lr, beta, wd, scale, params_out=W2, momentum_out=M2)
    for i in range(count):
        m = beta * f64(M[i]) + f64(G[i])
        X = project(f64(G[i]) + beta * m if nesterov else m)
        want = (1 - lr * wd) * f64(W[i]) - lr * scale * X
        assert np.abs(f64(M2[i]) - m).max() <= 2.0 ** -22 * np.abs(m).max()
        tol = lr * scale * TOL[2 if prec == "f32" else 1] * np.linalg.norm(X)
        tol += (2.0 ** -23 if prec == "f32" else 2.0 ** -8) * np.linalg.norm(want)
        assert np.linalg.norm(f64(W2[i]) - want) <= tol
    # in place: the same bits
    plan.step(W, G, M, ws, lr, beta, wd, scale)
    assert all(torch.equal(a, b) for a, b in zip(W + M, W2 + M2))
    assert plan.status(ws) == 0


def test_zero_nan_and_extreme_scales_stay_with_their_matrix():
    import torch
    rng = np.random.default_rng(2)
    base = rng.standard_normal((96, 160))
    U = tensors([np.zeros_like(base), base * 1e-18, base, base * 1e18, base], "f32")
    U[4][3, 7] = float("nan")
    plan = mwb.Orth(96, 160, 5, "f32")
    ws = plan.alloc_workspace()
    X = plan.project(U, ws)
    assert not X[0].any()
    for i in (1, 2, 3):
        assert rel(f64(X[i]), project(f64(U[i]))) <= TOL[2]
    assert bool(torch.isnan(X[4]).all()) and plan.status(ws) == 0


def test_other_step_counts_and_coefficients():
    rng = np.random.default_rng(4)
    U = tensors([rng.standard_normal((128, 200))], "f32")
    for steps, coef in ((1, COEF), (2, COEF), (8, COEF), (12, (1.5, -0.5, 0.0))):
        plan = mwb.Orth(128, 200, 1, "f32", steps=steps, coef=coef)
        x = plan.project(U, plan.alloc_workspace())[0]
        assert rel(f64(x), project(f64(U[0]), steps, coef)) <= TOL[2], steps


def test_a_workspace_serves_several_calls_and_streams():
    import torch
    rng = np.random.default_rng(5)
    a = tensors([rng.standard_normal((300, 300)) for _ in range(2)], "bf16_f32acc")
    b = tensors([rng.standard_normal((300, 300)) for _ in range(2)], "bf16_f32acc")
    plan = mwb.Orth(300, 300, 2, "bf16_f32acc")
    ws = plan.alloc_workspace()
    ws.fill_(255)                       # nothing in it may matter
    xa, xb = plan.project(a, ws), plan.project(b, ws)
    other = plan.alloc_workspace()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        xa2 = plan.project(a, other)
    s.synchronize()
    xb2 = plan.project(b, other)
    assert all(torch.equal(p, q) for p, q in zip(xa + xb, xa2 + xb2))
    inplace = [t.clone() for t in a]
    plan.project(inplace, ws, out=inplace)
    assert all(torch.equal(p, q) for p, q in zip(inplace, xa))


def test_refusals():
    import torch
    for kw in (dict(rows=0, cols=4), dict(rows=4, cols=4, count=0), dict(rows=4, cols=4, prec="f64"),
               dict(rows=4, cols=4, steps=17), dict(rows=4, cols=4, terms=3),
               dict(rows=4, cols=4, coef=(float("nan"), 0, 0))):
        with pytest.raises(mwb.MwError):
            mwb.Orth(**kw)
    plan = mwb.Orth(8, 8, 2, "f32")
    ws = plan.alloc_workspace()
    t = [torch.zeros((8, 8), device="cuda") for _ in range(2)]
    for bad in (lambda: plan.project(t[:1], ws), lambda: plan.project([t[0], t[1].bfloat16()], ws),
                lambda: plan.project([t[0], t[1][:4]], ws), lambda: plan.project([t[0], t[1].cpu()], ws), lambda: plan.project(t, ws[:512]),
                lambda: plan.step(t, t, t, ws, lr=float("inf"))):
        with pytest.raises((ValueError, mwb.MwError)):
            bad()
