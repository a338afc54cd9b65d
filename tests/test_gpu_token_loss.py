"""mw_token_loss_* against the formulas in 64 bits, evaluated on the same inputs.

Tolerances.  u = 2^-24; ur: half a step of the result's type; S_ij = |scale| sum |h_i| |w_j|.
A logit: 16 products join an accumulator at a time, which may be cut off at its last place: (D / 16 + 8) 2^-23 S, and for
float operands, held in two terms of eleven bits, 2^-21 S more (what neither term holds, and the product of the two
second terms).  dz_ij follows with twice the largest such error of its row, relative to p_ij, and is rounded on its way:
twice to half precision for bf16 operands (2^-11 each), to 2^-21 for float ones; a value below 2^-38 of the largest may be
lost.  Its products are cut off as the logits' are, once for 16 terms: (K / 16 + 8) 2^-23 of the sum of absolute values,
or 2^-20 of it, whichever is more.  The sums over a row (V terms in blocks of 128) are good to 2^-18.
The loss: twice its row's largest logit error, and 2^-20 of |lse| + |z_t| + 1."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


def make(N, V, D, dtype, seed=0, left_out=0.0, lean=8.0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    h = torch.randn(N, D, generator=g, device="cuda") * std + lean * torch.rand(N, 1, generator=g, device="cuda") * W[t].float()
    h = h.to(dtype)
    if left_out:
        out = torch.rand(N, generator=g, device="cuda") < left_out
        t[out] = torch.where(torch.arange(N, device="cuda") % 2 == 0, -100, V)[out]
        h[out] = float("nan")
    return h, W, t


def reference(h, W, t, scale=1.0, weight=None):
    """Everything in 64 bits, with bounds: {name: (value, bound before the last rounding)}."""
    f32 = h.dtype == F32
    N, D = h.shape
    V = W.shape[0]
    on = (t >= 0) & (t < V)
    if weight is not None:
        on = on & (weight != 0)
    g = (on.double() / on.sum().clamp(min=1)) if weight is None else torch.where(on, weight.double(), 0.0)
    hd, Wd = torch.where(on[:, None], h.double(), 0.0), W.double()
    z, S = scale * hd @ Wd.T, abs(scale) * hd.abs() @ Wd.abs().T
    lse = torch.logsumexp(z, 1)
    at = torch.where(on, t.long(), 0)[:, None]
    zt = z.gather(1, at)[:, 0]
    loss = torch.where(on, lse - zt, 0.0)
    ez = ((D / 16 + 8) * 2.0 ** -23 + (2.0 ** -21 if f32 else 0.0)) * S.amax(1)
    eloss = torch.where(on, 2 * ez + 2.0 ** -20 * (lse.abs() + zt.abs() + 1), 0.0)
    p = torch.exp(z - lse[:, None])
    dz = p.scatter_add(1, at, -torch.ones_like(zt)[:, None])
    rel = (2 * ez + 2.0 ** -18)[:, None] + (2.0 ** -20 if f32 else 2.0 ** -10 * 1.01)
    # (of the target's p - 1 the part p is off as any p; the rounding is of the difference)
    edz = rel * p + (2.0 ** -20 if f32 else 2.0 ** -11 * 1.01) * dz.abs() + 2.0 ** -38
    dz, edz = g[:, None] * dz, g.abs()[:, None] * edz + (2.0 ** -38 * g.abs().max() if N else 0)
    edz = torch.where(on[:, None], edz, 0.0)
    cut = lambda k: max((k / 16 + 8) * 2.0 ** -23, 2.0 ** -20) + 2.0 ** -20
    s = abs(scale)
    out = {"loss": (loss, eloss), "total": ((g * loss).sum(), (g.abs() * (eloss + 2 * U * loss.abs())).sum() + U * (g * loss).sum().abs())}
    out["dh"] = (scale * dz @ Wd, s * (edz @ Wd.abs() + cut(V) * (dz.abs() @ Wd.abs())))
    out["dweight"] = (scale * dz.T @ hd, s * (edz.T @ hd.abs() + cut(N) * (dz.abs().T @ hd.abs())))
    return out


def check(r, want, names):
    for name in names:
        got, (value, bound) = getattr(r, name), want[name]
        assert got.shape == value.shape
        off = (got.double() - value).abs() - (bound + HALF[got.dtype] * (value.abs() + bound) + 1e-30)
        assert bool((off <= 0).all()), (name, float(off.max()), float((got.double() - value).abs().max()))


ALL = ("loss", "total", "dh", "dweight")
SIZES = [(1, 1, 1), (1, 2, 64), (2, 130, 3), (64, 64, 64), (100, 515, 67), (129, 257, 65), (255, 1000, 128), (300, 2049, 512),
         (257, 12345, 200), (1100, 700, 1030), (40, 40000, 96)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_loss_and_gradients(N, V, D, dtype):
    h, W, t = make(N, V, D, dtype, seed=N)
    want = reference(h, W, t)
    check(mwb.token_loss(h, W, t), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t.to(torch.int32)), want, ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,left_out", [(50, 0.5), (700, 0.9), (2500, 0.3), (2500, 1.0), (65, 1.0)])
def test_rows_left_out_hold_nan(N, left_out, dtype):
    h, W, t = make(N, 333, 136, dtype, seed=N, left_out=left_out)
    want = reference(h, W, t, scale=0.7)
    r = mwb.token_loss_gradient(h, W, t, scale=0.7)
    check(r, want, ALL)
    out = (t < 0) | (t >= 333)
    assert bool((r.loss[out] == 0).all() and (r.dh[out] == 0).all())
    check(mwb.token_loss(h, W, t, scale=0.7), want, ("loss", "total"))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_row_weights(dtype):
    h, W, t = make(400, 600, 192, dtype, left_out=0.2)
    w = torch.randn(400, device="cuda") * 3
    w[::7] = 0
    h[::7] = float("inf")                          # left out by their weight
    want = reference(h, W, t, weight=w)
    check(mwb.token_loss_gradient(h, W, t, row_weight=w), want, ALL)
    check(mwb.token_loss(h, W, t, row_weight=w), want, ("loss", "total"))
    w.mul_(1e-6)
    check(mwb.token_loss_gradient(h, W, t, row_weight=w), reference(h, W, t, weight=w), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("piece", [1, 64, 100, 256, 300, 5000])
def test_pieces_of_rows(piece, dtype):
    h, W, t = make(700, 300, 128, dtype, left_out=0.2)
    check(mwb.token_loss_gradient(h, W, t, piece_rows=piece), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, -2.0, 30.0])
def test_scales_and_sure_rows(scale, dtype):
    h, W, t = make(200, 500, 256, dtype, lean=20.0)
    check(mwb.token_loss_gradient(h, W, t, scale=scale), reference(h, W, t, scale=scale), ALL)


def test_wide_ranges_of_operands():
    """Operands of one magnitude far from one, and rows that differ by 2^20: float operands are scaled by one power of
    two a tensor, so what a small element loses is relative to the largest."""
    h, W, t = make(150, 400, 128, F32)
    check(mwb.token_loss_gradient(h * 2.0 ** 40, W * 2.0 ** -40, t), reference(h * 2.0 ** 40, W * 2.0 ** -40, t), ALL)
    hb, Wb, t = make(150, 400, 128, BF16)
    check(mwb.token_loss_gradient(hb * 2.0 ** 40, Wb * 2.0 ** -40, t), reference(hb * 2.0 ** 40, Wb * 2.0 ** -40, t), ALL)
    zero = torch.zeros_like(h)
    check(mwb.token_loss_gradient(zero, W, t), reference(zero, W, t), ALL)
    check(mwb.token_loss_gradient(h, torch.zeros_like(W), t), reference(h, torch.zeros_like(W), t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("at", [0, 1, 8])
def test_windows_of_wider_rows(dtype, at):
    N, V, D = 90, 210, 128
    h, W, t = make(N, V, D, dtype)
    wide = lambda x, fill: torch.full((x.shape[0], 301 if at == 1 else 304), fill, device="cuda").to(dtype)
    hw, Ww, dhw, dWw = wide(h, float("nan")), wide(W, float("nan")), wide(h, 7.0), wide(W, 7.0)
    win = lambda x: x[:, at:at + D]
    win(hw).copy_(h), win(Ww).copy_(W)
    r = mwb.token_loss_gradient(win(hw), win(Ww), t, dh=win(dhw), dweight=win(dWw))
    check(r, reference(h, W, t), ALL)
    for x in (dhw, dWw):
        assert bool((x[:, :at] == 7).all() and (x[:, at + D:] == 7).all())
    check(mwb.token_loss(win(hw), win(Ww), t), reference(h, W, t), ("loss", "total"))


def test_wanted_gradients_types_and_places():
    h, W, t = make(300, 200, 64, BF16, left_out=0.3)
    want = reference(h, W, t)
    full = mwb.token_loss_gradient(h, W, t)
    a = mwb.token_loss_gradient(h, W, t, want=(True, False))
    assert a.dweight is None and torch.equal(a.dh, full.dh)
    b = mwb.token_loss_gradient(h, W, t, want=(False, True), grad_dtype=F32)
    assert b.dh is None and b.dweight.dtype == F32
    check(b, want, ("loss", "total", "dweight"))
    c = mwb.token_loss_gradient(h, W, t, want=(False, False))
    assert c.dh is None and c.dweight is None and torch.equal(c.loss, full.loss)
    own = h.clone()
    d = mwb.token_loss_gradient(own, W, t, dh=own)
    assert d.dh is own and torch.equal(own, full.dh) and torch.equal(d.dweight, full.dweight)
    one = torch.randn(1, 64, device="cuda").to(BF16)
    e = mwb.token_loss_gradient(one.expand(300, 64), W, t)
    assert torch.equal(e.dh, mwb.token_loss_gradient(one.expand(300, 64).contiguous(), W, t).dh)


def test_no_rows():
    W = torch.randn(50, 64, device="cuda")
    r = mwb.token_loss_gradient(torch.empty(0, 64, device="cuda"), W, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert r.loss.shape == (0,) and float(r.total) == 0 and r.dh.shape == (0, 64) and bool((r.dweight == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_that_are_not_finite_stay_in_their_rows(dtype):
    h, W, t = make(200, 300, 64, dtype)
    h[5, 3], h[150, 0] = float("nan"), float("inf")
    r = mwb.token_loss_gradient(h, W, t)
    bad = torch.zeros(200, dtype=torch.bool, device="cuda")
    bad[5] = bad[150] = True
    assert not bool(torch.isfinite(r.loss[bad]).any()) and not bool(torch.isfinite(r.dh[bad]).any())
    assert bool(torch.isfinite(r.loss[~bad]).all() and torch.isfinite(r.dh[~bad]).all())
    hc = torch.where(bad[:, None], torch.zeros_like(h), h)
    w = torch.where(bad, 0.0, 1 / 200)
    want = reference(hc, W, t, weight=w)
    clean = mwb.TokenLoss(torch.where(bad, 0.0, r.loss), None, torch.where(bad[:, None], 0.0, r.dh.float()).to(dtype))
    check(clean, want, ("loss", "dh"))
    # a vocabulary's row of -inf is never chosen: h >= 0 makes its logits -inf (float operands are two terms, whose
    # products with an infinity have either sign: their logits are NaN, as documented)
    hp, W, t = make(60, 300, 64, dtype)
    hp = hp.abs() + 0.5
    t[t == 17] = 18
    W[17] = float("-inf")
    r = mwb.token_loss(hp, W, t)
    if dtype == F32:
        assert not bool(torch.isfinite(r.loss).any())
        return
    W2 = torch.cat([W[:17], W[18:]])
    check(r, reference(hp, W2, torch.where(t > 17, t - 1, t)), ("loss", "total"))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_repeated_calls_agree_bit_for_bit(dtype):
    h, W, t = make(777, 3001, 320, dtype, left_out=0.1)
    a = mwb.token_loss_gradient(h, W, t)
    for _ in range(3):
        b = mwb.token_loss_gradient(h, W, t)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gradient_against_differences():
    """Along a direction d of size 1 an entry: (f(h + e d) - f(h - e d)) / 2e is off by e^2 / 6 of the third derivative
    (logits move by |d| |w| < 4 a unit of e; at most 4^3) and by the total's error, 2^-18 of 10, over e."""
    h, W, t = make(128, 200, 64, F32, lean=2.0)
    e = 2.0 ** -6
    r = mwb.token_loss_gradient(h, W, t)
    for x, dx, f in ((h, r.dh, lambda v: mwb.token_loss(v, W, t).total), (W, r.dweight, lambda v: mwb.token_loss(h, v, t).total)):
        way = torch.randn_like(x) * (1.0 if x is h else 1 / 8)
        rise = (float(f(x + e * way)) - float(f(x - e * way))) / (2 * e)
        along = float((dx.double() * way.double()).sum())
        assert abs(rise - along) <= e * e / 6 * 64 + 2.0 ** -18 * 10 / e


def test_another_stream_and_a_captured_call():
    h, W, t = make(300, 900, 128, BF16, left_out=0.2)
    want = mwb.token_loss_gradient(h, W, t)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = mwb.token_loss_gradient(h, W, t, stream=side)
    only = mwb.token_loss(h, W, t, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = mwb.token_loss_gradient(h, W, t)
    for seed, out in ((3, 0.0), (4, 0.6)):
        new = make(300, 900, 128, BF16, seed=seed, left_out=out)
        for a, b in zip((h, W, t), new):
            a.copy_(b)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, mwb.token_loss_gradient(*new)))
