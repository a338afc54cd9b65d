"""mw_residual_norm_* against the formulas in 64 bits.

Tolerances (u = 2^-24).  A mean of squares of D terms is good to (log2 D + 8) u < 24 u, its inverse root to
half of that; x' and n are a handful of products: 32 u of the row's largest value.  The cotangents sum three
such terms whose sizes are bounded by |dx_out| + |q| (|xh|^2 + 1) ...: 256 u of the largest value in the
row's sums.  Sums over R rows add R u sqrt-wise, bounded here by 1e-5 of the sum of absolute values.
bf16 results add half a unit in the last place: 2^-8 of the value with room for the double rounding.
"""
import numpy as np
import pytest

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def reference(x, b, z, wp, sc, wn, eps, dxo=None, dn=None):
    R, D = x.shape
    bh = xh = None
    xo, t, p = x, None, None
    sig = None
    if b is not None:
        rb = 1 / np.sqrt((b * b).mean(1, keepdims=True) + eps) if wp is not None else np.ones((R, 1))
        bh = b * rb
        p = bh * (1.0 if wp is None else wp)
        sig = None if z is None else 1 / (1 + np.exp(-z))
        gate = 1.0 if z is None else z * sig
        t = (1.0 if sc is None else sc) * gate * np.ones_like(x)
        xo = x + t * p
    out = {"x_out": xo, "n": None}
    rx = 1 / np.sqrt((xo * xo).mean(1, keepdims=True) + eps)
    xh = xo * rx
    if wn is not None:
        out["n"] = xh * wn
    if dxo is None and dn is None:
        return out
    dxo = np.zeros_like(x) if dxo is None else dxo
    dx = dxo
    if wn is not None:
        d = np.zeros_like(x) if dn is None else dn
        q = d * wn
        dx = dxo + rx * (q - xh * (q * xh).mean(1, keepdims=True))
        out["dw_pre"], out["dw_pre_abs"] = (d * xh).sum(0), np.abs(d * xh).sum(0)
    out["dx"] = dx
    if b is not None:
        dp = dx * t
        if wp is not None:
            q = dp * wp
            out["db"] = rb * (q - bh * (q * bh).mean(1, keepdims=True))
            out["dw_post"], out["dw_post_abs"] = (dp * bh).sum(0), np.abs(dp * bh).sum(0)
        else:
            out["db"] = dp
        if z is not None:
            out["dz"] = dx * (1.0 if sc is None else sc) * p * sig * (1 + z * (1 - sig))
        if sc is not None:
            e = dx * (1.0 if z is None else z * sig) * p
            out["dscale"], out["dscale_abs"] = e.sum(0), np.abs(e).sum(0)
    return out


def make(R, D, dtype, seed, have="bzpsn", pad=0):
    import torch
    rng = np.random.default_rng(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def put(x):
        if pad:
            wide = torch.full((R, D + 2 * pad), float("nan"), dtype=dt, device="cuda")
            w = wide[:, pad:pad + D]
        else:
            w = torch.empty((R, D), dtype=dt, device="cuda")
        w.copy_(torch.from_numpy(x).to(dt))
        return w

    def vec(mean):
        return torch.from_numpy(mean + 0.2 * rng.standard_normal(D)).float().cuda()

    x = put(2 * rng.standard_normal((R, D)))
    b = put(rng.standard_normal((R, D)) * 0.7) if "b" in have else None
    z = put(rng.standard_normal((R, D))) if "z" in have else None
    wp = vec(1.0) if "p" in have else None
    sc = vec(0.4) if "s" in have else None
    wn = vec(1.0) if "n" in have else None
    dxo, dn = (torch.from_numpy(rng.standard_normal((R, D))).to(dt).cuda() for _ in range(2))
    return x, b, z, wp, sc, wn, dxo, dn if "n" in have else None


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def run_and_check(R, D, dtype, have="bzpsn", pad=0, seed=0, eps=1e-6):
    x, b, z, wp, sc, wn, dxo, dn = make(R, D, dtype, seed, have, pad)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn, eps=eps)
    xo, n, rms = mwb.residual_norm(x, b, keep_rms=True, **kw)
    g = mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, **kw)
    ref = reference(*(f64(t) for t in (x, b, z, wp, sc, wn)), eps, f64(dxo), f64(dn))
    ulp = 2.0 ** -8 if dtype == "bf16" else 0.0
    big = np.abs(ref["x_out"]).max(1, keepdims=True) + 1
    for name, t in (("x_out", xo), ("n", n)):
        if ref[name] is None:
            assert t is None
            continue
        tol = 32 * U * big * (1 if name == "x_out" else max(1.0, float(np.abs(f64(wn)).max()))) + ulp * np.abs(ref[name])
        scale = 1.0 if name == "x_out" else 1 / np.sqrt((ref["x_out"] ** 2).mean(1, keepdims=True) + eps)
        assert (np.abs(f64(t) - ref[name]) <= tol * np.maximum(1.0, scale)).all(), name
    for name in ("dx", "db", "dz"):
        t = getattr(g, name)
        if name not in ref:
            assert t is None, name
            continue
        size = np.abs(ref[name]).max(1, keepdims=True) + np.abs(ref["dx"]).max(1, keepdims=True)
        # (a row of almost no spread, D = 1 above all, is the difference of two equal terms: their size counts)
        amp = 1.0
        if name == "db" and wp is not None:
            amp = max(1.0, float((1 / np.sqrt((f64(b) ** 2).mean(1) + eps)).max()))
        if wn is not None:
            amp *= max(1.0, float((1 / np.sqrt((ref["x_out"] ** 2).mean(1) + eps)).max()))
        err = np.abs(f64(t) - ref[name])
        assert (err <= 256 * U * amp * (size + 4) + ulp * np.abs(ref[name])).all(), (name, err.max())
    for name in ("dw_post", "dscale", "dw_pre"):
        t = getattr(g, name)
        if name not in ref:
            assert t is None, name
            continue
        assert (np.abs(f64(t) - ref[name]) <= 1e-5 * (ref[name + "_abs"] + 1) * (1 if D > 4 else 100)).all(), name


SIZES = [(1, 1), (1, 8), (3, 2), (2, 33), (5, 64), (7, 100), (4, 512), (3, 513), (9, 1000), (300, 1024), (2, 1111),
         (33, 2048), (5, 4096), (3, 5000), (700, 264), (2, 8192), (2, 16384), (1, 20001), (2, 32768),
         (3000, 16), (1500, 72), (400, 96), (200, 8200), (170, 5003), (60, 16392), (40, 32760)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
def test_forward_and_backward_match_the_formulas(size, dtype):
    run_and_check(*size, dtype, seed=size[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("have", ["n", "b", "bn", "bp", "bzn", "bs", "bps", "bzs", "bpsn", "bzpn"])
def test_parts_left_out(have, dtype):
    run_and_check(6, 200, dtype, have=have, seed=1)


@pytest.mark.parametrize("pad", [1, 8])
def test_windows_of_wider_rows(pad):
    run_and_check(10, 256, "bf16", pad=pad, seed=2)
    run_and_check(10, 256, "f32", pad=pad, seed=2)


def test_in_place_and_none_cotangents():
    import torch
    x, b, z, wp, sc, wn, dxo, dn = make(20, 384, "bf16", 3)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn)
    xo, n, rms = mwb.residual_norm(x, b, keep_rms=True, **kw)
    g0 = mwb.residual_norm_backward(x, b, rms, dx_out=torch.zeros_like(dxo), dn=dn, **kw)
    g1 = mwb.residual_norm_backward(x, b, rms, dx_out=None, dn=dn, **kw)
    assert all(torch.equal(p, q) for p, q in zip(g0, g1))
    g2 = mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=None, **kw)
    g3 = mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=torch.zeros_like(dn), **kw)
    assert all(torch.equal(p, q) for p, q in zip(g2, g3)) and not g2.dw_pre.any()
    x2 = x.clone()
    xo2, n2 = mwb.residual_norm(x2, b, x_out=x2, **kw)
    assert torch.equal(xo, xo2) and torch.equal(n, n2) and xo2.data_ptr() == x2.data_ptr()


def test_zero_rows_of_input_zero_rows_and_large_values():
    import torch
    # a row of zeros: eps keeps the norm finite; no rows at all: the sums are zero
    w = torch.ones(64, device="cuda")
    x = torch.zeros((2, 64), device="cuda")
    xo, n, rms = mwb.residual_norm(x, x, w_post=w, w_pre=w, keep_rms=True)
    assert not xo.any() and not n.any()
    g = mwb.residual_norm_backward(x, x, rms, w_post=w, w_pre=w, dx_out=torch.ones_like(x), dn=torch.ones_like(x))
    assert all(bool(torch.isfinite(t).all()) for t in g if t is not None)
    e = torch.empty((0, 64), device="cuda")
    xo, n, rms = mwb.residual_norm(e, e, w_post=w, w_pre=w, keep_rms=True)
    g = mwb.residual_norm_backward(e, e, rms, w_post=w, w_pre=w, dx_out=e, dn=e)
    assert xo.shape == (0, 64) and not g.dw_post.any() and not g.dw_pre.any()
    # a gate far out on either side; a NaN stays in its row
    z = torch.tensor([[1e4] * 64, [-1e4] * 64], device="cuda")
    b = torch.randn((2, 64), device="cuda")
    xo, _ = mwb.residual_norm(x, b, z=z)
    assert bool(torch.isfinite(xo).all()) and not xo[1].any()
    b[0, 5] = float("nan")
    xo, n = mwb.residual_norm(x, b, w_post=w, w_pre=w)
    assert bool(torch.isnan(n[0]).all()) and bool(torch.isfinite(n[1]).all())


def test_repeated_calls_and_other_streams_give_the_same_bits():
    import torch
    x, b, z, wp, sc, wn, dxo, dn = make(1500, 320, "bf16", 5)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn)

    def once(stream=None):
        xo, n, rms = mwb.residual_norm(x, b, keep_rms=True, stream=stream, **kw)
        return (xo, n) + tuple(mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, stream=stream, **kw))

    a = once()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c = once()
    d = once(s)                       # tensors of one stream, work on another
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, c)) and all(torch.equal(p, q) for p, q in zip(a, d))


def test_work_on_another_stream_does_not_meet_freed_memory():
    # a tensor freed while the current stream still has to write it: its memory must not become the output of a
    # call on another stream, which does not wait for that write
    import torch
    x, b, z, wp, sc, wn, dxo, dn = make(1500, 320, "bf16", 5)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn)
    xo, n, rms = mwb.residual_norm(x, b, keep_rms=True, **kw)
    g = mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, **kw)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty_like(t) for t in (xo, n, rms) + tuple(g)]
    torch.cuda._sleep(20_000_000)
    for t in old:
        t.fill_(7.0)
    del old, t
    xo2, n2, rms2 = mwb.residual_norm(x, b, keep_rms=True, stream=s, **kw)
    g2 = mwb.residual_norm_backward(x, b, rms2, dx_out=dxo, dn=dn, stream=s, **kw)
    torch.cuda.synchronize()
    for p, q in zip((xo, n, rms) + tuple(g), (xo2, n2, rms2) + tuple(g2)):
        assert torch.equal(p, q)


def test_gradients_match_differences():
    # directional derivatives of sum(dx_out x') + sum(dn n) in 64 bits; central differences of step 1e-4 are
    # good to 1e-6 of the terms they sum, the fp32 gradients to 2e-5 of them
    x, b, z, wp, sc, wn, dxo, dn = make(6, 90, "f32", 7)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn)
    _, _, rms = mwb.residual_norm(x, b, keep_rms=True, **kw)
    grads = [f64(t) for t in mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, **kw)]
    args = [f64(t) for t in (x, b, z, wp, sc, wn)]
    G, N = f64(dxo), f64(dn)

    def loss(a):
        o = reference(*a, 1e-6)
        return float((o["x_out"] * G).sum() + (o["n"] * N).sum())

    rng = np.random.default_rng(1)
    for i in range(6):
        d = rng.standard_normal(args[i].shape)
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + 1e-4 * d, args[i] - 1e-4 * d
        num = (loss(hi) - loss(lo)) / 2e-4
        ana = float((grads[i] * d).sum())
        assert abs(num - ana) <= 2e-5 * float(np.abs(grads[i] * d).sum()) + 1e-5, (i, num, ana)


def test_refusals():
    import torch
    x = torch.zeros((4, 32), device="cuda")
    w = torch.ones(32, device="cuda")
    for bad in (lambda: mwb.residual_norm(x.double()), lambda: mwb.residual_norm(x, x.bfloat16()),
                lambda: mwb.residual_norm(x, x[:2]), lambda: mwb.residual_norm(x, z=x),
                lambda: mwb.residual_norm(x, w_post=w), lambda: mwb.residual_norm(x, x, w_post=w[:3]),
                lambda: mwb.residual_norm(x, x, w_post=w, eps=0.0), lambda: mwb.residual_norm(x[:, ::2], None, w_pre=w),
                lambda: mwb.residual_norm(torch.zeros((1, 32769), device="cuda")),
                lambda: mwb.residual_norm(x, x, w_post=w.cpu()), lambda: mwb.residual_norm(x.cpu(), x.cpu()),
                lambda: mwb.residual_norm_backward(x, x, torch.ones((2, 4), device="cuda"), dn=x)):
        with pytest.raises((TypeError, ValueError, mwb.MwError)):
            bad()
