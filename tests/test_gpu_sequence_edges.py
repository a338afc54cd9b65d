"""Sequence-block operators at their edges: operands that share memory, values out of range, single far-out gates,
other streams and devices."""
import numpy as np
import pytest

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T", [1, 9, 300])
def test_expanded_scan_operands_equal_dense_ones(T, dtype):
    import torch
    dt = getattr(torch, dtype)
    B, D = 3, 72
    rand = lambda *s: torch.randn(*s, device="cuda").to(dt)
    for v, f, dy in ((rand(B, T, D), rand(1, 1, D).expand(B, T, D), rand(()).expand(B, T, D)),
                     (rand(1, T, D).expand(B, T, D), rand(B, 1, D).expand(B, T, D), rand(1, 1, D).expand(B, T, D)),
                     (rand(B, T, 1).expand(B, T, D), rand(B, T, D), rand(1, T, 1).expand(B, T, D))):
        y, hl, st = mwb.gated_scan(v, f, keep_states=True)
        g = mwb.gated_scan_backward(v, f, dy, st)
        dense = [t.contiguous() for t in (v, f, dy)]
        y2, hl2, st2 = mwb.gated_scan(*dense[:2], keep_states=True)
        g2 = mwb.gated_scan_backward(*dense, st2)
        assert all(torch.equal(a, b) for a, b in zip((y, hl, st) + g, (y2, hl2, st2) + g2))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_expanded_norm_operands_equal_dense_ones(dtype):
    import torch
    dt = getattr(torch, dtype)
    R, D = 37, 136
    rand = lambda *s: torch.randn(*s, device="cuda").to(dt)
    w = torch.rand(D, device="cuda") + 0.5
    dxo, dn = rand(R, D), rand(R, D)
    full = [rand(R, D) for _ in range(3)]
    for i in range(3):
        for shape in ((1, D), (R, 1), (1, 1)):
            ops = list(full)
            ops[i] = rand(*shape).expand(R, D)
            results = []
            for x, b, z in (ops, [t.contiguous() for t in ops]):
                kw = dict(z=z, w_post=w, scale=w, w_pre=w)
                xo, n, rms = mwb.residual_norm(x, b, keep_rms=True, **kw)
                results.append((xo, n) + tuple(mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, **kw)))
            assert all(torch.equal(p, q) for p, q in zip(*results))


def far_gates(T, D, B, gate, dtype, seed):
    """Gates that forget almost all, and the backward recurrence from dh_last alone in 64 bits."""
    import torch
    rng = np.random.default_rng(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    v = torch.from_numpy(rng.standard_normal((B, T, D))).to(dt).cuda()
    f = torch.from_numpy(np.linspace(-20, -6, D) + 0.5 * rng.standard_normal((B, T, D))).to(dt).cuda()
    h0, dh = (torch.from_numpy(rng.standard_normal((B, D))).float().cuda() for _ in range(2))
    V, F, H, g = (t.double().cpu().numpy() for t in (v, f, h0, dh))
    a, w = 1 / (1 + np.exp(-F)), 1 / (1 + np.exp(F))
    u = w if gate == "complement" else np.sqrt(w * (1 + a))
    slope = -a * w if gate == "complement" else -a * a * np.sqrt(w / (1 + a))
    before = np.zeros((B, T, D))
    for t in range(T):
        before[:, t] = H
        H = a[:, t] * H + u[:, t] * V[:, t]
    dv, df, size = np.zeros((B, T, D)), np.zeros((B, T, D)), np.zeros((B, T, D))
    for t in range(T - 1, -1, -1):
        dv[:, t] = u[:, t] * g
        df[:, t] = g * (a[:, t] * w[:, t] * before[:, t] + slope[:, t] * V[:, t])
        size[:, t] = np.abs(g) * (a[:, t] * w[:, t] * np.abs(before[:, t]) + np.abs(slope[:, t] * V[:, t]))
        g = a[:, t] * g
    return v, f, h0, dh, dv, df, size, g


# Each gate carries a relative error of (|f| + 4) 2^-24 (the rounding of f log2(e), then an exponential and a reciprocal
# of one or two units), so after k steps a cotangent is off by k (|f| + 4) 2^-24 of itself: |f| < 23 here.  bf16
# results add 2^-8 of their value.  Values below 1e-30 (products of a few gates) are left out: what they are multiplied
# from is near the smallest normal number.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["complement", "energy"])
@pytest.mark.parametrize("shape", [(2, 1, 64), (2, 15, 64), (2, 16, 64), (2, 17, 66), (2, 17, 64), (1, 400, 64), (1, 400, 66),
                                   (3, 2100, 64), (230, 40, 264)], ids=lambda s: "x".join(map(str, s)))
def test_cotangents_through_gates_that_forget(shape, gate, dtype):
    import torch
    B, T, D = shape
    v, f, h0, dh, dv, df, size, dh0 = far_gates(T, D, B, gate, dtype, sum(shape))
    _, _, st = mwb.gated_scan(v, f, h0=h0, input_gate=gate, keep_states=True)
    none = torch.zeros((B, T), dtype=torch.uint8, device="cuda")
    back = np.arange(T, 0, -1)[None, :, None]
    ulp = 2.0 ** -8 if dtype == "bf16" else 0.0
    for reset in (None, none):
        got = [t.double().cpu().numpy() for t in mwb.gated_scan_backward(v, f, None, st, reset=reset, dh_last=dh, input_gate=gate)]
        for g, want, scale, steps, r in ((got[0], dv, np.abs(dv), back + 1, ulp), (got[1], df, size, back + 1, ulp),
                                         (got[2], dh0, np.abs(dh0), T + 1, 0.0)):
            err = np.abs(g - want) - r * np.abs(want) - scale * steps * 27 * 2.0 ** -24
            assert (err[scale > 1e-30] <= 0).all()
            assert np.isfinite(g).all()


def scan_inputs(B, T, D, dtype, seed, logit=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    v, f, dy = (torch.randn(B, T, D, generator=g, device="cuda") for _ in range(3))
    h0 = torch.randn(B, D, generator=g, device="cuda")
    return v.to(dt), (f + logit).to(dt), dy.to(dt), h0


# 12 steps are walked, 400 are one piece of a few blocks, 3000 several
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 66])
@pytest.mark.parametrize("T", [12, 400, 3000])
def test_a_reset_keeps_out_a_gate_that_is_not_a_number(T, D, dtype):
    import torch
    v, f, dy, h0 = scan_inputs(1, T, D, dtype, 12)
    at = T // 2
    reset = torch.zeros((1, T), dtype=torch.uint8, device="cuda")
    reset[0, at] = 1
    y0, h_last0, st0 = mwb.gated_scan(v, f, reset=reset, h0=h0, keep_states=True)
    g0 = mwb.gated_scan_backward(v, f, dy, st0, reset=reset)
    before, after = f.clone(), f.clone()
    before[0, at - 3] = float("nan")
    after[0, at + 2] = float("nan")
    y, h_last, st = mwb.gated_scan(v, before, reset=reset, h0=h0, keep_states=True)
    assert torch.equal(y[:, at:], y0[:, at:]) and torch.equal(h_last, h_last0)
    assert bool(torch.isnan(y[:, at - 3:at]).all())
    g = mwb.gated_scan_backward(v, before, dy, st, reset=reset)
    assert torch.equal(g[0][:, at:], g0[0][:, at:]) and torch.equal(g[1][:, at:], g0[1][:, at:])
    _, _, st = mwb.gated_scan(v, after, reset=reset, h0=h0, keep_states=True)
    g = mwb.gated_scan_backward(v, after, dy, st, reset=reset)
    assert torch.equal(g[0][:, :at], g0[0][:, :at]) and torch.equal(g[1][:, :at], g0[1][:, :at])
    assert torch.equal(g[2], g0[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 66])
@pytest.mark.parametrize("T", [600, 3000])
def test_without_a_reset_a_nan_stays_however_strong_the_decay(T, D, dtype):
    # the product of the gates underflows on the way; the reset array is there, but empty
    import torch
    v, f, dy, h0 = scan_inputs(2, T, D, dtype, 3, logit=-1.0)
    reset = torch.zeros((2, T), dtype=torch.uint8, device="cuda")
    bad = v.clone()
    bad[1, 100, 5] = float("nan")
    for r in (reset, None):
        y, h_last, _ = mwb.gated_scan(bad, f, reset=r, h0=h0, keep_states=True)
        nan = torch.isnan(y)
        assert bool(nan[1, 100:, 5].all()) and int(nan.sum()) == T - 100
        assert bool(torch.isnan(h_last[1, 5])) and int(torch.isnan(h_last).sum()) == 1
    _, _, st = mwb.gated_scan(v, f, reset=reset, h0=h0, keep_states=True)
    worse = dy.clone()
    worse[1, T - 50, 7] = float("nan")
    for r in (reset, None):
        dv, df, dh0 = mwb.gated_scan_backward(v, f, worse, st, reset=r)
        for t in (dv, df):
            nan = torch.isnan(t)
            assert bool(nan[1, :T - 49, 7].all()) and int(nan.sum()) == T - 49
        assert bool(torch.isnan(dh0[1, 7])) and int(torch.isnan(dh0).sum()) == 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 66])
@pytest.mark.parametrize("T", [12, 600, 3000])
def test_an_infinite_state_stays_infinite(T, D, dtype):
    # the recurrence keeps it, however far the product of the gates after it has underflowed
    import torch
    v, f, dy, h0 = scan_inputs(2, T, D, dtype, 4, logit=-1.0)
    none = torch.zeros((2, T), dtype=torch.uint8, device="cuda")
    at = min(T // 3, 100)
    bad, worse = v.clone(), dy.clone()
    bad[0, at, 3], bad[1, at, 5] = float("inf"), -float("inf")
    worse[0, T - at, 3], worse[1, T - at, 5] = float("inf"), -float("inf")
    for reset in (None, none):
        y0, _ = mwb.gated_scan(v, f, reset=reset, h0=h0)
        y, h_last, st = mwb.gated_scan(bad, f, reset=reset, h0=h0, keep_states=True)
        assert bool((y[0, at:, 3] == float("inf")).all()) and bool((y[1, at:, 5] == -float("inf")).all())
        assert float(h_last[0, 3]) == float("inf") and float(h_last[1, 5]) == -float("inf")
        rest = torch.ones_like(y, dtype=torch.bool)
        rest[0, at:, 3] = rest[1, at:, 5] = False
        assert torch.equal(y[rest], y0[rest])
        _, _, st = mwb.gated_scan(v, f, reset=reset, h0=h0, keep_states=True)
        dv, _, dh0 = mwb.gated_scan_backward(v, f, worse, st, reset=reset)
        assert bool((dv[0, :T - at + 1, 3] == float("inf")).all()) and bool((dv[1, :T - at + 1, 5] == -float("inf")).all())
        assert float(dh0[0, 3]) == float("inf") and float(dh0[1, 5]) == -float("inf")
        assert int((~torch.isfinite(dv)).sum()) == 2 * (T - at + 1)


# rows of 8 and 16 lanes, one to sixteen warps, element by element, and a cluster
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 96, 264, 1003, 2048, 4096, 9000])
def test_what_does_not_depend_on_the_sum_is_not_spoilt_by_it(D, dtype):
    # without a cotangent of n, dx is dx_out, and db and dz hold no x: an infinity, a NaN or a number whose square
    # overflows in x leaves them as they are
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(D)
    x, b, z, dxo = (torch.randn(5, D, generator=g, device="cuda").to(dt) for _ in range(4))
    wp, sc, wn = (torch.rand(D, generator=g, device="cuda") + 0.5 for _ in range(3))
    bad = x.clone()
    bad[0, 3], bad[1, D - 1], bad[2, 7], bad[3, 5] = float("inf"), -float("inf"), float("nan"), 3e38
    b[3, 5] = 1e30
    for kw in (dict(w_post=wp, scale=sc, z=z), dict(w_post=wp), dict(scale=sc, z=z), dict(w_post=wp, scale=sc, z=z, w_pre=wn)):
        out = []
        for t in (x, bad):
            _, _, rms = mwb.residual_norm(t, b, keep_rms=True, **kw)
            out.append(mwb.residual_norm_backward(t, b, rms, dx_out=dxo, dn=None, **kw))
        want, got = out
        assert torch.equal(got.dx, dxo) and torch.equal(want.dx, dxo)
        for name in ("db", "dz", "dw_post", "dscale"):
            p, q = getattr(got, name), getattr(want, name)
            if p is not None:
                assert bool(torch.isfinite(p).all()) and torch.equal(p, q), name
        if got.dw_pre is not None:
            assert not got.dw_pre.any()


def test_inputs_dropped_while_another_stream_still_reads_them():
    # the stream is busy, the caller drops its only references and fills as much memory with something else
    import torch
    v, f, dy, h0 = scan_inputs(2, 700, 192, "bf16", 6)
    x, b, dxo, dn = (torch.randn(1500, 320, device="cuda").bfloat16() for _ in range(4))
    w = torch.rand(320, device="cuda") + 0.5
    mats = [torch.randn(96, 160, device="cuda") for _ in range(3)]
    plan = mwb.Orth(96, 160, 3, "f32")
    y, hl, st = mwb.gated_scan(v, f, h0=h0, keep_states=True)
    g = mwb.gated_scan_backward(v, f, dy, st)
    xo, n, rms = mwb.residual_norm(x, b, w_post=w, w_pre=w, keep_rms=True)
    gn = mwb.residual_norm_backward(x, b, rms, w_post=w, w_pre=w, dx_out=dxo, dn=dn)
    X = plan.project(mats, plan.alloc_workspace())
    s = torch.cuda.Stream()
    calls = [((v, f, h0), lambda v, f, h0: mwb.gated_scan(v, f, h0=h0, stream=s), (y, hl)),
             ((v, f, dy, st), lambda v, f, dy, st: mwb.gated_scan_backward(v, f, dy, st, stream=s), g),
             ((x, b, w), lambda x, b, w: mwb.residual_norm(x, b, w_post=w, w_pre=w, stream=s), (xo, n)),
             ((x, b, rms, w, dxo, dn),
              lambda x, b, rms, w, dxo, dn: mwb.residual_norm_backward(x, b, rms, w_post=w, w_pre=w, dx_out=dxo, dn=dn, stream=s),
              (gn.dx, gn.db, None, gn.dw_post, None, gn.dw_pre)),
             (tuple(mats) + (plan.alloc_workspace(),),
              lambda *t: plan.project(t[:3], t[3], out=[torch.empty_like(m) for m in t[:3]], stream=s), X)]
    for inputs, call, want in calls:
        copies = [t.clone() for t in inputs]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
        got = call(*copies)
        del copies
        other = [torch.full_like(t, 7) for t in inputs for _ in range(2)]
        torch.cuda.synchronize()
        assert len(got) == len(want)
        for p, q in zip(got, want):
            assert (p is None and q is None) or torch.equal(p, q)
        del other
