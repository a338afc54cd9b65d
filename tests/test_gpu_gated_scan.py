"""mw_gated_scan_* against the recurrence written out in 64 bits.

Tolerances.  The gate a = sigmoid(f) carries a relative error of a few 2^-24 in 1 - a, which moves h by
the same share of max|h|; each step adds a rounding of 2^-24 max|h|, remembered for 1/(1 - a) steps.
With f <= 5 that is at most 150 steps: 1e-5 max|h| in all.  df is a product of two such quantities:
4e-5 of the product of their maxima.  bf16 results add half a unit in the last place, 2^-8 of the value
with room for the double rounding.
"""
import numpy as np
import pytest

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu


def reference(v, f, gate, reset=None, lengths=None, h0=None, dy=None, dh_last=None):
    """Everything in numpy float64; loops over time."""
    B, T, D = v.shape
    with np.errstate(over="ignore"):
        a, w = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    u = w if gate == "complement" else np.sqrt(w * (1 + a))
    slope = -a * w if gate == "complement" else -a * a * np.sqrt(w / (1 + a))    # a (1 - a) du/da
    r = np.ones((B, T)) if reset is None else 1.0 - reset
    n = np.full(B, T) if lengths is None else lengths
    h = np.zeros((B, D)) if h0 is None else h0.copy()
    y, before = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        for t in range(n[b]):
            before[b, t] = r[b, t] * h[b]
            h[b] = a[b, t] * before[b, t] + u[b, t] * v[b, t]
            y[b, t] = h[b]
    out = {"y": y, "h_last": h}
    if dy is not None or dh_last is not None:
        g = np.zeros((B, D)) if dh_last is None else dh_last.copy()
        dv, df = np.zeros((B, T, D)), np.zeros((B, T, D))
        for b in range(B):
            for t in range(n[b] - 1, -1, -1):
                if dy is not None:
                    g[b] = g[b] + dy[b, t]
                dv[b, t] = u[b, t] * g[b]
                df[b, t] = g[b] * (a[b, t] * w[b, t] * before[b, t] + slope[b, t] * v[b, t])
                g[b] = r[b, t] * a[b, t] * g[b]
        out.update(dv=dv, df=df, dh0=g)
    return out


def make(B, T, D, dtype, seed=0, ragged=False, pad=0):
    """Tensors on the GPU (windows of wider rows when pad > 0) and their float64 copies."""
    import torch
    rng = np.random.default_rng(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def put(x):
        wide = torch.full((B, T, 2 * (D + pad)), float("nan"), dtype=dt, device="cuda")
        w = wide[:, :, pad:pad + D] if pad else torch.empty((B, T, D), dtype=dt, device="cuda")
        w.copy_(torch.from_numpy(x).to(dt))
        return w

    v = put(rng.standard_normal((B, T, D)))
    f = put(np.clip(rng.standard_normal((B, T, D)) * 2 + np.linspace(-1, 4, D), -6, 5))
    dy = put(rng.standard_normal((B, T, D)))
    h0, dh = (torch.from_numpy(rng.standard_normal((B, D))).float().cuda() for _ in range(2))
    reset = lengths = None
    if ragged:
        reset = torch.from_numpy((rng.random((B, T)) < 0.05).astype(np.uint8)).cuda()
        n = rng.integers(0, T + 1, B)
        n[0] = T
        n[-1] = 0 if B > 1 else T
        if B > 2:
            n[1] = 1
        lengths = torch.from_numpy(n.astype(np.int32)).cuda()
        for t in (v, f, dy):          # what stands in the padding must not matter
            for b in range(B):
                t[b, int(n[b]):] = float("nan")
    return v, f, dy, h0, dh, reset, lengths


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def run_both(B, T, D, dtype, gate, ragged, pad=0, seed=0, with_h0=True, stream=None):
    v, f, dy, h0, dh, reset, lengths = make(B, T, D, dtype, seed, ragged, pad)
    kw = dict(reset=reset, lengths=lengths, h0=h0 if with_h0 else None, input_gate=gate)
    y, h_last, st = mwb.gated_scan(v, f, keep_states=True, **kw)
    dv, df, dh0 = mwb.gated_scan_backward(v, f, dy, st, dh_last=dh, **kw)
    n = None if lengths is None else lengths.cpu().numpy()
    V, F, G = (np.nan_to_num(f64(t)) for t in (v, f, dy))
    ref = reference(V, F, gate, None if reset is None else reset.cpu().numpy().astype(float), n,
                    f64(h0) if with_h0 else None, G, f64(dh))
    got = {k: f64(t) for k, t in dict(y=y, h_last=h_last, dv=dv, df=df, dh0=dh0).items()}
    return got, ref, V


def check(got, ref, V, dtype):
    hmax = max(np.abs(ref["y"]).max(initial=0), np.abs(ref["h_last"]).max(), np.abs(V).max(initial=0), 1.0)
    gmax = max(np.abs(ref["dh0"]).max(), np.abs(ref["dv"]).max(initial=0), 1.0) * 2
    ulp = 2.0 ** -8 if dtype == "bf16" else 0.0
    for name, tol in (("y", 1e-5 * hmax), ("h_last", 1e-5 * hmax), ("dv", 1e-5 * gmax), ("dh0", 1e-5 * gmax),
                      ("df", 4e-5 * hmax * gmax)):
        r = ulp if name in ("y", "dv", "df") else 0.0
        assert got[name].shape == ref[name].shape
        if got[name].size:
            assert np.isfinite(got[name]).all(), name
            excess = np.abs(got[name] - ref[name]) - tol - r * np.abs(ref[name])
            assert excess.max() <= 0, (name, excess.max(), tol)


SIZES = [(1, 1, 1), (3, 1, 130), (2, 2, 64), (1, 15, 65), (2, 16, 128), (1, 17, 63), (3, 33, 96), (2, 255, 64),
         (1, 256, 72), (2, 257, 66), (1, 1000, 40), (2, 2049, 64), (5, 300, 520), (1, 5000, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("gate,ragged", [("complement", False), ("energy", True)])
def test_forward_and_backward_match_the_recurrence(size, dtype, gate, ragged):
    got, ref, V = run_both(*size, dtype, gate, ragged, seed=sum(size))
    check(got, ref, V, dtype)


# more sequences than SMs, a length of several rounds for one block of 128 (16 steps a thread) or 256; 66 columns
# leave rows off the 16-byte boundaries
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(230, 150, 64), (230, 300, 8), (230, 140, 66), (80, 520, 64), (40, 700, 40)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("gate,ragged", [("complement", True), ("energy", False)])
def test_many_sequences(size, dtype, gate, ragged):
    got, ref, V = run_both(*size, dtype, gate, ragged, seed=sum(size))
    check(got, ref, V, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 2, 8])
def test_windows_of_wider_rows(dtype, pad):
    got, ref, V = run_both(3, 70, 64, dtype, "complement", True, pad=pad, with_h0=False)
    check(got, ref, V, dtype)


def test_time_major_arrays():
    import torch
    v, f, dy, h0, dh, _, _ = make(3, 50, 64, "f32", 5)
    y, hl, st = mwb.gated_scan(v, f, h0=h0, keep_states=True)
    want = mwb.gated_scan_backward(v, f, dy, st, dh_last=dh)
    tm = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (v, f, dy)]
    y2, hl2, st2 = mwb.gated_scan(tm[0], tm[1], h0=h0, keep_states=True, y=torch.empty_like(tm[0]))
    got = mwb.gated_scan_backward(tm[0], tm[1], tm[2], st2, dh_last=dh)
    assert torch.equal(y, y2) and torch.equal(hl, hl2)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_steps_one_at_a_time_equal_the_whole_scan():
    # the serving form: the state lives in one buffer, updated in place
    import torch
    v, f, _, h0, _, _, _ = make(4, 40, 200, "bf16", 9)
    y, h_last = mwb.gated_scan(v, f, h0=h0, input_gate="energy")
    state = h0.clone()
    for t in range(40):
        yt, _ = mwb.gated_scan(v[:, t:t + 1], f[:, t:t + 1], h0=state, h_last=state, input_gate="energy")
        d = (yt[:, 0].float() - y[:, t].float()).abs()
        assert float((d - 2.0 ** -7 * y[:, t].float().abs()).max()) <= 1e-4
    assert float((state - h_last).abs().max()) <= 1e-5 * max(1.0, float(h_last.abs().max()))


@pytest.mark.parametrize("gate", ["complement", "energy"])
def test_saturated_gates(gate):
    # f = +-inf and +-100: the state is kept exactly, or replaced; nothing becomes NaN
    import torch
    f = torch.tensor([float("inf"), -float("inf"), 100.0, -100.0, 88.0, 0.0], device="cuda")
    B, T, D = 1, 20, f.numel()
    v = torch.randn(B, T, D, device="cuda")
    h0 = torch.randn(B, D, device="cuda")
    ff = f.expand(B, T, D).contiguous()
    y, hl, st = mwb.gated_scan(v, ff, h0=h0, keep_states=True, input_gate=gate)
    dv, df, dh0 = mwb.gated_scan_backward(v, ff, torch.ones_like(v), st, input_gate=gate)
    assert all(bool(torch.isfinite(t).all()) for t in (y, hl, dv, df, dh0))
    assert torch.equal(hl[:, [0, 2]], h0[:, [0, 2]])
    assert float((y[:, :, [1, 3]] - v[:, :, [1, 3]]).abs().max()) <= 1e-6


def test_nan_stays_in_its_channel_and_after_its_step():
    import torch
    v, f, _, h0, _, _, _ = make(2, 100, 70, "f32", 3)
    clean, _ = mwb.gated_scan(v, f, h0=h0)
    v[1, 37, 11] = float("nan")
    y, _ = mwb.gated_scan(v, f, h0=h0)
    bad = torch.isnan(y)
    assert bool(bad[1, 37:, 11].all()) and int(bad.sum()) == 63
    assert torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [12, 400, 3000])
def test_a_reset_keeps_out_what_came_before(T, dtype):
    # NaN and infinities before a reset do not reach the steps after it, nor cotangents the steps before
    import torch
    v, f, dy, h0, _, _, _ = make(1, T, 64, dtype, 12)
    at = T // 2
    reset = torch.zeros((1, T), dtype=torch.uint8, device="cuda")
    reset[0, at] = 1
    y0, h_last0, st0 = mwb.gated_scan(v, f, reset=reset, h0=h0, keep_states=True)
    g0 = mwb.gated_scan_backward(v, f, dy, st0, reset=reset)
    bad = v.clone()
    bad[0, at - 3, :32] = float("nan")
    bad[0, at - 2, 32:] = float("inf")
    y, h_last, st = mwb.gated_scan(bad, f, reset=reset, h0=h0, keep_states=True)
    assert torch.equal(y[:, at:], y0[:, at:]) and torch.equal(h_last, h_last0)
    g = mwb.gated_scan_backward(bad, f, dy, st, reset=reset)
    assert torch.equal(g[0][:, at:], g0[0][:, at:]) and torch.equal(g[1][:, at:], g0[1][:, at:])
    worse = dy.clone()
    worse[0, at + 2] = float("nan")
    g = mwb.gated_scan_backward(v, f, worse, st0, reset=reset)
    assert torch.equal(g[0][:, :at], g0[0][:, :at]) and torch.equal(g[1][:, :at], g0[1][:, :at])
    assert torch.equal(g[2], g0[2])


def test_no_cotangents_and_empty_sizes():
    import torch
    v, f, _, h0, dh, _, _ = make(2, 30, 64, "f32", 4)
    _, _, st = mwb.gated_scan(v, f, h0=h0, keep_states=True)
    dv, df, dh0 = mwb.gated_scan_backward(v, f, None, st)
    assert not dv.any() and not df.any() and not dh0.any()
    e = torch.empty((2, 0, 64), device="cuda")
    y, hl, st = mwb.gated_scan(e, e, h0=h0, keep_states=True)
    assert y.numel() == 0 and torch.equal(hl, h0)
    _, _, d0 = mwb.gated_scan_backward(e, e, None, st, dh_last=dh)
    assert torch.equal(d0, dh)
    y, hl = mwb.gated_scan(torch.empty((0, 5, 8), device="cuda"), torch.empty((0, 5, 8), device="cuda"))
    assert y.shape == (0, 5, 8) and hl.shape == (0, 8)


def test_repeated_calls_and_other_streams_give_the_same_bits():
    import torch
    v, f, dy, h0, dh, reset, lengths = make(2, 700, 192, "bf16", 6, ragged=True)
    kw = dict(reset=reset, lengths=lengths, h0=h0)

    def once(stream=None):
        y, hl, st = mwb.gated_scan(v, f, keep_states=True, stream=stream, **kw)
        return (y, hl, st) + mwb.gated_scan_backward(v, f, dy, st, dh_last=dh, reset=reset, lengths=lengths, stream=stream)

    a = once()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = once()
    c = once(s)                       # tensors of one stream, work on another
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b)) and all(torch.equal(p, q) for p, q in zip(a, c))


def test_work_on_another_stream_does_not_meet_freed_memory():
    # a tensor freed while the current stream still has to write it: its memory must not become the output of a
    # call on another stream, which does not wait for that write
    import torch
    v, f, dy, h0, dh, reset, lengths = make(2, 700, 192, "bf16", 6, ragged=True)
    kw = dict(reset=reset, lengths=lengths, h0=h0)
    y, hl, st = mwb.gated_scan(v, f, keep_states=True, **kw)
    dv, df, dh0 = mwb.gated_scan_backward(v, f, dy, st, dh_last=dh, reset=reset, lengths=lengths)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty_like(t) for t in (y, hl, st, dv, df)]
    torch.cuda._sleep(20_000_000)
    for t in old:
        t.fill_(7.0)
    del old, t
    y2, hl2, st2 = mwb.gated_scan(v, f, keep_states=True, stream=s, **kw)
    grads = mwb.gated_scan_backward(v, f, dy, st2, dh_last=dh, reset=reset, lengths=lengths, stream=s)
    torch.cuda.synchronize()
    for a, b in zip((y, hl, st, dv, df, dh0), (y2, hl2, st2) + grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("gate", ["complement", "energy"])
def test_gradients_match_differences(gate):
    # directional derivatives of sum(dy y) + sum(dh_last h_last), taken in 64 bits: central differences of
    # step 1e-4 are good to 1e-7 of the terms they sum; the fp32 gradient to 4e-5 of them
    v, f, dy, h0, dh, reset, lengths = make(3, 60, 48, "f32", 8, ragged=True)
    kw = dict(reset=reset, lengths=lengths, h0=h0, input_gate=gate)
    _, _, st = mwb.gated_scan(v, f, keep_states=True, **kw)
    grads = [f64(t) for t in mwb.gated_scan_backward(v, f, dy, st, dh_last=dh, **kw)]
    V, F, G, H, L = (np.nan_to_num(f64(t)) for t in (v, f, dy, h0, dh))
    R, n = reset.cpu().numpy().astype(float), lengths.cpu().numpy()

    def loss(V, F, H):
        o = reference(V, F, gate, R, n, H)
        return float((o["y"] * G).sum() + (o["h_last"] * L).sum())

    rng = np.random.default_rng(1)
    for i in range(3):
        d = rng.standard_normal([V, F, H][i].shape)
        args = [[V, F, H], [V, F, H]]
        args[0][i] = args[0][i] + 1e-4 * d
        args[1][i] = args[1][i] - 1e-4 * d
        num = (loss(*args[0]) - loss(*args[1])) / 2e-4
        ana = float((grads[i] * d).sum())
        assert abs(num - ana) <= 4e-5 * float(np.abs(grads[i] * d).sum()) + 1e-6, (i, num, ana)


def test_refusals():
    import torch
    v = torch.zeros((2, 8, 16), device="cuda")
    for bad in (lambda: mwb.gated_scan(v.double(), v.double()), lambda: mwb.gated_scan(v, v.bfloat16()),
                lambda: mwb.gated_scan(v, v[:, :4]), lambda: mwb.gated_scan(v[:, :, ::2], v[:, :, ::2]),
                lambda: mwb.gated_scan(v[0], v[0]), lambda: mwb.gated_scan(v, v, input_gate="other"),
                lambda: mwb.gated_scan(v, v, h0=torch.zeros((2, 8), device="cuda")),
                lambda: mwb.gated_scan(v, v, lengths=torch.zeros(2, device="cuda")),
                lambda: mwb.gated_scan(v, v, reset=torch.zeros((2, 7), dtype=torch.uint8, device="cuda")),
                lambda: mwb.gated_scan(v, v, h0=torch.zeros((2, 16))), lambda: mwb.gated_scan(v.cpu(), v.cpu()),
                lambda: mwb.gated_scan_backward(v, v, v, None)):
        with pytest.raises((TypeError, ValueError, mwb.MwError)):
            bad()
