"""What the sequence-block bindings hand to the library, seen without a GPU: CPU tensors stand in for CUDA ones,
and a recorder stands in for the library."""
import contextlib

import pytest
import torch

from paper_2402_14212_b200 import binding as mwb


class OnDevice(torch.Tensor):
    """A CPU tensor that calls itself a CUDA one."""
    is_cuda = True


def on_device(t):
    return t.as_subclass(OnDevice)


class Recorder:
    """Takes the place of the loaded library: every call succeeds and is remembered."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return mwb.MW_OK
        return call


@pytest.fixture
def recorder(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(mwb, "lib", lambda: rec)
    monkeypatch.setattr(mwb, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(mwb, "_passed", {})
    monkeypatch.setattr(mwb, "_current_device", lambda: torch.device("cpu").index)
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    # bytes from the address of a tensor that was asked for it to the end of its memory
    rec.room = {}
    plain = torch.Tensor.data_ptr

    def data_ptr(t):
        p = plain(t)
        if t.numel():
            s = t.untyped_storage()
            rec.room[p] = s.data_ptr() + s.nbytes() - p
        return p

    monkeypatch.setattr(torch.Tensor, "data_ptr", data_ptr)
    return rec


class OnSecond(OnDevice):
    device = torch.device("cuda", 1)


@pytest.fixture
def devices(monkeypatch, recorder):
    """The device that is current, as the bindings see and set it; every recorded call notes it."""
    current = [0]

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    monkeypatch.setattr(mwb, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    recorder.at = []
    plain = Recorder.__getattr__

    def noted(self, name):
        call = plain(self, name)

        def both(*args):
            recorder.at.append((name, current[0]))
            return call(*args)
        return both

    monkeypatch.setattr(Recorder, "__getattr__", noted)
    return current


class Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)
        self.cuda_stream = 64 + index


def scan_reach(d, which):
    """Bytes from a tensor's first element to the end of the last that the library touches."""
    b, t = getattr(d, which + "_batch"), getattr(d, which + "_time")
    if b == 0 and t == 0:              # the library's sign for dense
        t = d.channels
        b = t * d.length
    return ((d.batch - 1) * b + (d.length - 1) * t + d.channels) * (4 if d.dtype == 1 else 2)


def norm_reach(d, which):
    ld = getattr(d, "ld_" + which) or d.cols
    return ((d.rows - 1) * ld + d.cols) * (4 if d.dtype == 1 else 2)


B, T, D, R = 3, 40, 16, 24
EXPANDED = {"all": lambda: torch.randn(1, 1, D).expand(B, T, D), "time": lambda: torch.randn(B, 1, D).expand(B, T, D),
            "batch": lambda: torch.randn(1, T, D).expand(B, T, D), "scalar": lambda: torch.randn(()).expand(B, T, D)}


@pytest.mark.parametrize("how", sorted(EXPANDED))
@pytest.mark.parametrize("which", ["v", "f", "dy"])
def test_scan_reads_expanded_inputs_inside_their_memory(recorder, which, how):
    dense = {k: on_device(torch.randn(B, T, D)) for k in ("v", "f", "dy")}
    dense[which] = on_device(EXPANDED[how]())
    want = dense[which].clone()
    v, f, dy = dense["v"], dense["f"], dense["dy"]
    y, _, states = mwb.gated_scan(v, f, keep_states=True)
    mwb.gated_scan_backward(v, f, dy, states)
    for name, args in recorder.calls:
        d = args[0]
        places = {"v": args[1], "f": args[2]}
        if name.endswith("backward"):
            places["y"], places["dv"], places["df"] = args[6], args[8], args[9]
        else:
            places["y"] = args[6]
        for field, at in places.items():
            assert scan_reach(d, field) <= recorder.room[at], (name, field)
    assert y.shape == (B, T, D) and torch.equal(dense[which], want)


def test_scan_reads_the_cotangent_of_a_sum(recorder):
    # the cotangent that y.sum() hands back, of one channel too
    for shape in ((B, T, D), (B, T, 1)):
        recorder.calls.clear()
        v = on_device(torch.randn(shape))
        dy = on_device(torch.ones(()).expand(shape))
        _, _, states = mwb.gated_scan(v, v, keep_states=True)
        mwb.gated_scan_backward(v, v, dy, states)
        name, args = recorder.calls[-1]
        assert name == "mw_gated_scan_backward" and scan_reach(args[0], "y") <= recorder.room[args[6]]


def test_scan_refuses_outputs_that_repeat_elements(recorder):
    v = on_device(torch.randn(B, T, D))
    _, _, states = mwb.gated_scan(v, v, keep_states=True)
    n = len(recorder.calls)
    for how in EXPANDED.values():
        out = on_device(how())
        with pytest.raises(ValueError):
            mwb.gated_scan(v, v, y=out)
        with pytest.raises(ValueError):
            mwb.gated_scan_backward(v, v, v, states, dv=out)
        with pytest.raises(ValueError):
            mwb.gated_scan_backward(v, v, v, states, df=out)
    assert len(recorder.calls) == n


@pytest.mark.parametrize("which", ["x", "b", "z"])
def test_norm_reads_expanded_inputs_inside_their_memory(recorder, which):
    t = {k: on_device(torch.randn(R, D)) for k in ("x", "b", "z")}
    t[which] = on_device(torch.randn(1, D).expand(R, D))
    w = on_device(torch.ones(D))
    _, _, rms = mwb.residual_norm(t["x"], t["b"], z=t["z"], w_post=w, w_pre=w, keep_rms=True)
    g = on_device(torch.randn(R, D))
    mwb.residual_norm_backward(t["x"], t["b"], rms, z=t["z"], w_post=w, w_pre=w, dx_out=g, dn=g)
    checked = 0
    for name, args in recorder.calls:
        if name.endswith(("forward", "backward")):
            for field, at in zip("xbz", args[1:4]):
                assert norm_reach(args[0], field) <= recorder.room[at], (name, field)
                checked += 1
    assert checked == 6


def second(*shape, dtype=torch.float32):
    return torch.randn(*shape).to(dtype).as_subclass(OnSecond)


def orth_lists(count=2):
    return [[second(8, 8) for _ in range(count)] for _ in range(3)]


def test_calls_run_with_the_tensors_device_current(devices, recorder):
    v, h = second(B, T, D), second(B, D)
    st = second(B, -(-T // mwb.SCAN_STATE_EVERY), D)
    x, w = second(R, D), second(D)
    plan = mwb.Orth(8, 8, 2, "f32")
    ws = torch.empty(1 << 16, dtype=torch.uint8).as_subclass(OnSecond)
    W, G, M = orth_lists()
    recorder.at.clear()
    for _ in range(2):                 # the first call of a layout and a remembered one
        mwb.gated_scan(v, v, h0=h, y=second(B, T, D), h_last=h)
        mwb.gated_scan_backward(v, v, v, st, dh_last=h, dv=second(B, T, D), df=second(B, T, D))
        mwb.residual_norm(x, x, w_pre=w, x_out=second(R, D), n=second(R, D))
        plan.step(W, G, M, ws, lr=0.1)
        plan.project(W, ws, out=M)
        plan.status(ws)
    assert len(recorder.at) == 12 and all(at == 1 for _, at in recorder.at), recorder.at
    assert devices[0] == 0


def test_backward_of_the_norm_runs_with_the_tensors_device_current(devices, recorder, monkeypatch):
    # (the call allocates its scratch: on the CPU here)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    x, w, rms = second(R, D), second(D), second(2, R)
    mwb.residual_norm_backward(x, x, rms, w_pre=w, dx_out=x, dn=x)
    assert recorder.at == [("mw_residual_norm_scratch_bytes", 1), ("mw_residual_norm_backward", 1)] and devices[0] == 0


def test_orth_refuses_a_stream_of_another_device(devices, recorder):
    plan = mwb.Orth(8, 8, 2, "f32")
    ws = torch.empty(1 << 16, dtype=torch.uint8).as_subclass(OnSecond)
    W, G, M = orth_lists()
    n = len(recorder.calls)
    for bad in (lambda: plan.step(W, G, M, ws, lr=0.1, stream=Stream(0)), lambda: plan.project(W, ws, out=M, stream=Stream(0)),
                lambda: plan.status(ws, stream=Stream(0))):
        with pytest.raises(ValueError):
            bad()
    assert len(recorder.calls) == n


@pytest.fixture
def streams(monkeypatch, devices):
    """Which tensors (by address) were marked as used on which stream, in the order of the calls."""
    marks = []
    here = Stream(1)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw).as_subclass(OnSecond))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: here)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: marks.append((t.data_ptr(), s)))
    return marks


def test_everything_a_call_on_another_stream_touches_is_marked_for_it(streams, recorder):
    # memory of a tensor that the caller drops after the call is not given out before the work there is done
    s = Stream(1)

    def check(tensors, call):
        streams.clear()
        call()
        for i, t in enumerate(tensors):
            assert (t.data_ptr(), s) in streams, i

    v, f, dy, y, dv, df = (second(B, T, D) for _ in range(6))
    h0, hl, dh = (second(B, D) for _ in range(3))
    reset = torch.zeros((B, T), dtype=torch.uint8).as_subclass(OnSecond)
    lengths = torch.full((B,), T, dtype=torch.int32).as_subclass(OnSecond)
    st = second(B, -(-T // mwb.SCAN_STATE_EVERY), D)
    check([v, f, reset, lengths, h0, y, hl],
          lambda: mwb.gated_scan(v, f, reset=reset, lengths=lengths, h0=h0, y=y, h_last=hl, stream=s))
    check([v, f, dy, st, reset, lengths, dh, dv, df],
          lambda: mwb.gated_scan_backward(v, f, dy, st, reset=reset, lengths=lengths, dh_last=dh, dv=dv, df=df, stream=s))
    x, b, z, xo, n, dxo, dn = (second(R, D) for _ in range(7))
    wp, sc, wn = (second(D) for _ in range(3))
    rms = second(2, R)
    kw = dict(z=z, w_post=wp, scale=sc, w_pre=wn, stream=s)
    check([x, b, z, wp, sc, wn, xo, n], lambda: mwb.residual_norm(x, b, x_out=xo, n=n, **kw))
    check([x, b, z, wp, sc, wn, rms, dxo, dn], lambda: mwb.residual_norm_backward(x, b, rms, dx_out=dxo, dn=dn, **kw))
    plan = mwb.Orth(8, 8, 2, "f32")
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    W, G, M = orth_lists()
    W2, M2, _ = orth_lists()
    check(W + G + M + W2 + M2 + [ws],
          lambda: plan.step(W, G, M, ws, lr=0.1, params_out=W2, momentum_out=M2, stream=s))
    check(W + W2 + [ws], lambda: plan.project(W, ws, out=W2, stream=s))
    check(W + [ws], lambda: plan.project(W, ws, stream=s))
