"""Host-side checks of the sequence-block operators and the orthogonalised update: bad descriptions are
refused before any GPU work, sizes come out as documented (runs without a GPU)."""
import ctypes as C

import pytest

from paper_2402_14212_b200 import binding as mwb

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def scan_desc(**kw):
    d = dict(batch=2, length=40, channels=64, dtype=1, input_gate=0, reserved=0)
    d.update(kw)
    return mwb.GatedScanDesc(**d)


def test_scan_descriptions():
    L = mwb.lib()
    n = C.c_size_t()
    assert L.mw_gated_scan_states_bytes(scan_desc(), C.byref(n)) == 0 and n.value == 2 * 3 * 64 * 4
    for kw, code in ((dict(batch=-1), INVALID), (dict(length=-1), INVALID), (dict(channels=0), INVALID),
                     (dict(dtype=0), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(input_gate=2), INVALID),
                     (dict(reserved=1), INVALID)):
        assert L.mw_gated_scan_states_bytes(scan_desc(**kw), C.byref(n)) == code, kw
        assert L.mw_gated_scan_forward(scan_desc(**kw), 256, 256, None, None, None, 256, None, None, None) == code
    fwd = lambda d, v=256, f=256, y=256: L.mw_gated_scan_forward(d, v, f, None, None, None, y, None, None, None)
    assert fwd(scan_desc(), v=None) == INVALID and fwd(scan_desc(), y=None) == INVALID
    assert fwd(scan_desc(v_batch=4096, v_time=63)) == INVALID          # steps overlap
    assert fwd(scan_desc(f_batch=63, f_time=64)) == INVALID            # sequences overlap
    assert fwd(scan_desc(batch=0), v=None, f=None, y=None) == 0        # nothing to do
    assert L.mw_gated_scan_backward(scan_desc(), 256, 256, None, None, None, 256, None, 256, 256, None, None) == INVALID
    assert L.mw_gated_scan_states_bytes(None, C.byref(n)) == INVALID


def test_norm_descriptions():
    L = mwb.lib()
    n = C.c_size_t()

    def desc(**kw):
        d = dict(rows=4, cols=64, dtype=2, eps=1e-6, ld_x=0, ld_b=0, ld_z=0)
        d.update(kw)
        return mwb.ResidualNormDesc(**d)

    def fwd(d, x=256, b=256, z=None, wp=None, sc=None, wn=None, xo=512, nn=None):
        return L.mw_residual_norm_forward(d, x, b, z, wp, sc, wn, xo, nn, None, None)

    for kw, code in ((dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=32769), UNSUPPORTED),
                     (dict(dtype=0), UNSUPPORTED), (dict(dtype=7), INVALID), (dict(eps=0.0), INVALID),
                     (dict(eps=float("nan")), INVALID), (dict(ld_b=63), INVALID)):
        assert fwd(desc(**kw)) == code, kw
    assert fwd(desc(), x=None) == INVALID
    assert fwd(desc(), b=None, z=256) == INVALID and fwd(desc(), b=None, wp=256) == INVALID
    assert fwd(desc(), wn=256) == INVALID and fwd(desc(), nn=256) == INVALID and fwd(desc(), xo=None) == INVALID
    assert fwd(desc(ld_x=128), x=256, xo=256) == INVALID               # in place needs dense rows
    assert fwd(desc(rows=0), x=None, b=None, xo=None) == 0
    assert L.mw_residual_norm_scratch_bytes(desc(), C.byref(n)) == 0 and n.value >= 3 * 64 * 4

    def bwd(rms=256, dn=None, dw=None, scratch=None, size=0, db=256):
        return L.mw_residual_norm_backward(desc(), 256, 256, None, dw, None, None, rms, 256, dn, 256, db, None, dw,
                                           None, None, scratch, size, None)

    assert bwd(rms=None) == INVALID and bwd(dn=256) == INVALID
    assert bwd(dw=256) == WORKSPACE and bwd(dw=256, scratch=257, size=1 << 20) == WORKSPACE
    assert bwd(dw=256, scratch=256, size=16) == WORKSPACE


def test_orth_descriptions():
    L = mwb.lib()
    plan = mwb.Orth(48, 80, 3, "f32")
    n = plan.workspace_bytes()
    assert n > 0
    arr = (C.c_void_p * 3)(256, 256, 256)
    hole = (C.c_void_p * 3)(256, None, 256)
    step = lambda p=arr, ws=256, size=n, lr=0.1: L.mw_orth_step(plan._h, p, arr, arr, arr, arr, lr, 0.9, 0.0, 1.0, ws,
                                                                size, None)
    assert step(p=hole) == INVALID and step(lr=float("nan")) == INVALID
    assert step(ws=None) == WORKSPACE and step(ws=128) == WORKSPACE and step(size=n - 1) == WORKSPACE
    assert L.mw_orth_project(plan._h, hole, arr, 256, n, None) == INVALID
    assert L.mw_orth_project(None, arr, arr, 256, n, None) == INVALID
    for kw in (dict(rows=0, cols=4), dict(rows=4, cols=4, count=0), dict(rows=4, cols=4, prec="f64"),
               dict(rows=4, cols=4, steps=17), dict(rows=4, cols=4, steps=-1), dict(rows=4, cols=4, terms=3),
               dict(rows=4, cols=4, coef=(float("inf"), 0.0, 0.0))):
        with pytest.raises(mwb.MwError):
            mwb.Orth(**kw)
    for _ in range(100):                       # host objects only
        p = mwb.Orth(100, 64, 2, "bf16_f32acc")
        p.close()
        p.close()
