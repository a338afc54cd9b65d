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
