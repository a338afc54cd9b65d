"""mw_clip_gradients against the formula in 64 bits.

Tolerances (u = 2^-24, ur = half a step of the type).  The norm is summed in 64 bits and rounded once: 2 u.  A scaled value
is a factor (rounded once, u) times the value (u), rounded to its type: 4 u + ur of it."""
import math

import pytest
import torch

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def make(shapes, dtypes, size=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(s, generator=g, device="cuda") * size).to(dtypes[i % len(dtypes)]) for i, s in enumerate(shapes)]


def norm_of(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def check(before, after, norm, most):
    want = norm_of(before)
    assert abs(float(norm) - want) <= 2 * U * want
    k = min(1.0, most / want) if want > 0 else 1.0
    for b, a in zip(before, after):
        w = b.double() * k
        assert bool(((a.double() - w).abs() <= (4 * U + HALF[a.dtype]) * w.abs()).all())


SHAPES = {"one": [(1,)], "odd": [(3,), (1537, 67), (677,), (8191,), (8192,), (8193,)], "none": [(0,), (5, 0)],
          "mixed": [(0,), (64, 64), (0, 3), (100001,)], "large": [(3000, 4001)], "long": [(2500000,), (7,)]}


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("which", sorted(SHAPES))
@pytest.mark.parametrize("most", [0.5, 1e9, float("inf")])
def test_norm_and_scaling(which, dtypes, most):
    grads = make(SHAPES[which], dtypes)
    out = [torch.full_like(t, 7.0) for t in grads]
    kept = [t.clone() for t in grads]
    norm = mwb.clip_gradients(grads, most, out=out)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    check(kept, out, norm, most)
    assert torch.equal(norm, mwb.clip_gradients(grads, most))         # in place
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
    if most >= 1e9:
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))


@pytest.mark.parametrize("count", [255, 256, 257, 600])
def test_many_tensors(count):
    grads = make([(1 + 37 * i % 211,) for i in range(count)], (torch.float32, torch.bfloat16))
    kept = [t.clone() for t in grads]
    check(kept, grads, mwb.clip_gradients(grads, 1.0), 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("at", [1, 2, 3, 4, 5])
def test_windows_off_the_boundaries(dtype, at):
    base, to = torch.randn(70000, device="cuda").to(dtype), torch.zeros(70000, device="cuda", dtype=dtype)
    g, o = base[at:at + 60001], to[2 * at:2 * at + 60001]
    kept = g.clone()
    check([kept], [o], mwb.clip_gradients([g], 2.0, out=[o]), 2.0)
    assert bool((to[:2 * at] == 0).all() and (to[2 * at + 60001:] == 0).all())
    check([kept], [g], mwb.clip_gradients([g], 2.0), 2.0)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e19, 1e30])
def test_squares_beyond_the_range_of_32_bits(size):
    grads = make([(1000,), (333, 3)], (torch.float32, torch.bfloat16), size)
    kept = [t.clone() for t in grads]
    most = norm_of(kept) / 3
    check(kept, grads, mwb.clip_gradients(grads, most), most)


def test_zero_and_values_that_are_not_finite():
    zero = [torch.zeros(100, device="cuda")]
    assert float(mwb.clip_gradients(zero, 1.0)) == 0.0 and bool((zero[0] == 0).all())
    for bad in (float("inf"), float("nan")):
        grads = make([(100,), (5000,)], (torch.float32, torch.bfloat16))
        grads[1][3000] = bad
        kept = [t.clone() for t in grads]
        out = [torch.zeros_like(t) for t in grads]
        norm = float(mwb.clip_gradients(grads, 1.0, out=out))
        assert math.isinf(norm) if math.isinf(bad) else math.isnan(norm)
        for k, g, o in zip(kept, grads, out):
            assert torch.equal(k.nan_to_num(), g.nan_to_num()) and torch.equal(k.nan_to_num(), o.nan_to_num())


def test_another_stream_and_a_captured_call():
    grads = make([(300, 70), (11,)], (torch.float32, torch.bfloat16))
    out, want = [torch.empty_like(t) for t in grads], [torch.empty_like(t) for t in grads]
    norm = mwb.clip_gradients(grads, 1.0, out=want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other = mwb.clip_gradients(grads, 1.0, out=out, stream=side)
    side.synchronize()
    assert torch.equal(norm, other) and all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = mwb.clip_gradients(grads, 1.0, out=out)
    for seed in (3, 4):
        new = make([(300, 70), (11,)], (torch.float32, torch.bfloat16), seed=seed)
        for a, b in zip(grads, new):
            a.copy_(b)
        graph.replay()
        assert torch.equal(held, mwb.clip_gradients(new, 1.0, out=want)) and all(torch.equal(a, b) for a, b in zip(out, want))
