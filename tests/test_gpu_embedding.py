"""mw_embedding_* against the formulas in 64 bits.

Tolerances (u = 2^-24, ur = half a step of the result's type).  A looked-up value is one product and one rounding:
(u + ur) of it.  A gradient sums k values in float, in any order k u of the sum of their absolute values, times scale
(u more) and rounded once (twice where it is added to what is there): ur of the values."""
import numpy as np
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.bfloat16]


def make(n, V, D, dtype, seed=0, common=0.0, outside=True, ids=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    if common:
        t = torch.where(torch.rand(n, generator=g, device="cuda") < common, V // 2, t)
    if outside and n > 4:
        t[n // 3], t[n // 2] = -1, V
    if outside and n > 6 and ids == torch.int64:
        t[n // 5] = 1 << 40
    table = torch.randn(V, D, generator=g, device="cuda").to(dtype)
    dout = torch.randn(n, D, generator=g, device="cuda").to(dtype)
    return t.to(ids), table, dout


def expected_rows(t, table, scale):
    V = table.shape[0]
    ok = (t >= 0) & (t < V)
    rows = table.double()[torch.where(ok, t.long(), 0)] * scale
    return torch.where(ok[..., None], rows, 0.0)


def expected_gradient(t, dout, V, scale):
    """(sums, sums of absolute values, counts)"""
    ok = (t >= 0) & (t < V)
    at, d = t[ok].long(), dout[ok].double() * scale
    s = torch.zeros(V, dout.shape[-1], dtype=torch.float64, device=dout.device).index_add_(0, at, d)
    a = torch.zeros_like(s).index_add_(0, at, d.abs())
    k = torch.zeros(V, dtype=torch.float64, device=dout.device).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    return s, a, k


def check_gradient(got, t, dout, V, scale, before=None):
    s, a, k = expected_gradient(t, dout, V, scale)
    bound = (k[:, None] + 1) * U * a
    if before is not None:
        s, bound = s + before.double(), bound + U * (a + before.double().abs())
    bound += HALF[got.dtype] * s.abs() * (1 + 2.0 ** -7)
    assert bool(((got.double() - s).abs() <= bound).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 300, 64), (7, 5, 3), (33, 1000, 515), (257, 70000, 128), (1000, 17, 2048),
                                   (3, 9, 20000), (4099, 255, 8), (4099, 256, 24)])
def test_lookup_and_gradient(n, V, D, dtype):
    t, table, dout = make(n, V, D, dtype)
    out = mwb.embedding(t, table, scale=1.7)
    want = expected_rows(t, table, 1.7)
    assert bool(((out.double() - want).abs() <= (U + HALF[dtype]) * want.abs()).all())
    for kind in TYPES:
        got = mwb.embedding_backward(t, dout, V, scale=1.7, grad_dtype=kind)
        assert got.dtype == kind and got.shape == (V, D)
        check_gradient(got, t, dout, V, float(np.float32(1.7)))


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,common", [(31, 1.0), (32, 1.0), (33, 1.0), (64, 0.9), (3000, 0.5), (20000, 1.0), (70001, 0.3)])
def test_runs_of_any_length(n, common, ids):
    t, _, dout = make(n, 37, 72, torch.bfloat16, seed=n, common=common, ids=ids)
    got = mwb.embedding_backward(t, dout, 37, grad_dtype=torch.float32)
    check_gradient(got, t, dout, 37, 1.0)
    assert torch.equal(got, mwb.embedding_backward(t, dout, 37, grad_dtype=torch.float32))


@pytest.mark.parametrize("bits", [1, 7, 8, 9, 15, 16, 17, 20])
def test_vocabularies_of_any_size(bits):
    V = (1 << bits) - (bits > 16)
    t, _, dout = make(5000, V, 4, torch.float32, seed=bits)
    check_gradient(mwb.embedding_backward(t, dout, V), t, dout, V, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_accumulating_adds_to_the_rows_that_tokens_name(dtype):
    t, table, dout = make(600, 50, 96, dtype, common=0.4)
    t[t == 3] = 4
    before = torch.randn(50, 96, device="cuda").to(dtype)
    before[3] = float("nan")                       # named by no token: left alone
    got = before.clone()
    assert mwb.embedding_backward(t, dout, 50, scale=0.5, dtable=got, accumulate=True) is got
    assert bool(torch.isnan(got[3]).all())
    rest = torch.arange(50, device="cuda") != 3
    clean = torch.where(rest[:, None], before, 0.0)
    check_gradient(torch.where(rest[:, None], got, 0.0), t, dout, 50, 0.5, before=clean)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_windows_of_wider_rows(dtype, shift):
    t, table, dout = make(40, 30, 64, dtype)
    wide = torch.full((30, 200), float("nan"), device="cuda").to(dtype)
    wide[:, shift:shift + 64] = table
    assert torch.equal(mwb.embedding(t, wide[:, shift:shift + 64]), mwb.embedding(t, table))
    wd = torch.full((40, 200), float("nan"), device="cuda").to(dtype)
    wd[:, shift:shift + 64] = dout
    want = mwb.embedding_backward(t, dout, 30)
    assert torch.equal(mwb.embedding_backward(t, wd[:, shift:shift + 64], 30), want)
    out = torch.full((30, 200), 7.0, device="cuda").to(dtype)
    mwb.embedding_backward(t, dout, 30, dtable=out[:, shift:shift + 64])
    assert torch.equal(out[:, shift:shift + 64], want)
    assert bool((out[:, :shift] == 7).all() and (out[:, shift + 64:] == 7).all())      # between the rows


def test_shapes_of_tokens_and_expanded_operands():
    t, table, dout = make(60, 30, 64, torch.float32)
    want = mwb.embedding(t, table)
    assert torch.equal(mwb.embedding(t.view(3, 4, 5), table), want.view(3, 4, 5, 64))
    assert torch.equal(mwb.embedding(t.view(10, 6).T, table), want.view(10, 6, 64).transpose(0, 1))
    d3 = dout.view(10, 6, 64)
    grad = mwb.embedding_backward(t, dout, 30)
    assert torch.equal(mwb.embedding_backward(t.view(10, 6), d3, 30), grad)
    one = torch.randn(1, 64, device="cuda")
    assert torch.equal(mwb.embedding(t, one.expand(30, 64)), mwb.embedding(t, one.expand(30, 64).contiguous()))
    assert torch.equal(mwb.embedding_backward(t, one.expand(60, 64), 30),
                       mwb.embedding_backward(t, one.expand(60, 64).contiguous(), 30))


def test_no_tokens_and_values_that_are_not_finite():
    table = torch.randn(6, 5, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert mwb.embedding(none, table).shape == (0, 5)
    assert bool((mwb.embedding_backward(none, torch.empty(0, 5, device="cuda"), 6) == 0).all())
    kept = torch.ones(6, 5, device="cuda")
    mwb.embedding_backward(none, torch.empty(0, 5, device="cuda"), 6, dtable=kept, accumulate=True)
    assert bool((kept == 1).all())
    t = torch.tensor([0, 1, 1, 2, -1], device="cuda")
    dout = torch.ones(5, 5, device="cuda")
    dout[1, 2], dout[3, 0], dout[4] = float("inf"), float("nan"), float("nan")
    got = mwb.embedding_backward(t, dout, 6)
    assert bool(torch.isinf(got[1, 2])) and bool(torch.isnan(got[2, 0]))
    got[1, 2], got[2, 0] = 2, 1
    want = torch.tensor([1.0, 2, 1, 0, 0, 0], device="cuda")[:, None].expand(6, 5)
    assert torch.equal(got, want)
    table[3] = float("nan")                        # a row that no token names
    assert not bool(torch.isnan(mwb.embedding(t, table)).any())


def test_gradient_against_differences():
    """Linear in the table: the difference of <out, dout> along a direction is <dtable, direction> up to rounding:
    600 x 32 terms of size 1, each 4 u off in either sum."""
    t, table, dout = make(600, 50, 32, torch.float32, common=0.2)
    way = torch.randn(50, 32, device="cuda")
    f = lambda e: (mwb.embedding(t, e, scale=3.0).double() * dout.double()).sum()
    rise = (f(table + way) - f(table - way)) / 2
    along = (mwb.embedding_backward(t, dout, 50, scale=3.0).double() * way.double()).sum()
    assert abs(float(rise - along)) <= 600 * 32 * 3.0 * 8 * 4 * U


@pytest.mark.parametrize("n", [500, 70001])
def test_another_stream_and_a_captured_call(n):
    t, table, dout = make(n, 40, 128, torch.bfloat16, common=0.3)
    want, grad = mwb.embedding(t, table), mwb.embedding_backward(t, dout, 40)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a, b = mwb.embedding(t, table, stream=side), mwb.embedding_backward(t, dout, 40, stream=side)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, d = mwb.embedding(t, table), mwb.embedding_backward(t, dout, 40)
    for seed in (5, 6):
        t2, table2, dout2 = make(n, 40, 128, torch.bfloat16, seed=seed)
        t.copy_(t2), table.copy_(table2), dout.copy_(dout2)
        graph.replay()
        assert torch.equal(c, mwb.embedding(t2, table2)) and torch.equal(d, mwb.embedding_backward(t2, dout2, 40))
