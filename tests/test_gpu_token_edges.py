"""The lookup and the vocabulary's loss where their kernels change course: operands of unusual sizes, few rows taken
as they lie, waves of tiles with a rest, pieces with gradients off the copy engine's boundaries, places beyond 2^31, two
calls at once.  Formulas and tolerances are those of test_gpu_token_loss.py and test_gpu_embedding.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_embedding import check_gradient
from test_gpu_token_loss import ALL, BF16, F32, check, make, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", ["as it is", "outlier", "zeros", "small and large rows", "large and small rows"])
def test_operands_of_unusual_sizes(how, dtype):
    """Operands are written for numbers of the usual size, and again where their largest lies elsewhere."""
    V, D, N = (4300 if dtype == F32 else 8600), 2048, 200
    h, W, t = make(N, V, D, dtype, lean=0.0)
    sampled = torch.arange(V, device="cuda") % 16 == 0
    if how == "outlier":
        W[1, 5] = 3.0e4
        h[:, 5] = 0
    elif how == "zeros":
        W[sampled] = 0
    elif how == "small and large rows":
        W[sampled] *= 2.0 ** -12
    elif how == "large and small rows":
        W[~sampled] *= 2.0 ** -12
    check(mwb.token_loss_gradient(h, W, t), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [-30, -12, -9, -8, -3, 4, 6, 7, 8, 9, 10, 14, 30])
def test_operands_of_every_size(size, dtype):
    h, W, t = make(150, 400, 192, dtype)
    h, W = h * 2.0 ** size, W * 2.0 ** -size
    check(mwb.token_loss_gradient(h, W, t), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lean", [0.0, 15.0, 40.0, 200.0])
def test_losses_of_sure_rows(lean, dtype):
    """The others' terms against the target's: a loss near zero keeps its digits.  Relative to e = exp(loss) - 1 it is
    off by what the differences of logits are, each ((D / 16 + 8) 2^-23 and 2^-21) of S."""
    h, W, t = make(300, 700, 128, dtype, lean=lean)
    r = mwb.token_loss(h, W, t)
    z, S = h.double() @ W.double().T, h.double().abs() @ W.double().abs().T
    ez = 2 * ((128 / 16 + 8) * 2.0 ** -23 + 2.0 ** -21) * S.amax(1) + 2.0 ** -18
    odds = torch.exp(z - z.gather(1, t[:, None]))
    odds.scatter_(1, t[:, None], 0.0)
    want = torch.log1p(odds.sum(1))
    assert bool(((r.loss.double() - want).abs() <= torch.expm1(ez) * -torch.expm1(-want) + 2.0 ** -22 * want + 1e-36).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V,D,piece", [(2100, 200, 100, 0), (2100, 300, 64, 1024), (5000, 60, 520, 0), (1500, 2500, 128, 512), (1024, 256, 256, 0)])
def test_few_tiles_of_the_weight_gradient(N, V, D, piece, dtype):
    h, W, t = make(N, V, D, dtype, left_out=0.3)
    for kind in (F32, BF16):
        check(mwb.token_loss_gradient(h, W, t, piece_rows=piece, grad_dtype=kind), reference(h, W, t), ALL)
    t[:] = -1
    r = mwb.token_loss_gradient(h, W, t, piece_rows=piece)
    assert bool((r.dweight == 0).all() and (r.dh == 0).all() and (r.loss == 0).all()) and float(r.total) == 0


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 33, 64, 65, 128, 129, 200, 256, 257])
def test_few_rows_taken_as_they_lie(N, ids):
    h, W, t = make(N, 3001, 264, BF16, seed=N, left_out=0.3)
    w = torch.rand(N, device="cuda")
    w[::5] = 0
    h[::5] = float("nan")
    for weight in (None, w):
        on = h.clone() if weight is not None else torch.where(h.isnan(), 0.5, h.float()).to(BF16)
        check(mwb.token_loss(on, W, t.to(ids), row_weight=weight), reference(on, W, t, weight=weight), ("loss", "total"))
    # rows off the copy engine's boundaries
    wide = torch.zeros(N, 300, device="cuda", dtype=BF16)
    off = wide[:, 1:265]
    off.copy_(on)
    check(mwb.token_loss(off, W, t.to(ids), row_weight=w), reference(on, W, t, weight=w), ("loss", "total"))


@pytest.mark.parametrize("V", [1, 31, 63, 64, 65, 4736, 4737, 18944, 18945, 20000])
def test_vocabularies_of_few_rows(V):
    h, W, t = make(20, V, 72, BF16, seed=V)
    check(mwb.token_loss(h, W, t), reference(h, W, t), ("loss", "total"))


def test_a_weight_that_starts_off_its_boundary():
    h, W, t = make(300, 200, 64, BF16)
    wide = torch.zeros(200, 72, device="cuda", dtype=BF16)
    wide[:, 1:65] = W
    check(mwb.token_loss(h, wide[:, 1:65], t), reference(h, W, t), ("loss", "total"))
    check(mwb.token_loss_gradient(h, wide[:, 1:65], t), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V,D", [(256, 520, 64), (256, 8200, 300), (1300, 4100, 260), (2600, 2100, 2050), (5000, 1100, 1024)])
def test_waves_of_tiles_with_a_rest(N, V, D, dtype):
    h, W, t = make(N, V, D, dtype, left_out=0.05)
    check(mwb.token_loss_gradient(h, W, t), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("D", [65, 64, 130])
def test_pieces_with_gradients_off_the_boundaries(D, kind, dtype):
    h, W, t = make(900, 301, D, dtype, left_out=0.4)
    wide = torch.full((301, D + 7), 5.0, device="cuda", dtype=kind)
    r = mwb.token_loss_gradient(h, W, t, piece_rows=256, dweight=wide[:, 3:3 + D])
    check(r, reference(h, W, t), ALL)
    assert bool((wide[:, :3] == 5).all() and (wide[:, 3 + D:] == 5).all())
    r = mwb.token_loss_gradient(h, W, t, piece_rows=256, grad_dtype=kind)
    check(r, reference(h, W, t), ALL)


def test_lookup_in_a_table_beyond_2_31_elements():
    V, D = 2200000, 1024
    table = torch.zeros(V, D, device="cuda", dtype=BF16)
    t = torch.tensor([V - 1, 0, V - 1, V, V - 2, -1], device="cuda")
    rows = torch.randn(6, D, device="cuda").to(BF16)
    table[V - 1], table[V - 2], table[0] = rows[0], rows[1], rows[2]
    out = mwb.embedding(t, table)
    zero = torch.zeros_like(rows[0])
    assert torch.equal(out, torch.stack([rows[0], rows[2], rows[0], zero, rows[1], zero]))
    d = mwb.embedding_backward(t, rows, V)
    near = torch.cat([d[:3], d[-3:]])
    s = torch.tensor([0, -1, 2, -1, -1, 1], device="cuda")
    check_gradient(near, torch.tensor([5, 0, 5, -1, 4, -1], device="cuda"), rows, 6, 1.0)
    assert s.shape == (6,) and float(d[3:-3].abs().amax()) == 0.0


def test_exponentials_beyond_2_31_elements():
    N, V, D = 16384, 140000, 64
    h, W, t = make(N, V, D, BF16, lean=4.0)
    r = mwb.token_loss_gradient(h, W, t, piece_rows=N)
    at = torch.tensor([0, 77777, V - 1], device="cuda")
    lse = torch.cat([torch.logsumexp(p.double() @ W.double().T, 1) for p in h.split(1024)])
    hd = h.double()
    loss = lse - (hd * W[t].double()).sum(1)
    assert float((r.loss.double() - loss).abs().max()) <= 1e-4          # (S < 100 here: 12 x 2^-23 x 100, twice, and 2^-20 x 20)
    # dW of three rows of the vocabulary: relative errors of p of 2^-10, of its products of 2^-13 and less
    dz = (torch.exp(hd @ W[at].double().T - lse[:, None]) - (t[:, None] == at).double()) / N
    want, size = dz.T @ hd, dz.abs().T @ hd.abs()
    off = (r.dweight[at].double() - want).abs()
    assert bool((off <= 1.2e-3 * size + 2.0 ** -8 * want.abs() + 2.0 ** -38).all())
    # dh of the last rows
    p = torch.exp(hd[-64:] @ W.double().T - lse[-64:, None]) / N
    p[torch.arange(64, device="cuda"), t[-64:]] -= 1 / N
    want, size = p @ W.double(), p.abs() @ W.double().abs()
    off = (r.dh[-64:].double() - want).abs()
    assert bool((off <= 2.2e-3 * size + 2.0 ** -8 * want.abs() + 2.0 ** -38).all())          # (140000 / 16 cut-offs: 1e-3)


def test_two_calls_at_once():
    a, b = make(600, 5000, 256, BF16, seed=1), make(500, 4000, 320, F32, seed=2)
    t = torch.randint(0, 300, (5000,), device="cuda")
    d = torch.randn(5000, 256, device="cuda")
    want = (mwb.token_loss_gradient(*a), mwb.token_loss_gradient(*b), mwb.embedding_backward(t, d, 300))
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        got = (mwb.token_loss_gradient(*a, stream=s[0]), mwb.token_loss_gradient(*b, stream=s[1]),
               mwb.embedding_backward(t, d, 300, stream=s[2]))
        torch.cuda.synchronize()
        for x, y in zip(got[:2], want[:2]):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
        assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V,piece", [(2500, 700, 0), (2500, 700, 512), (1030, 5000, 256)])
def test_captured_calls_of_many_rows_and_pieces(N, V, piece, dtype):
    h, W, t = make(N, V, 128, dtype)
    call = lambda: mwb.token_loss_gradient(h, W, t, piece_rows=piece)
    call(), mwb.token_loss(h, W, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, only = call(), mwb.token_loss(h, W, t)
    for seed, out in ((3, 0.0), (4, 0.8), (5, 1.0)):
        for a, b in zip((h, W, t), make(N, V, 128, dtype, seed=seed, left_out=out)):
            a.copy_(b)
        graph.replay()
        got = [x.clone() for x in (*held, only.loss, only.total)]
        fresh, loss = call(), mwb.token_loss(h, W, t)
        assert all(torch.equal(a, b) for a, b in zip(got, (*fresh, loss.loss, loss.total)))
        check(fresh, reference(h, W, t), ALL)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("N,V,D", [(1, 1, 64), (1, 5000, 128), (3, 70, 64), (64, 333, 320), (65, 20000, 64), (128, 4097, 192), (129, 4097, 192)])
def test_gradients_of_few_rows(N, V, D, kind):
    h, W, t = make(N, V, D, BF16, seed=N, left_out=0.3 if N > 3 else 0.0)
    check(mwb.token_loss_gradient(h, W, t, grad_dtype=kind, scale=1.3), reference(h, W, t, scale=1.3), ALL)
    w = torch.randn(N, device="cuda") * 1e-4
    w[::4] = 0
    h[::4] = float("inf")
    want = reference(h, W, t, weight=w)
    r = mwb.token_loss_gradient(h, W, t, row_weight=w, grad_dtype=kind, piece_rows=1)
    check(r, want, ALL)
    full = mwb.token_loss_gradient(h, W, t, row_weight=w, grad_dtype=kind)
    own, wide = h.clone(), torch.zeros(V, D + 8, device="cuda", dtype=BF16)
    wide[:, 8:] = W
    again = mwb.token_loss_gradient(own, wide[:, 8:], t, row_weight=w, grad_dtype=kind, dh=own)
    assert all(torch.equal(a, b) for a, b in zip(full, again)) and again.dh is own
    wide[:, 1:D + 1] = W.clone()                   # off the boundary: copied
    check(mwb.token_loss_gradient(h, wide[:, 1:D + 1], t, row_weight=w, grad_dtype=kind), want, ALL)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("N,V,D", [(1, 12353, 1088), (17, 13001, 1024), (64, 6151, 2112), (100, 12288, 1024), (128, 12353, 1088), (129, 12353, 1088), (8, 200000, 64)])
def test_gradients_of_few_rows_and_a_large_weight(N, V, D, kind):
    h, W, t = make(N, V, D, BF16, seed=N, left_out=0.3 if N > 1 else 0.0)
    if N > 1:
        t[N - 1] = V - 1
        h[N - 1] = W[V - 1]
    check(mwb.token_loss_gradient(h, W, t, grad_dtype=kind, scale=-1.3), reference(h, W, t, scale=-1.3), ALL)
    w = torch.randn(N, device="cuda") * 1e-4 * (torch.arange(N, device="cuda") % 4 != 1)
    h[1::4] = float("inf")                         # left out by their weight
    want = reference(h * 2.0 ** 30, W * 2.0 ** -30, t, weight=w)
    full = mwb.token_loss_gradient(h * 2.0 ** 30, W * 2.0 ** -30, t, row_weight=w, grad_dtype=kind)
    check(full, want, ALL)
    own, wide, out = h * 2.0 ** 30, torch.zeros(V, D + 8, device="cuda", dtype=BF16), torch.full((V, D + 7), 5.0, device="cuda", dtype=kind)
    wide[:, 8:] = W * 2.0 ** -30
    again = mwb.token_loss_gradient(own, wide[:, 8:], t, row_weight=w, grad_dtype=kind, dh=own, dweight=out[:, 3:D + 3])
    assert all(torch.equal(a, b) for a, b in zip(full, again)) and again.dh is own
    assert bool((out[:, :3] == 5).all() and (out[:, D + 3:] == 5).all())
    part = mwb.token_loss_gradient(h * 2.0 ** 30, W * 2.0 ** -30, t, row_weight=w, grad_dtype=kind, piece_rows=1)
    assert all(torch.equal(a, b) for a, b in zip(full, part))
    if N > 2:
        h, W, t = make(N, V, D, BF16, seed=N)
        clean = mwb.token_loss_gradient(h, W, t)
        h[2] = float("nan")
        r = mwb.token_loss_gradient(h, W, t)
        rest = torch.arange(N, device="cuda") != 2
        assert bool(r.loss[2].isnan()) and bool(r.dh[2].isnan().all())
        assert torch.equal(r.loss[rest], clean.loss[rest]) and torch.equal(r.dh[rest], clean.dh[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V", [(1, 30000), (3, 20001), (70, 8300), (128, 8192), (129, 8193), (290, 700), (300, 700)])
def test_rows_of_several_blocks(N, V, dtype):
    h, W, t = make(N, V, 136, dtype, seed=V, left_out=0.2 if N > 1 else 0.0)
    t[0] = V - 1
    h[0] = W[V - 1]
    check(mwb.token_loss_gradient(h, W, t), reference(h, W, t), ALL)
    check(mwb.token_loss_gradient(h, W, t, piece_rows=256), reference(h, W, t), ALL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,D", [(4103, 1030), (65601, 64), (1031, 4100), (1039, 4101), (70, 60000)])
@pytest.mark.parametrize("N", [1, 3, 4, 5, 8, 9, 16, 17])
def test_very_few_rows(N, V, D, dtype):
    h, W, t = make(N, V, D, dtype, seed=N + V, left_out=0.3 if N > 1 else 0.0)
    t[0], h[0] = V - 1, W[V - 1]
    want = reference(h, W, t, scale=-0.7)
    check(mwb.token_loss(h, W, t, scale=-0.7), want, ("loss", "total"))
    kind = F32 if N % 2 else BF16
    r = mwb.token_loss_gradient(h, W, t.to(torch.int32), scale=-0.7, grad_dtype=kind)
    check(r, want, ALL)
    out = (t < 0) | (t >= V)
    assert bool((r.loss[out] == 0).all() and (r.dh[out] == 0).all())
    w = torch.randn(N, device="cuda") * 1e3 * (torch.arange(N, device="cuda") % 4 != 1)
    h[1::4] = float("nan")
    want = reference(h, W, t, weight=w)
    check(mwb.token_loss(h, W, t, row_weight=w), want, ("loss", "total"))
    full = mwb.token_loss_gradient(h, W, t, row_weight=w, grad_dtype=kind)
    check(full, want, ALL)
    # windows of wider rows at odd places, h's own place for dh: other loads, the same numbers to rounding
    wide, hw, grad = (torch.full((n, D + 9), 5.0, device="cuda", dtype=k) for n, k in ((V, dtype), (N, dtype), (V, kind)))
    wide[:, 1:D + 1], hw[:, 5:D + 5] = W, h
    again = mwb.token_loss_gradient(hw[:, 5:D + 5], wide[:, 1:D + 1], t, row_weight=w, dh=hw[:, 5:D + 5], dweight=grad[:, 3:D + 3], piece_rows=1)
    check(again, want, ALL)
    for x, at in ((hw, 5), (grad, 3)):
        assert bool((x[:, :at] == 5).all() and (x[:, at + D:] == 5).all())
    only = mwb.token_loss_gradient(h, W, t, row_weight=w, grad_dtype=kind, want=(False, True))
    assert only.dh is None and torch.equal(only.dweight, full.dweight)
    only = mwb.token_loss_gradient(h, W, t, row_weight=w, want=(True, False))
    assert only.dweight is None and torch.equal(only.dh, full.dh)


@pytest.mark.parametrize("left_out", [0.0, 1.0])
def test_very_few_rows_captured_and_not_finite(left_out):
    h, W, t = make(12, 9001, 520, F32, left_out=left_out)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
    for seed in (1, 2):
        h2, W2, t2 = make(12, 9001, 520, F32, seed=seed, left_out=left_out)
        h.copy_(h2), W.copy_(W2), t.copy_(t2)
        graph.replay()
        check(b, reference(h, W, t), ALL)
        c, d = mwb.token_loss(h, W, t), mwb.token_loss_gradient(h, W, t)
        assert torch.equal(a.loss, c.loss) and torch.equal(a.total, c.total) and all(torch.equal(x, y) for x, y in zip(b, d))
    if left_out == 0.0:
        h[5, 3] = float("nan")
        r = mwb.token_loss_gradient(h, W, t)
        rest = torch.arange(12, device="cuda") != 5
        assert bool(r.loss[5].isnan()) and bool(r.dh[5].isnan().all())
        assert torch.equal(r.loss[rest], d.loss[rest]) and torch.equal(r.dh[rest], d.dh[rest])


@pytest.mark.parametrize("N,V,D", [(1, 1, 1), (2, 63, 5), (8, 64, 128), (3, 65, 129), (8, 20011, 4), (5, 1000, 257), (8, 3, 2050), (7, 500, 8200)])
def test_very_few_rows_of_small_sizes(N, V, D):
    h, W, t = make(N, V, D, F32, seed=V, std=3.0)
    t[0] = V - 1
    want = reference(h, W, t, scale=2.0)
    check(mwb.token_loss(h, W, t, scale=2.0), want, ("loss", "total"))
    check(mwb.token_loss_gradient(h, W, t, scale=2.0), want, ALL)
    check(mwb.token_loss_gradient(h, W, t, scale=0.0), reference(h, W, t, scale=0.0), ALL)
    big = 2.0 ** 60
    check(mwb.token_loss_gradient(h * big, W / big, t, scale=2.0), reference(h * big, W / big, t, scale=2.0), ALL)
    h, W, t = make(N, V, D, F32, seed=V, lean=200.0 if V > 1 and D > 4 else 0.0)
    check(mwb.token_loss_gradient(h, W, t), reference(h, W, t), ALL)
    if V > 1:
        # a row of the vocabulary that is never chosen
        h, t = h.abs() + 0.5, t.clamp(min=1)
        W[0] = float("-inf")
        check(mwb.token_loss(h, W, t), reference(h, W[1:], t - 1), ("loss", "total"))
