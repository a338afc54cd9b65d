"""The table's gradient of more tokens than one cluster sorts (65536): tables of one, two and three digits, both sides of the
switch, added gradients, replayed graphs.  Formulas and tolerances are those of test_gpu_embedding.py."""
import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_gpu_embedding import check_gradient, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("V", [255, 256, 70000, (1 << 20) - 1])
@pytest.mark.parametrize("n", [65536, 65537, 200003])
def test_tables_of_several_digits(n, V, ids):
    t, _, dout = make(n, V, 4, torch.float32, seed=n % 97 + V, common=0.2, ids=ids)
    got = mwb.embedding_backward(t, dout, V, scale=0.5)
    check_gradient(got, t, dout, V, 0.5)
    assert torch.equal(got, mwb.embedding_backward(t, dout, V, scale=0.5))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [200, 70000])
@pytest.mark.parametrize("n", [65536, 65537, 131073])
def test_added_gradients(n, V, dtype):
    t, _, dout = make(n, V, 24, dtype, seed=n % 89, common=0.3)
    t[(t >= 5) & (t < 9)] = 9
    before = torch.randn(V, 24, device="cuda").to(dtype)
    before[5:9] = float("nan")                       # named by no token: left alone
    got = before.clone()
    mwb.embedding_backward(t, dout, V, dtable=got, accumulate=True)
    assert bool(got[5:9].isnan().all())
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[5:9] = False
    check_gradient(torch.where(rest[:, None], got, 0.0), t, dout, V, 1.0, before=torch.where(rest[:, None], before, 0.0))


def test_tokens_that_name_no_row():
    n, V = 70000, 300
    t, dout = torch.full((n,), -1, device="cuda"), torch.full((n, 8), float("nan"), device="cuda")
    assert bool((mwb.embedding_backward(t, dout, V) == 0).all())
    kept = torch.randn(V, 8, device="cuda")
    got = kept.clone()
    mwb.embedding_backward(t, dout, V, dtable=got, accumulate=True)
    assert torch.equal(got, kept)


def test_a_captured_call():
    n, V = 80000, 70000
    t, _, dout = make(n, V, 16, torch.bfloat16)
    call = lambda: mwb.embedding_backward(t, dout, V)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed, common in ((1, 0.0), (2, 0.9)):
        new, _, d = make(n, V, 16, torch.bfloat16, seed=seed, common=common)
        t.copy_(new), dout.copy_(d)
        graph.replay()
        assert torch.equal(held, call())
        check_gradient(held, t, dout, V, 1.0)
