"""Plans of the orthogonalised update and threads."""
import threading

import pytest

from paper_2402_14212_b200 import binding as mwb

pytestmark = pytest.mark.gpu


def test_a_call_may_be_its_threads_first_touch_of_the_device():
    import torch
    plan = mwb.Orth(300, 260, 2, "bf16_f32acc")
    mats = [torch.randn(300, 260, device="cuda").bfloat16() for _ in range(2)]
    spaces, bad = [plan.alloc_workspace() for _ in range(2)], []
    want = plan.project(mats, spaces[0])
    out = [torch.empty_like(m) for m in mats]
    torch.cuda.synchronize()

    def work():
        try:
            plan.project(mats, spaces[1], out=out)
        except Exception as e:          # noqa: BLE001 (reported below)
            bad.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join(120)
    assert not bad and plan.status(spaces[1]) == 0 and all(torch.equal(p, q) for p, q in zip(out, want))


def test_threads_share_a_plan_with_a_workspace_each():
    import torch
    plan = mwb.Orth(300, 260, 2, "bf16_f32acc")
    inputs = [[torch.randn(300, 260, device="cuda").bfloat16() for _ in range(2)] for _ in range(4)]
    want = [plan.project(m, plan.alloc_workspace()) for m in inputs]
    spaces = [plan.alloc_workspace() for _ in inputs]
    bad, start = [], threading.Barrier(len(inputs))

    def work(i):
        try:
            start.wait(20)
            got = [plan.project(inputs[i], spaces[i]) for _ in range(40)]
            torch.cuda.synchronize()
            if not all(torch.equal(p, q) for g in got for p, q in zip(g, want[i])):
                bad.append(i)
        except Exception as e:          # noqa: BLE001 (reported below)
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(inputs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not bad and not any(t.is_alive() for t in threads)
    assert all(plan.status(ws) == 0 for ws in spaces)


# one CTA a matrix; a few tiles; more tiles a phase than CTA pairs
@pytest.mark.parametrize("prec", ["f32", "bf16_f32acc"])
@pytest.mark.parametrize("rows,cols,count", [(64, 64, 3), (300, 260, 2), (1100, 1030, 8)])
def test_a_wait_that_runs_out_leaves_the_weights_alone(rows, cols, count, prec):
    import torch
    timeout = mwb.STATUS_NAMES.index("MW_ERR_TIMEOUT")
    plan = mwb.Orth(rows, cols, count, prec)
    ws = plan.alloc_workspace()
    rand = lambda dt: [torch.randn(rows, cols, device="cuda").to(dt) for _ in range(count)]
    W, G, M = rand(plan.storage_dtype()), rand(torch.float32), rand(torch.float32)
    fresh = lambda ts: [t.clone() for t in ts]
    want_w, want_m = fresh(W), fresh(M)
    plan.step(want_w, G, want_m, ws, lr=0.02)
    want_x = plan.project(W, ws)
    assert plan.status(ws) == 0
    for _ in range(2):
        w, m, x = fresh(W), fresh(M), fresh(W)
        plan.selftest_unmet_wait(5)
        plan.step(w, G, m, ws, lr=0.02)
        assert plan.status(ws) == timeout
        plan.project(x, ws, out=x)
        assert plan.status(ws) == timeout
        assert all(torch.equal(p, q) for p, q in zip(w + x, W + W)) and all(torch.equal(p, q) for p, q in zip(m, want_m))
        # counters and tensor memory were left in order: the same call right after is correct
        plan.selftest_unmet_wait(0)
        m = fresh(M)
        plan.step(w, G, m, ws, lr=0.02)
        assert plan.status(ws) == 0 and all(torch.equal(p, q) for p, q in zip(w + m, want_w + want_m))
        assert all(torch.equal(p, q) for p, q in zip(plan.project(W, ws), want_x))


def test_the_self_test_refuses_limits_out_of_range():
    plan = mwb.Orth(8, 8, 1, "f32")
    with pytest.raises(mwb.MwError):
        plan.selftest_unmet_wait(1001)
