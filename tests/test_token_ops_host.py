"""What the bindings of the lookup, the vocabulary's loss and the clipping hand to the library and what they refuse, seen
without a GPU: CPU tensors stand in for CUDA ones, and a recorder stands in for the library."""
import ctypes as C

import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from test_sequence_ops_host import OnSecond, Stream, devices, on_device, recorder, second, streams  # noqa: F401

N, V, D = 24, 50, 16


def ids(*shape, dtype=torch.int64, V=V):
    return on_device(torch.randint(0, V, shape, dtype=dtype))


def reach(rows, ld, cols, size):
    return ((rows - 1) * (ld or cols) + cols) * size if rows else 0


@pytest.fixture
def allocations(monkeypatch):
    """Memory that the bindings ask for on a device is the CPU's here."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))


def test_lookup_reads_and_writes_inside_its_memory(recorder, allocations):
    wide = on_device(torch.randn(V, 40))
    for table in (on_device(torch.randn(V, D)), wide[:, 3:3 + D], on_device(torch.randn(1, D).expand(V, D)),
                  on_device(torch.randn(()).expand(V, D))):
        for tokens in (ids(N), ids(4, 6), ids(6, 4).T, ids(N, dtype=torch.int32), ids(0)):
            recorder.calls.clear()
            out = mwb.embedding(tokens, table, scale=2.0)
            name, (d, t, w, o, _) = recorder.calls[-1]
            assert name == "mw_embedding_forward" and out.shape == (*tokens.shape, D)
            assert (d.tokens, d.vocab, d.dim, d.index_bytes, d.scale) == (tokens.numel(), V, D, tokens.element_size(), 2.0)
            if tokens.numel():
                assert tokens.numel() * d.index_bytes <= recorder.room[t]
                assert reach(V, d.ld_table, D, 4) <= recorder.room[w] and reach(N, d.ld_out, D, 4) <= recorder.room[o]


def test_table_gradient_reads_and_writes_inside_its_memory(recorder, allocations):
    wide = on_device(torch.randn(N, 40))
    for dout in (on_device(torch.randn(N, D)), wide[:, 1:1 + D], on_device(torch.ones(()).expand(N, D)),
                 on_device(torch.randn(4, 6, D)), on_device(torch.randn(6, 4, D)).transpose(0, 1), wide.view(4, 6, 40)[:, :, :D]):
        tokens = ids(*dout.shape[:-1])
        for dtable in (None, on_device(torch.zeros(V, 30))[:, 2:2 + D]):
            recorder.calls.clear()
            got = mwb.embedding_backward(tokens, dout, V, dtable=dtable)
            name, (d, t, y, g, add, ws, size, _) = recorder.calls[-1]
            assert name == "mw_embedding_backward" and got.shape == (V, D) and add == 0
            assert d.tokens == N and N * 8 <= recorder.room[t]
            assert reach(N, d.ld_out, D, 4) <= recorder.room[y] and reach(V, d.ld_dtable, D, 4) <= recorder.room[g]


def test_loss_reads_and_writes_inside_its_memory(recorder, allocations):
    wide, wider = on_device(torch.randn(N, 40)), on_device(torch.randn(V, 33))
    for h in (on_device(torch.randn(N, D)), wide[:, 5:5 + D], on_device(torch.randn(1, D).expand(N, D)), on_device(torch.randn(0, D))):
        for w in (on_device(torch.randn(V, D)), wider[:, 1:1 + D], on_device(torch.randn(V, 1).expand(V, D))):
            rows = h.shape[0]
            t, g = ids(rows), on_device(torch.ones(rows))

            def check(name):             # (at once: memory that a call lets go of is soon another tensor's)
                called, args = recorder.calls[-1]
                d = args[0]
                assert called == name and (d.rows, d.vocab, d.dim, d.index_bytes) == (rows, V, D, 8)
                assert reach(V, d.ld_weight, D, 4) <= recorder.room[args[2]]
                if rows:
                    assert reach(rows, d.ld_h, D, 4) <= recorder.room[args[1]]
                    assert rows * 8 <= recorder.room[args[3]] and rows * 4 <= recorder.room[args[4]]
                    assert rows * 4 <= recorder.room[args[5]] and 4 <= recorder.room[args[6]]
                if name.endswith("gradient"):
                    assert rows == 0 or reach(rows, d.ld_dh, D, 4) <= recorder.room[args[7]]
                    assert reach(V, d.ld_dweight, D, 4) <= recorder.room[args[8]]

            r = mwb.token_loss(h, w, t, row_weight=g)
            check("mw_token_loss_forward")
            assert r.loss.shape == (rows,) and r.total.shape == () and r.dh is None
            q = mwb.token_loss_gradient(h, w, t, row_weight=g)
            check("mw_token_loss_gradient")
            assert q.dh.shape == h.shape and q.dweight.shape == w.shape


def test_loss_copies_a_weight_that_starts_off_its_boundary(recorder, allocations):
    base = on_device(torch.randn(V * 24 + 8).bfloat16())
    off = (-base.data_ptr() // 2) % 8 + 1                      # two bytes beyond a 16-byte boundary
    w = torch.as_strided(base, (V, D), (24, 1), off)
    assert w.data_ptr() % 16 == 2
    mwb.token_loss(on_device(torch.randn(N, D).bfloat16()), w, ids(N))
    d, _, at = recorder.calls[-1][1][:3]
    assert at % 16 == 0 and reach(V, d.ld_weight, D, 2) <= recorder.room[at]


def test_clip_hands_over_what_it_is_given(recorder, allocations, monkeypatch):
    g = [on_device(torch.randn(3, 5)), on_device(torch.randn(7).bfloat16()), on_device(torch.randn(0))]
    o = [torch.empty_like(t) for t in g]
    seen = []

    def clip(n, src, dst, sizes, kinds, most, norm, ws, size, stream):
        at = lambda kind, address: list((kind * n).from_address(address))
        seen.append((at(C.c_uint64, src), at(C.c_uint64, dst), at(C.c_int64, sizes), at(C.c_int32, kinds), most, norm))
        return mwb.MW_OK

    monkeypatch.setattr(recorder, "mw_clip_gradients", clip, raising=False)
    for out in (None, o):
        norm = mwb.clip_gradients(g, 2.0, out=out)
        assert norm.shape == () and seen.pop() == ([t.data_ptr() for t in g], [t.data_ptr() for t in out or g], [15, 7, 0],
                                                   [1, 2, 1], 2.0, norm.data_ptr())


def refuse(call, kind=ValueError):
    with pytest.raises(kind):
        call()


def test_refusals(recorder, allocations):
    t, table, dout = ids(N), on_device(torch.randn(V, D)), on_device(torch.randn(N, D))
    h, w = on_device(torch.randn(N, D)), table
    g = [on_device(torch.randn(4, 4)), on_device(torch.randn(9))]
    half = lambda x: on_device(x.half())
    rep = on_device(torch.zeros(1, D))
    refuse(lambda: mwb.embedding(t, torch.randn(V, D)))                                     # on the CPU
    refuse(lambda: mwb.embedding(t, half(table)), TypeError)
    refuse(lambda: mwb.embedding(on_device(t.float()), table), TypeError)
    refuse(lambda: mwb.embedding(t, on_device(torch.randn(D, V)).T))                        # columns apart
    refuse(lambda: mwb.embedding(t, on_device(torch.randn(V))))
    refuse(lambda: mwb.embedding(t, on_device(torch.randn(0, D))))
    refuse(lambda: mwb.embedding(t, table, out=on_device(torch.zeros(N, D + 1))))
    refuse(lambda: mwb.embedding(t, table, out=on_device(torch.zeros(N, D).bfloat16())))
    refuse(lambda: mwb.embedding(t, table, out=rep.expand(N, D)))
    refuse(lambda: mwb.embedding_backward(t, on_device(torch.randn(N + 1, D)), V))
    refuse(lambda: mwb.embedding_backward(t, half(dout), V), TypeError)
    refuse(lambda: mwb.embedding_backward(t, dout, V, grad_dtype=torch.float16), TypeError)
    refuse(lambda: mwb.embedding_backward(t, dout, V, accumulate=True))                     # nothing to add to
    refuse(lambda: mwb.embedding_backward(t, dout, V, dtable=on_device(torch.zeros(V + 1, D))))
    refuse(lambda: mwb.embedding_backward(t, dout, V, dtable=rep.expand(V, D)))
    refuse(lambda: mwb.embedding_backward(t, dout, V, dtable=on_device(torch.zeros(V, D)), grad_dtype=torch.bfloat16))
    for f in (mwb.token_loss, mwb.token_loss_gradient):
        refuse(lambda: f(torch.randn(N, D), w, t))
        refuse(lambda: f(h, on_device(torch.randn(V, D + 1)), t))
        refuse(lambda: f(h, on_device(w.bfloat16()), t))
        refuse(lambda: f(half(h), half(w), t), TypeError)
        refuse(lambda: f(h, w, ids(N + 1)))
        refuse(lambda: f(h, w, ids(N, 2)[:, 0]))
        refuse(lambda: f(h, w, on_device(t.to(torch.int16))), TypeError)
        refuse(lambda: f(h, w, t, row_weight=on_device(torch.ones(N).double())))
        refuse(lambda: f(h, w, t, row_weight=on_device(torch.ones(N + 1))))
        refuse(lambda: f(on_device(torch.randn(D, N)).T, w, t))
        refuse(lambda: f(on_device(torch.randn(N, 2, D)), w, t))
    refuse(lambda: mwb.token_loss_gradient(h, w, t, dh=rep.expand(N, D)))
    refuse(lambda: mwb.token_loss_gradient(h, w, t, dh=on_device(torch.zeros(N, D).bfloat16())))
    refuse(lambda: mwb.token_loss_gradient(h, w, t, dweight=rep.expand(V, D)))
    refuse(lambda: mwb.token_loss_gradient(h, w, t, dweight=on_device(torch.zeros(V, D)), grad_dtype=torch.bfloat16))
    refuse(lambda: mwb.clip_gradients([], 1.0))
    refuse(lambda: mwb.clip_gradients([torch.randn(3)], 1.0))
    refuse(lambda: mwb.clip_gradients(g, 1.0, out=g[:1]))
    refuse(lambda: mwb.clip_gradients([g[0].T[:3]], 1.0))                                   # rows apart
    refuse(lambda: mwb.clip_gradients([half(g[0])], 1.0))
    refuse(lambda: mwb.clip_gradients(g, 1.0, out=[on_device(torch.zeros(4, 4)), on_device(torch.zeros(8))]))
    refuse(lambda: mwb.clip_gradients(g, 1.0, out=[on_device(torch.zeros(4, 4)), on_device(torch.zeros(9).bfloat16())]))
    work = {"mw_embedding_forward", "mw_embedding_backward", "mw_token_loss_forward", "mw_token_loss_gradient", "mw_clip_gradients"}
    assert not work & {name for name, _ in recorder.calls}


def sec(*shape, dtype=torch.float32):
    return second(*shape, dtype=dtype)


def sec_ids(*shape):
    return torch.randint(0, V, shape).as_subclass(OnSecond)


def test_calls_run_with_the_tensors_device_current(devices, recorder, allocations):
    t, table, h, w = sec_ids(N), sec(V, D), sec(N, D), sec(V, D)
    g = [sec(3, 4)]
    for _ in range(2):                 # the first call of a layout and a remembered one
        mwb.embedding(t, table, out=sec(N, D))
        mwb.embedding_backward(t, h, V, dtable=sec(V, D))
        mwb.token_loss(h, w, t)
        mwb.token_loss_gradient(h, w, t, dh=sec(N, D), dweight=sec(V, D))
        mwb.clip_gradients(g, 1.0)
    launched = [c for c in recorder.at if not c[0].endswith("scratch_bytes")]
    assert len(launched) == 12 and all(at == 1 for _, at in launched), recorder.at
    assert devices[0] == 0


def test_tensors_of_two_devices_are_refused(devices, recorder, allocations):
    other = on_device(torch.randn(V, D))
    refuse(lambda: mwb.embedding(sec_ids(N), other))
    refuse(lambda: mwb.embedding_backward(sec_ids(N), sec(N, D), V, dtable=other))
    refuse(lambda: mwb.token_loss(sec(N, D), other, sec_ids(N)))
    refuse(lambda: mwb.token_loss_gradient(sec(N, D), sec(V, D), sec_ids(N), dweight=other))
    refuse(lambda: mwb.embedding(sec_ids(N), sec(V, D), stream=Stream(0)))
    refuse(lambda: mwb.token_loss(sec(N, D), sec(V, D), sec_ids(N), stream=Stream(0)))


def test_everything_a_call_on_another_stream_touches_is_marked_for_it(streams, recorder):
    s = Stream(1)

    def check(tensors, call):
        streams.clear()
        call()
        for i, t in enumerate(tensors):
            assert (t.data_ptr(), s) in streams, i

    t, table, out, dout, dtable = sec_ids(N), sec(V, D), sec(N, D), sec(N, D), sec(V, D)
    check([t, table, out], lambda: mwb.embedding(t, table, out=out, stream=s))
    check([t, dout, dtable], lambda: mwb.embedding_backward(t, dout, V, dtable=dtable, stream=s))
    h, w, dh, dw, g = sec(N, D), sec(V, D), sec(N, D), sec(V, D), sec(N)
    check([h, w, t, g], lambda: mwb.token_loss(h, w, t, row_weight=g, stream=s))
    check([h, w, t, g, dh, dw], lambda: mwb.token_loss_gradient(h, w, t, row_weight=g, dh=dh, dweight=dw, stream=s))
    grads, clipped = [sec(4, 4), sec(9)], [sec(4, 4), sec(9)]
    check(grads + clipped, lambda: mwb.clip_gradients(grads, 1.0, out=clipped, stream=s))
    check(grads, lambda: mwb.clip_gradients(iter(grads), 1.0, stream=s))
