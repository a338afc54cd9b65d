"""Host-side checks of the lookup, the vocabulary's loss and the clipping: bad descriptions are refused before any GPU
work, sizes come out as documented (runs without a GPU)."""
import ctypes as C

import pytest

from paper_2402_14212_b200 import binding as mwb

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def embed(**kw):
    d = dict(tokens=40, vocab=100, dim=64, dtype=1, grad_dtype=0, index_bytes=8, reserved=0, ld_table=0, ld_out=0,
             ld_dtable=0, scale=1.0)
    d.update(kw)
    return mwb.EmbeddingDesc(**d)


BAD_EMBED = [(dict(tokens=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(dtype=0), UNSUPPORTED),
             (dict(dtype=3), INVALID), (dict(grad_dtype=3), INVALID), (dict(index_bytes=2), INVALID),
             (dict(reserved=1), INVALID), (dict(ld_table=63), INVALID), (dict(ld_out=1), INVALID),
             (dict(ld_dtable=63), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
             (dict(tokens=(1 << 30) + 1), UNSUPPORTED), (dict(vocab=2 ** 31 - 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_EMBED)
def test_embedding_descriptions(kw, code):
    L, n = mwb.lib(), C.c_size_t()
    d = embed(**kw)
    assert L.mw_embedding_scratch_bytes(d, C.byref(n)) == code
    assert L.mw_embedding_forward(d, 256, 256, 256, None) == code
    assert L.mw_embedding_backward(d, 256, 256, 256, 0, 256, 1 << 40, None) == code


def test_embedding_calls():
    L, n = mwb.lib(), C.c_size_t()
    assert L.mw_embedding_scratch_bytes(embed(), None) == INVALID
    assert L.mw_embedding_scratch_bytes(None, C.byref(n)) == INVALID
    # two copies of keys and positions, and two sums for 32 tokens
    assert L.mw_embedding_scratch_bytes(embed(), C.byref(n)) == OK and n.value >= 40 * 16 + 2 * 2 * 64 * 4
    for hole in range(3):
        p = [256, 256, 256]
        p[hole] = None
        assert L.mw_embedding_forward(embed(), *p, None) == INVALID
        assert L.mw_embedding_backward(embed(), *p, 0, 256, n.value, None) == INVALID
    assert L.mw_embedding_forward(embed(tokens=0), None, None, None, None) == OK
    back = lambda acc=0, ws=256, size=n.value: L.mw_embedding_backward(embed(), 256, 256, 256, acc, ws, size, None)
    assert back(acc=2) == INVALID and back(ws=None) == WORKSPACE and back(ws=128) == WORKSPACE and back(size=n.value - 1) == WORKSPACE


def loss(**kw):
    d = dict(rows=40, vocab=1000, dim=64, dtype=2, grad_dtype=0, index_bytes=8, piece_rows=0, ld_h=0, ld_weight=0, ld_dh=0,
             ld_dweight=0, scale=1.0)
    d.update(kw)
    return mwb.TokenLossDesc(**d)


BAD_LOSS = [(dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(dtype=0), UNSUPPORTED),
            (dict(dtype=3), INVALID), (dict(grad_dtype=-1), INVALID), (dict(index_bytes=1), INVALID),
            (dict(piece_rows=-1), INVALID), (dict(ld_h=63), INVALID), (dict(ld_weight=63), INVALID), (dict(ld_dh=63), INVALID),
            (dict(ld_dweight=63), INVALID), (dict(scale=float("nan")), INVALID), (dict(rows=(1 << 24) + 1), UNSUPPORTED),
            (dict(vocab=(1 << 24) + 1), UNSUPPORTED), (dict(rows=1 << 24, vocab=1 << 24), UNSUPPORTED), (dict(dim=(1 << 16) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_LOSS)
def test_loss_descriptions(kw, code):
    L, n = mwb.lib(), C.c_size_t()
    d = loss(**kw)
    assert L.mw_token_loss_workspace_bytes(d, 1, C.byref(n)) == code
    assert L.mw_token_loss_forward(d, 256, 256, 256, None, 256, 256, 256, 1 << 50, None) == code
    assert L.mw_token_loss_gradient(d, 256, 256, 256, None, 256, 256, 256, 256, 256, 1 << 50, None) == code


def test_loss_calls():
    L = mwb.lib()

    def need(gradient, **kw):
        n = C.c_size_t()
        assert L.mw_token_loss_workspace_bytes(loss(**kw), gradient, C.byref(n)) == OK
        return n.value

    n, m = need(1), need(0)
    assert L.mw_token_loss_workspace_bytes(loss(), 2, C.byref(C.c_size_t())) == INVALID
    assert L.mw_token_loss_workspace_bytes(loss(), 0, None) == INVALID
    assert need(0, rows=0) > 0
    fwd = lambda h=256, w=256, t=256, l=256, ws=256, size=m, **kw: L.mw_token_loss_forward(loss(**kw), h, w, t, None, l, None, ws, size, None)
    assert fwd(h=None) == fwd(w=None) == fwd(t=None) == fwd(l=None) == INVALID
    assert fwd(w=264) == INVALID                               # rows that are read in place start on 16 bytes
    assert fwd(ws=None) == fwd(ws=128) == fwd(size=m - 1) == WORKSPACE
    grad = lambda dh=256, dw=256, size=n, **kw: L.mw_token_loss_gradient(loss(**kw), 512, 256, 256, None, 256, None, dh, dw, 256, size, None)
    assert grad(size=n - 1) == WORKSPACE
    assert grad(dh=512, ld_h=80) == INVALID                    # in place needs the same rows
    assert L.mw_token_loss_status(None, None) == INVALID


def test_memory_of_the_gradient_goes_by_the_piece():
    """Exponentials are held for a piece of rows: half precision for bf16 operands (float for float ones), 1 GiB of them
    by default; the rest is operands, sums and the gradients' partial sums."""
    L = mwb.lib()

    def need(**kw):
        n = C.c_size_t()
        d = loss(rows=16384, vocab=131072, dim=512, **kw)
        assert L.mw_token_loss_workspace_bytes(d, 1, C.byref(n)) == OK
        return n.value

    whole = need(piece_rows=16384)
    operands = (16384 + 131072) * 512 * 2
    assert whole >= 16384 * 131072 * 2 + operands
    default, small = need(), need(piece_rows=1024)
    assert (1 << 30) + operands <= default <= (1 << 30) + 3 * (1 << 29) + operands
    assert default - small >= (4096 - 1024) * 131072 * 2
    assert need(dtype=1) >= (1 << 30) + 2 * operands


def test_clip_calls():
    L, n = mwb.lib(), C.c_size_t()
    assert L.mw_clip_scratch_bytes(-1, C.byref(n)) == INVALID and L.mw_clip_scratch_bytes(1, None) == INVALID
    assert L.mw_clip_scratch_bytes(1000, C.byref(n)) == OK and n.value >= 8
    two = (C.c_void_p * 2)(256, 512)
    hole = (C.c_void_p * 2)(256, None)
    sizes, types = (C.c_int64 * 2)(10, 20), (C.c_int32 * 2)(1, 2)

    def call(count=2, src=two, dst=two, size=sizes, kind=types, most=1.0, norm=256, ws=256, room=n.value):
        return L.mw_clip_gradients(count, src, dst, size, kind, most, norm, ws, room, None)

    for kw in (dict(count=-1), dict(src=None), dict(dst=None), dict(size=None), dict(kind=None), dict(src=hole), dict(dst=hole),
               dict(most=0.0), dict(most=-1.0), dict(most=float("nan")), dict(norm=None), dict(size=(C.c_int64 * 2)(10, -1)),
               dict(kind=(C.c_int32 * 2)(1, 0)), dict(kind=(C.c_int32 * 2)(3, 1))):
        assert call(**kw) == INVALID, kw
    assert call(ws=None) == call(ws=64) == call(room=0) == WORKSPACE
