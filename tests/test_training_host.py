"""Host-side checks of the entry points around an encoder's layers (no GPU
needed): arguments are refused before any launch, and workspaces hold what the
calls lay out in them."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    return g


D = C.c_void_p(1 << 20)        # never dereferenced
AT = [C.c_void_p((i + 1) << 40) for i in range(12)]      # buffers far apart
ODD = C.c_void_p((1 << 40) + 1)
WS = (C.c_void_p(1 << 46), 1 << 45)


def _made(cls, base, kw):
    p = cls(**base)
    for k, v in kw.items():
        setattr(p, k, v)
    return C.byref(p)


def _norm(g, **kw):
    return _made(g.NormParams, dict(n=10, k=16, ldx=16, ldy=16, eps=1e-5, dtype=2), kw)


def _drop(g, **kw):
    return _made(g.DropoutParams, dict(n=10, m=16, ldx=16, ldr=16, ldy=16, seed=1, offset=2, p=0.1,
                                       dtype=2, reserved=0), kw)


def _embed(g, **kw):
    return _made(g.EmbeddingParams, dict(n=10, k=16, rows=30, ldt=16, ldy=16, scale=1.0, dtype=2,
                                         id_bytes=8, accumulate=0), kw)


def _loss(g, **kw):
    return _made(g.LossParams, dict(n=10, k=16, v=30, ldx=16, ldw=16, dtype=2, id_bytes=8,
                                    aligned16=1, reserved=0), kw)


SIDES = [dict(n=-1), dict(n=2 ** 31), dict(dtype=3), dict(dtype=-1)]
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw", SIDES + [dict(k=0), dict(k=2 ** 20 + 1), dict(ldx=15), dict(ldy=15),
                                        dict(ldx=2 ** 22 + 1), dict(ldy=2 ** 22 + 1),
                                        dict(eps=-1.0), dict(eps=NAN), dict(eps=INF)], ids=str)
def test_norm_parameters_are_refused(g, kw):
    L, p = g.lib(), _norm(g, **kw)
    assert L.gpic_layer_norm(p, *AT[:5], None) == 1
    assert L.gpic_layer_norm_backward(p, *AT[:7], *WS, None) == 1
    assert L.gpic_layer_norm_workspace_bytes(p) == 0


def test_norm_buffers_are_refused(g):
    L, p, a = g.lib(), _norm(g), AT
    assert L.gpic_layer_norm(None, *a[:5], None) == 1
    assert L.gpic_layer_norm(p, None, a[1], a[2], a[3], a[4], None) == 1
    assert L.gpic_layer_norm(p, a[0], a[1], a[2], None, a[4], None) == 1
    for i in range(4):
        bad = list(a[:5])
        bad[i] = ODD
        assert L.gpic_layer_norm(p, *bad, None) == 1
    bad = list(a[:5])
    bad[4] = C.c_void_p((1 << 40) + 4)                   # stats are pairs
    assert L.gpic_layer_norm(p, *bad, None) == 1
    assert L.gpic_layer_norm(p, a[0], a[1], a[2], a[1], a[4], None) == 1        # Y over the weight
    assert b"overlaps" in L.gpic_last_error()
    over = C.c_void_p((1 << 40) + 32)                    # Y a row further on in X
    assert L.gpic_layer_norm(p, a[0], None, None, over, None, None) == 1
    assert L.gpic_layer_norm(_norm(g, ldy=32), a[0], None, None, a[0], None, None) == 1
    assert L.gpic_layer_norm(p, a[0], None, None, a[3], a[3], None) == 1        # stats over Y
    need = L.gpic_layer_norm_workspace_bytes(p)
    assert need >= 10 * 8 + 2 * 16 * 4
    call = lambda *b, ws=WS: L.gpic_layer_norm_backward(p, *b, *ws, None)  # noqa: E731
    assert call(None, *a[1:7]) == 1 and call(a[0], None, *a[2:7]) == 1
    assert call(*a[:3], None, *a[4:7]) == 1
    assert call(*a[:4], a[0], a[5], a[6]) == 1           # dX over dY
    assert call(*a[:4], a[4], a[5], a[5]) == 1           # dW and db one buffer
    assert call(*a[:7], ws=(WS[0], need - 1)) == 2 and call(*a[:7], ws=(None, 0)) == 2
    assert call(*a[:7], ws=(C.c_void_p(WS[0].value + 16), need)) == 1


@pytest.mark.parametrize("kw", SIDES + [dict(m=0), dict(m=2 ** 20 + 1), dict(ldx=15), dict(ldy=15),
                                        dict(ldr=15), dict(ldr=2 ** 22 + 1), dict(p=-0.1),
                                        dict(p=1.0), dict(p=1.0 - 2.0 ** -18), dict(p=NAN),
                                        dict(p=2.0), dict(reserved=1)], ids=str)
def test_dropout_parameters_are_refused(g, kw):
    assert g.lib().gpic_dropout(_drop(g, **kw), *AT[:4], None) == 1


def test_dropout_buffers_are_refused(g):
    L, p, a = g.lib(), _drop(g), AT
    assert L.gpic_dropout(None, *a[:4], None) == 1
    assert L.gpic_dropout(p, None, *a[1:4], None) == 1
    assert L.gpic_dropout(p, *a[:3], None, None) == 1
    for i in range(4):
        bad = list(a[:4])
        bad[i] = ODD
        assert L.gpic_dropout(p, *bad, None) == 1
    assert L.gpic_dropout(p, a[0], a[1], None, C.c_void_p((1 << 40) + 2), None) == 1
    assert L.gpic_dropout(_drop(g, ldy=24), a[0], a[1], None, a[0], None) == 1
    assert L.gpic_dropout(_drop(g, ldr=24), a[0], a[1], None, a[1], None) == 1
    assert L.gpic_dropout(p, a[0], a[1], a[2], a[2], None) == 1                 # Y over the step


@pytest.mark.parametrize("kw", SIDES + [dict(k=0), dict(k=2 ** 20 + 1), dict(rows=0),
                                        dict(rows=2 ** 31), dict(ldt=15), dict(ldy=15),
                                        dict(ldt=2 ** 22 + 1), dict(scale=NAN), dict(scale=INF),
                                        dict(id_bytes=2), dict(accumulate=2)], ids=str)
def test_embedding_parameters_are_refused(g, kw):
    L, p = g.lib(), _embed(g, **kw)
    assert L.gpic_embedding(p, *AT[:3], None) == 1
    assert L.gpic_embedding_backward(p, *AT[:3], *WS, None) == 1
    assert L.gpic_embedding_workspace_bytes(p) == 0


def test_embedding_buffers_are_refused(g):
    L, p, a = g.lib(), _embed(g), AT
    four = C.c_void_p((1 << 40) + 4)
    assert L.gpic_embedding(None, *a[:3], None) == 1
    for i in range(3):
        bad = list(a[:3])
        bad[i] = None
        assert L.gpic_embedding(p, *bad, None) == 1
        assert L.gpic_embedding_backward(p, *bad, *WS, None) == 1
        bad[i] = ODD
        assert L.gpic_embedding(p, *bad, None) == 1
        assert L.gpic_embedding_backward(p, *bad, *WS, None) == 1
    assert L.gpic_embedding(p, four, a[1], a[2], None) == 1                    # 64-bit ids
    assert L.gpic_embedding(p, a[0], a[1], a[1], None) == 1
    assert L.gpic_embedding(p, a[0], a[1], a[0], None) == 1
    assert L.gpic_embedding_backward(p, a[0], a[1], a[0], *WS, None) == 1
    assert L.gpic_embedding_workspace_bytes(p) == 0                           # few ids
    big = dict(n=5000)
    need = L.gpic_embedding_workspace_bytes(_embed(g, **big))
    assert need >= 5000 * 24 + 31 * 4
    assert L.gpic_embedding_backward(_embed(g, **big), *a[:3], WS[0], need - 1, None) == 2


@pytest.mark.parametrize("kw", SIDES + [dict(k=0), dict(k=2 ** 20 + 1), dict(v=0),
                                        dict(v=2 ** 20 + 1), dict(ldx=15), dict(ldw=15),
                                        dict(ldw=2 ** 22 + 1), dict(id_bytes=1), dict(aligned16=2),
                                        dict(reserved=3)], ids=str)
def test_loss_parameters_are_refused(g, kw):
    L, p = g.lib(), _loss(g, **kw)
    assert L.gpic_cross_entropy(p, *AT[:6], *WS, None) == 1
    assert L.gpic_cross_entropy_backward(p, *AT[:10], *WS, None) == 1
    assert L.gpic_cross_entropy_workspace_bytes(0, p) == 0
    assert L.gpic_cross_entropy_workspace_bytes(1, p) == 0


def test_loss_buffers_are_refused(g):
    L, p, a = g.lib(), _loss(g), AT
    assert L.gpic_cross_entropy(None, *a[:6], *WS, None) == 1
    for i in (0, 1, 3, 4):
        bad = list(a[:6])
        bad[i] = None
        assert L.gpic_cross_entropy(p, *bad, *WS, None) == 1
    for i in range(6):
        bad = list(a[:6])
        bad[i] = ODD
        assert L.gpic_cross_entropy(p, *bad, *WS, None) == 1
    assert L.gpic_cross_entropy(p, C.c_void_p((1 << 40) + 8), *a[1:6], *WS, None) == 1  # aligned16
    assert L.gpic_cross_entropy(p, *a[:5], a[4], *WS, None) == 1               # lse over loss
    assert L.gpic_cross_entropy(p, *a[:4], a[0], a[5], *WS, None) == 1
    for i in (0, 1, 2, 4, 5, 6):
        bad = list(a[:10])
        bad[i] = None
        assert L.gpic_cross_entropy_backward(p, *bad, *WS, None) == 1
    for i in range(10):
        bad = list(a[:10])
        bad[i] = ODD
        assert L.gpic_cross_entropy_backward(p, *bad, *WS, None) == 1
    assert L.gpic_cross_entropy_backward(p, *a[:7], a[1], a[8], a[9], *WS, None) == 1   # dX over X
    assert L.gpic_cross_entropy_backward(p, *a[:8], a[7], a[9], *WS, None) == 1         # dW over dX
    for back, call in ((0, lambda *w: L.gpic_cross_entropy(p, *a[:6], *w, None)),
                       (1, lambda *w: L.gpic_cross_entropy_backward(p, *a[:10], *w, None))):
        need = L.gpic_cross_entropy_workspace_bytes(back, p)
        assert need > 0
        assert call(WS[0], need - 1) == 2 and call(None, 0) == 2
        assert call(C.c_void_p(WS[0].value + 8), need) == 1
    assert L.gpic_cross_entropy_workspace_bytes(2, p) == 0


def test_loss_workspaces(g):
    """No logits: the forward call keeps 8 bytes a row and tile, the gradients
    a piece of up to 512 MB whatever the vocabulary."""
    L = g.lib()

    def size(back, **kw):
        w = dict(n=8192, k=512, ldx=512, ldw=512)
        w.update(kw)
        return L.gpic_cross_entropy_workspace_bytes(back, _loss(g, **w))

    for v in (50000, 100000, 1 << 20):
        assert size(0, v=v) <= 8192 * 8 * (v // 64 + 2) + 8192 * 16
        # dZ, dX's sum, X under its shares, sums of the bias, parts of split tiles
        assert size(1, v=v) <= (512 << 20) + 8192 * 512 * 6 + 8192 * 64 + 8192 // 32 * 32768 * 4 + \
            (64 << 20)
    assert size(0, v=50000, aligned16=0) >= size(0, v=50000) + (8192 + 50000) * 512 * 2


def test_too_many_workgroups_are_refused(g):
    L = g.lib()
    e = _embed(g, n=2 ** 31 - 1)
    assert L.gpic_embedding_backward(e, *AT[:3], *WS, None) == 5
    assert L.gpic_embedding_workspace_bytes(e) == 0
    p = _loss(g, n=2 ** 31 - 1, v=1 << 20)
    assert L.gpic_cross_entropy(p, *AT[:6], *WS, None) == 5
    assert L.gpic_cross_entropy_workspace_bytes(0, p) == 0


def test_the_binding_refuses_host_tensors(g):
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: g.gpic_layer_norm(x), lambda: g.gpic_dropout(x, 0.1, 1),
                 lambda: g.gpic_embedding(i, x), lambda: g.gpic_embedding_backward(x, i, 4),
                 lambda: g.gpic_cross_entropy(x, x, i),
                 lambda: g.gpic_cross_entropy_backward(x[:, 0], x, x, i, x[:, 0], x[:, 0]),
                 lambda: g.gpic_layer_norm_backward(x, x, None, x)):
        with pytest.raises(TypeError):
            call()
