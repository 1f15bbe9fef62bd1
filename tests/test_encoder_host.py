"""Host-side checks of the encoder operators' entry points (no GPU needed):
arguments are refused before any launch, workspaces grow with the sizes, and
the binding refuses tensors it cannot pass on."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    return g


def _layer(g, **kw):
    p = g.LayerParams(n=10, k=16, m=24, ldx=16, ldw=16, ldy=24, ldr=24, ldz=48, dtype=2,
                      activation=2, aligned16=1, reserved=0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_LAYERS = [dict(n=-1), dict(n=2 ** 31), dict(k=0), dict(k=2 ** 20 + 1), dict(m=0),
              dict(m=2 ** 20 + 1), dict(ldx=15), dict(ldw=15), dict(ldy=23), dict(ldx=2 ** 22 + 1),
              dict(ldw=2 ** 22 + 1), dict(dtype=3), dict(dtype=-1), dict(activation=4),
              dict(activation=-1), dict(aligned16=2), dict(reserved=1)]


@pytest.mark.parametrize("kw", BAD_LAYERS, ids=str)
def test_layer_parameters_are_refused(g, kw):
    L, d = g.lib(), C.c_void_p(4096)            # never dereferenced
    p = C.byref(_layer(g, **kw))
    ws = (d, 1 << 40)
    assert L.gpic_linear(p, d, d, d, d, d, d, *ws, None) == 1
    assert L.gpic_linear_backward(p, d, d, d, d, d, d, d, *ws, None) == 1
    assert L.gpic_gated(p, d, d, d, d, *ws, None) == 1
    assert L.gpic_gated_backward(p, d, d, d, d, d, d, *ws, None) == 1
    for op in range(4):
        assert L.gpic_layer_workspace_bytes(op, p) == 0


def test_layer_buffers_are_refused(g):
    L, d, odd, a8 = g.lib(), C.c_void_p(4096), C.c_void_p(4097), C.c_void_p(4104)
    ws = (d, 1 << 40)
    p = C.byref(_layer(g))
    assert L.gpic_linear(None, d, d, d, d, d, d, *ws, None) == 1
    assert L.gpic_linear(p, None, d, None, None, d, None, *ws, None) == 1
    assert L.gpic_linear(p, d, None, None, None, d, None, *ws, None) == 1
    assert L.gpic_linear(p, d, d, None, None, None, None, *ws, None) == 1
    assert L.gpic_linear(p, a8, d, None, None, d, None, *ws, None) == 1      # aligned16 promised
    assert L.gpic_linear(p, d, d, odd, None, d, None, *ws, None) == 1
    assert L.gpic_linear(p, d, d, None, odd, d, None, *ws, None) == 1
    assert L.gpic_linear(p, d, d, None, None, d, odd, *ws, None) == 1
    assert L.gpic_linear(C.byref(_layer(g, ldr=23)), d, d, None, d, d, None, *ws, None) == 1
    assert L.gpic_linear(C.byref(_layer(g, ldz=23)), d, d, None, None, d, d, *ws, None) == 1
    assert b"ldz" in L.gpic_last_error()
    assert L.gpic_linear_backward(p, d, d, d, None, d, d, d, *ws, None) == 1   # gelu needs Z
    assert L.gpic_linear_backward(p, None, d, d, d, d, d, d, *ws, None) == 1
    assert L.gpic_linear_backward(p, d, None, d, d, d, d, d, *ws, None) == 1   # dW needs X
    assert L.gpic_linear_backward(p, d, d, None, d, d, d, d, *ws, None) == 1   # dX needs W
    assert L.gpic_gated(C.byref(_layer(g, ldz=47)), d, d, d, d, *ws, None) == 1
    assert L.gpic_gated(C.byref(_layer(g, m=2 ** 19 + 1, ldy=2 ** 20)), d, d, d, d, *ws, None) == 1
    assert L.gpic_gated_backward(p, d, d, d, None, d, d, *ws, None) == 1
    # few rows are read as they lie; more rows of float32 need packed copies
    assert L.gpic_layer_workspace_bytes(0, C.byref(_layer(g, dtype=0))) == 0
    f = _layer(g, dtype=0, n=10000, k=80, ldx=80, ldw=80)
    need = L.gpic_layer_workspace_bytes(0, C.byref(f))
    assert need > 0
    assert L.gpic_linear(C.byref(f), d, d, None, None, d, None, d, need - 1, None) == 2
    assert L.gpic_linear(C.byref(f), d, d, None, None, d, None, None, 0, None) == 2
    assert L.gpic_linear(C.byref(f), d, d, None, None, d, None, C.c_void_p(4112), need, None) == 1


def test_gated_offsets_are_limited(g):
    """One half of the gated weights must be reachable with 32-bit offsets."""
    L, d = g.lib(), C.c_void_p(4096)
    p = _layer(g, m=2 ** 19, ldy=2 ** 19, k=8192, ldx=8192, ldw=8192, ldz=2 ** 20)
    assert L.gpic_gated(C.byref(p), d, d, d, d, d, 1 << 40, None) == 5


def test_layer_workspaces(g):
    L = g.lib()
    for op in range(4):
        for dt in range(3):
            def size(n, **kw):
                w = dict(k=80, ldx=80, ldw=80, ldy=24, ldz=48)
                w.update(kw)
                return L.gpic_layer_workspace_bytes(op, C.byref(_layer(g, n=n, dtype=dt, **w)))
            if dt == 0 or op in (1, 3):
                assert 0 < size(10 ** 5) < size(10 ** 6) and size(10 ** 6) >= 10 ** 6 * 2 * 16
                assert size(1000) == 0                           # small: read as they lie
            else:
                assert size(1000) == size(10 ** 6) == 0          # read as they lie
            # operands that may start anywhere are copied
            assert size(10 ** 6, aligned16=0) >= 10 ** 6 * 2 * 16
            # short contractions are read as they lie: float32 up to 32 values
            # or 2^23 results, 16 bits up to 64
            if op in (0, 2):
                assert size(10 ** 6, k=32, aligned16=0) == 0
                assert size(2 ** 23 // 48, k=64, aligned16=0) == 0
                assert (size(10 ** 6, k=64) > 0) == (dt == 0)
    assert L.gpic_layer_workspace_bytes(4, C.byref(_layer(g))) == 0
    assert L.gpic_layer_workspace_bytes(0, None) == 0


def _polar(g, **kw):
    p = g.PolarParams(batch=2, m=64, n=96, dtype=0, steps=5, a=3.4445, b=-4.775, c=2.0315,
                      reserved=0, eps=1e-7)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(batch=65536), dict(m=0), dict(n=0),
                                dict(m=2 ** 20 + 1), dict(n=2 ** 20 + 1), dict(dtype=3),
                                dict(steps=0), dict(steps=65), dict(a=17.0), dict(b=float("nan")),
                                dict(c=float("inf")), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(reserved=1)], ids=str)
def test_polar_parameters_are_refused(g, kw):
    L, d = g.lib(), C.c_void_p(4096)
    p = C.byref(_polar(g, **kw))
    h = g.MuonParams(lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, nesterov=1, reserved=0)
    assert L.gpic_orthogonalize(p, d, d, d, 1 << 40, None) == 1
    assert L.gpic_muon_step(p, C.byref(h), d, d, d, d, 1 << 40, None) == 1
    assert L.gpic_polar_workspace_bytes(p) == 0


def test_polar_buffers_and_step_are_refused(g):
    L, d, odd = g.lib(), C.c_void_p(4096), C.c_void_p(4098)
    assert L.gpic_polar_workspace_bytes(C.byref(_polar(g))) == 0      # fits a workgroup
    p = C.byref(_polar(g, m=640, n=960))
    need = L.gpic_polar_workspace_bytes(p)
    assert need >= 2 * 640 * 960 * 4 * 2
    assert L.gpic_orthogonalize(p, None, d, d, need, None) == 1
    assert L.gpic_orthogonalize(p, d, None, d, need, None) == 1
    assert L.gpic_orthogonalize(p, odd, d, d, need, None) == 1
    assert L.gpic_orthogonalize(p, d, d, d, need - 1, None) == 2
    ok = dict(lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, nesterov=1, reserved=0)
    for bad in (dict(lr=float("nan")), dict(momentum=float("inf")), dict(weight_decay=float("nan")),
                dict(scale=float("inf")), dict(nesterov=2), dict(reserved=1)):
        h = g.MuonParams(**{**ok, **bad})
        assert L.gpic_muon_step(p, C.byref(h), d, d, d, d, need, None) == 1
    h = C.byref(g.MuonParams(**ok))
    assert L.gpic_muon_step(p, None, d, d, d, d, need, None) == 1
    assert L.gpic_muon_step(p, h, None, d, d, d, need, None) == 1
    assert L.gpic_muon_step(p, h, d, d, odd, d, need, None) == 1
    assert L.gpic_muon_step(p, h, d, d, d, d, 0, None) == 2


def test_binding_refuses_host_tensors(g):
    x = torch.zeros((4, 8))
    for call in (lambda: g.gpic_linear(x, x), lambda: g.gpic_gated(x, x),
                 lambda: g.gpic_linear_backward(x, x, x), lambda: g.gpic_orthogonalize(x),
                 lambda: g.gpic_gated_backward(x, x, x, x),
                 lambda: g.gpic_muon_step(x, x, x, 0.1)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("steps, a, b, c, ok", [
    (64, 3.4445, -4.775, 2.0315, True), (64, 15 / 8, -10 / 8, 3 / 8, True), (64, 1.5, -0.5, 0.0, True),
    (1, 16.0, 0.0, 0.0, True), (1, 16.0, -16.0, 16.0, True), (64, 0.0, 0.0, 0.0, True),
    # singular values that grow from step to step: 1.9^3 = 6.9, 1.9^4 = 13
    (4, 1.9, 0.0, 0.0, True), (5, 1.9, 0.0, 0.0, False), (2, 16.0, 0.0, 0.0, False),
    # below 4 after a step, but b x^2 + c x^4 is not there
    (1, 1.0, 15.0, -15.0, True), (2, 1.0, 15.0, -15.0, False),
    # the largest value is inside the interval: 2.3 for a polynomial that is 0 at 1
    (2, 6.0, -6.0, 0.0, True), (3, 6.0, -6.0, 0.0, False)], ids=str)
def test_polynomials_that_leave_the_halves_are_refused(g, steps, a, b, c, ok):
    """Against the same bound by dense sampling; a refused step advances nothing."""
    import numpy as np
    top, fits = 1.0, True
    a32, b32, c32 = (float(np.float32(v)) for v in (a, b, c))
    for _ in range(steps):
        s = np.linspace(0.0, top, 200001)
        fits = fits and top * top <= 60 and float(np.abs(b32 * s ** 2 + c32 * s ** 4).max()) <= 60
        top = float(np.abs(a32 * s + b32 * s ** 3 + c32 * s ** 5).max()) * 257 / 256
    assert fits == ok
    L, d = g.lib(), C.c_void_p(4096)            # never dereferenced: refused, or no workspace
    p = C.byref(_polar(g, steps=steps, a=a, b=b, c=c, m=640, n=960))
    h = C.byref(g.MuonParams(lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, nesterov=1,
                             reserved=0))
    assert (L.gpic_polar_workspace_bytes(p) > 0) == ok
    assert L.gpic_orthogonalize(p, d, d, None, 0, None) == (2 if ok else 1)
    assert L.gpic_muon_step(p, h, d, d, d, None, 0, None) == (2 if ok else 1)
    assert ok or b"singular values" in L.gpic_last_error()


def test_rows_up_to_the_limit_of_a_launch(g):
    """A launch has fewer than 2^32 threads: narrow layers of 2^30 rows and
    more take larger tiles, and the last 127 row counts are refused before
    anything runs."""
    L, d = g.lib(), C.c_void_p(4096)            # never dereferenced: no workspace is given
    for dt in range(3):
        for n, ok in ((2 ** 30, True), (2 ** 31 - 128, True), (2 ** 31 - 127, False),
                      (2 ** 31 - 1, False)):
            p = _layer(g, n=n, k=80, m=8, ldx=80, ldw=80, ldy=8, ldr=8, ldz=16, dtype=dt,
                       aligned16=0)
            ref = C.byref(p)
            for op in range(4):
                assert (L.gpic_layer_workspace_bytes(op, ref) > 0) == ok
            want = 2 if ok else 5
            assert L.gpic_linear(ref, d, d, None, None, d, d, None, 0, None) == want
            assert L.gpic_linear_backward(ref, d, d, d, d, d, d, d, None, 0, None) == want
            assert L.gpic_gated(ref, d, d, d, d, None, 0, None) == want
            assert L.gpic_gated_backward(ref, d, d, d, d, d, d, None, 0, None) == want
    # rows that are read as they lie have no such limit
    p = _layer(g, n=2 ** 31 - 1)
    assert L.gpic_layer_workspace_bytes(0, C.byref(p)) == 0


@pytest.mark.parametrize("ldz", [0, -7, 2 ** 40, 2 ** 62, -2 ** 63])
def test_a_pitch_that_is_not_used_changes_nothing(g, ldz):
    """ldz without a Z that is read: no part in the choice of a kernel."""
    L, d = g.lib(), C.c_void_p(4096)
    for n in (50, 5000):
        for dt in range(3):
            p = _layer(g, n=n, activation=0, dtype=dt, aligned16=0, ldz=ldz)
            q = _layer(g, n=n, activation=0, dtype=dt, aligned16=0)
            for op in (0, 1):
                assert L.gpic_layer_workspace_bytes(op, C.byref(p)) \
                    == L.gpic_layer_workspace_bytes(op, C.byref(q))
            # where Z is read the call refuses it, and there is no workspace for it
            p = _layer(g, n=n, dtype=dt, aligned16=0, ldz=ldz)
            assert L.gpic_layer_workspace_bytes(1, C.byref(p)) == 0
            assert L.gpic_layer_workspace_bytes(3, C.byref(p)) == 0
            assert L.gpic_linear_backward(C.byref(p), d, d, d, d, d, d, d, None, 0, None) == 1
            assert L.gpic_gated_backward(C.byref(p), d, d, d, d, d, d, None, 0, None) == 1


def _at(address):
    return C.c_void_p(address)                  # never dereferenced


def test_results_over_operands_are_refused(g):
    """Shared bytes are refused before any launch (what shares none is called
    with memory of its own in the tests on the GPU)."""
    L = g.lib()
    base, far = 1 << 30, 1 << 34

    def linear(Y, X=base, W=far, R=None, Z=None, ldx=16, ldy=24, ldr=24, n=10):
        p = _layer(g, n=n, ldx=ldx, ldy=ldy, ldr=ldr, ldz=24, aligned16=0)
        st = L.gpic_linear(C.byref(p), _at(X), _at(W), None, R and _at(R), _at(Y), Z and _at(Z),
                           None, 0, None)
        return st, L.gpic_last_error()

    for Y in (base, base + 2, base + 10 * 32 - 2, base - 10 * 48 + 2):
        assert linear(Y) == (1, b"Y overlaps X")
    assert linear(far + 24 * 32 - 2) == (1, b"Y overlaps W")
    assert linear(2 * far, R=2 * far + 2)[1] == b"Y overlaps the residual"
    assert linear(2 * far, R=2 * far, ldr=26)[1] == b"Y overlaps the residual"
    assert linear(2 * far, Z=2 * far + 100)[1] == b"Z overlaps Y"
    # one table of 48 columns, X in 0 .. 15: Y a column early, Y past its row's end
    assert linear(base + 30, ldx=48, ldy=48) == (1, b"Y overlaps X")
    assert linear(base + 2 * (48 * 4 + 25), ldx=48, ldy=48) == (1, b"Y overlaps X")
    # pitches that differ: rows of Y in the gaps of a table of X but the last
    assert linear(base + 2 * 16, ldx=100, ldy=199, n=10) == (1, b"Y overlaps X")
    assert linear(base + 2 * 90, ldx=100, n=2, ldy=24) == (1, b"Y overlaps X")


def test_gradients_and_steps_over_operands_are_refused(g):
    L, f = g.lib(), 1 << 34
    p = C.byref(_layer(g, n=10, aligned16=0, ldz=48))
    a = [_at(f * i) for i in range(1, 9)]
    for bad in (dict(dX=a[0]), dict(dX=a[1]), dict(dX=a[2]), dict(dX=a[3]), dict(dW=a[4]),
                dict(db=a[5]), dict(dW=a[0])):
        o = {**dict(dX=a[4], dW=a[5], db=a[6]), **bad}
        assert L.gpic_linear_backward(p, a[0], a[1], a[2], a[3], o["dX"], o["dW"], o["db"], None, 0,
                                      None) == 1
        assert b"overlaps" in L.gpic_last_error()
        if "db" not in bad:
            assert L.gpic_gated_backward(p, a[0], a[1], a[2], a[3], o["dX"], o["dW"], None, 0,
                                         None) == 1
    for H, Z in ((a[0], a[2]), (a[1], a[2]), (a[2], a[2]), (a[2], a[0])):
        assert L.gpic_gated(p, a[0], a[1], H, Z, None, 0, None) == 1
    q = C.byref(_polar(g))
    h = C.byref(g.MuonParams(lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, nesterov=1,
                             reserved=0))
    assert L.gpic_orthogonalize(q, a[0], _at(f + 4), None, 0, None) == 1
    for W, G, M in ((a[0], a[1], a[1]), (a[0], a[1], a[0]),
                    (a[0], _at(f + 64), a[1])):
        assert L.gpic_muon_step(q, h, W, G, M, None, 0, None) == 1
