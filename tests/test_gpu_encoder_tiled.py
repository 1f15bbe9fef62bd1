"""The layers where they go through packed operands and the tiled product:
the same questions as test_gpu_encoder.py asks of small calls (views,
alignment, in-place results, non-finite rows, no rows, workspaces, streams,
graphs, offsets past 32 bits), at sizes that the one-launch kernels do not
take.  `_tiled` asserts that, so that a change of the rules that choose a
kernel cannot take the sizes away.  Tolerances as there."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_encoder import DEV, E, T, U, _act, _close, _product_error, _randn  # noqa: E402

N, K, M = 2100, 100, 140


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return g


def _tiled(g, op, n, k, m, dtype):
    """Operands that may start anywhere are copied on the tiled path, and
    read as they lie on the others: there is a workspace on that path only."""
    rows = 2 * m if "gated" in op else m
    p = g.LayerParams(n=n, k=k, m=m, ldx=k, ldw=k, ldy=m, ldr=m, ldz=rows,
                      dtype=g.DTYPES[T[dtype]], activation=2, aligned16=0, reserved=0)
    assert g.lib().gpic_layer_workspace_bytes(g.LAYER_OP[op], C.byref(p)) > 0, (op, n, k, m)


def _all_tiled(g, n, k, m, dtype):
    for op in g.LAYER_OP:
        _tiled(g, op, n, k, m, dtype)


def _wide(t, pad, first):
    """t as columns of a wider table of NaN, with a row of it before and after."""
    big = torch.full((t.shape[0] + 2, t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    v = big[1:1 + t.shape[0], first:first + t.shape[1]]
    v.copy_(t)
    return v


def _late(t):
    """t in a buffer of NaN that starts one value before it."""
    flat = torch.full((t.numel() + 1,), float("nan"), dtype=t.dtype, device=DEV)
    v = flat[1:].view(t.shape)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", [(2100, 96, 1800), (2101, 101, 137)], ids=str)
def test_every_activation(g, shape, dtype):
    n, k, m = shape
    _all_tiled(g, n, k, m, dtype)
    for act in ("none", "relu", "gelu", "silu"):
        print(f"tiled n={n} k={k} m={m} {dtype} {act}", flush=True)
        X, W = _randn((n, k), dtype, 1), _randn((2 * m, k), dtype, 2, k ** -0.5)
        b, R, dY = _randn((m,), dtype, 3), _randn((n, m), dtype, 4), _randn((n, m), dtype, 5, 0.01)
        x, w, dy = X.double(), W.double(), dY.double()
        Y, Z = g.gpic_linear(X, W[:m], b, act, R, want_pre=True)
        z = x @ w[:m].t() + b.double()
        pe = _product_error(x, w[:m], dtype) + 2 * E * z.abs()
        a = _act(z, act)[0]
        ref = a + R.double()
        _close(Z, z, pe, dtype, "Z")
        _close(Y, ref, 1.13 * pe + 2e-7 * z.abs() + 4 * E * (a.abs() + ref.abs()), dtype, "Y")
        gr = g.gpic_linear_backward(dY, X, W[:m], Z if act != "none" else None, act)
        zz = Z.double()
        dz = dy * _act(zz, act)[1]
        off = (U[dtype] if act != "none" and dtype != "f32" else 0.0) * dz.abs() \
            + 1e-6 * dy.abs() * (1 + zz.abs() * (act != "none"))
        _close(gr.dX, dz @ w[:m], off @ w[:m].abs() + _product_error(dz, w[:m].t(), dtype), dtype,
               "dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _product_error(dz.t(), x.t(), dtype), dtype,
               "dW")
        _close(gr.db, dz.sum(0), (1e-6 + 70 * E) * (dy.abs() * (1 + zz.abs())).sum(0), dtype, "db")

        H, Z = g.gpic_gated(X, W, act, want_pre=True)
        z = x @ w.t()
        pe = _product_error(x, w, dtype)
        _close(Z, z, pe, dtype, "gated Z")
        a, u = _act(z[:, :m], act)[0], z[:, m:]
        _close(H, a * u, (1.13 * pe[:, :m] + 2e-7 * z[:, :m].abs()) * (u.abs() + pe[:, m:])
               + a.abs() * pe[:, m:] + 4 * E * (a * u).abs(), dtype, "H")
        gr = g.gpic_gated_backward(dY, X, W, Z, act)
        zz = Z.double()
        a, da = _act(zz[:, :m], act)
        dz = torch.cat([dy * zz[:, m:] * da, dy * a], 1)
        off = (U[dtype] if dtype != "f32" else 0.0) * dz.abs() + 1e-6 * torch.cat(
            [(dy * zz[:, m:]).abs() * (1 + zz[:, :m].abs()), (dy * zz[:, :m]).abs()], 1)
        _close(gr.dX, dz @ w, off @ w.abs() + _product_error(dz, w.t(), dtype), dtype, "gated dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _product_error(dz.t(), x.t(), dtype), dtype,
               "gated dW")


@pytest.mark.parametrize("dtype", list(T))
def test_views_and_alignment(g, dtype):
    """Column and row slices, transposed operands, buffers that start one
    value late: the same bits as the contiguous tensors."""
    n, k, m = N, 104, 136
    _all_tiled(g, n, k, m, dtype)
    X, W, b, R = (_randn(s, dtype, i) for i, s in enumerate(((n, k), (2 * m, k), (m,), (n, m))))
    W *= 0.1
    Y, Z = g.gpic_linear(X, W[:m], b, "gelu", R, want_pre=True)
    gr = g.gpic_linear_backward(R, X, W[:m], Z, "gelu")
    plain = g.gpic_linear_backward(R, X, W[:m])
    H, ZZ = g.gpic_gated(X, W, want_pre=True)
    gg = g.gpic_gated_backward(R, X, W, ZZ)
    for i, make in enumerate((lambda t: _wide(t, 24, 8), lambda t: _wide(t, 5, 3), _late,
                              lambda t: t.t().contiguous().t())):
        print(f"views {dtype} {i}", flush=True)
        x, w, w2, r, z, zz = (make(t) for t in (X, W[:m], W, R, Z, ZZ))
        out = torch.empty_like(R)
        assert torch.equal(g.gpic_linear(x, w, _late(b[None])[0], "gelu", r, Y=out), Y)
        for got, want in ((g.gpic_linear_backward(r, x, w, z, "gelu"), gr),
                          (g.gpic_linear_backward(r, x, w), plain),
                          (g.gpic_gated_backward(r, x, w2, zz), gg)):
            assert torch.equal(got.dX, want.dX) and torch.equal(got.dW, want.dW)
            assert want.db is None or torch.equal(got.db, want.db)
        assert torch.equal(g.gpic_gated(x, w2), H)
    # results in place of a strided residual, and among other columns
    out = _wide(R, 7, 3)
    table = out._base.clone()
    assert torch.equal(g.gpic_linear(X, W[:m], b, "gelu", out, Y=out), Y)
    after = out._base.clone()
    after[1:1 + n, 3:3 + m] = table[1:1 + n, 3:3 + m]
    assert torch.equal(after.isnan(), table.isnan())          # nothing beside it was written
    out = _wide(torch.zeros_like(H), 3, 1)
    assert torch.equal(g.gpic_gated(X, W, H=out), H)
    assert bool(out._base[:, 0].isnan().all()) and bool(out._base[:, m + 1:].isnan().all())
    # gradients one at a time
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        one = g.gpic_linear_backward(R, X, W[:m], Z, "gelu", *want)
        for name, asked in zip(("dX", "dW", "db"), want):
            got = getattr(one, name)
            assert torch.equal(got, getattr(gr, name)) if asked else got is None


@pytest.mark.parametrize("dtype", list(T))
def test_no_rows(g, dtype):
    k, m = K, 2100
    _tiled(g, "linear_backward", 0, k, m, dtype)
    _tiled(g, "gated_backward", 0, k, m, dtype)
    X, W = _randn((0, k), dtype, 1), _randn((2 * m, k), dtype, 2)
    Y, Z = g.gpic_linear(X, W[:m], None, "gelu", want_pre=True)
    gr = g.gpic_linear_backward(Y, X, W[:m], Z, "gelu")
    assert gr.dX.shape == (0, k) and gr.dW.shape == (m, k)
    assert not bool(gr.dW.any()) and not bool(gr.db.any())
    H, Z = g.gpic_gated(X, W, want_pre=True)
    gr = g.gpic_gated_backward(H, X, W, Z)
    assert gr.dW.shape == (2 * m, k) and not bool(gr.dW.any())


@pytest.mark.parametrize("dtype", list(T))
def test_non_finite_values_stay_in_their_rows(g, dtype):
    _all_tiled(g, N, K, M, dtype)
    X, W = _randn((N, K), dtype, 1), _randn((2 * M, K), dtype, 2, 0.1)
    dY = _randn((N, M), dtype, 3, 0.1)
    clean, pre = g.gpic_linear(X, W[:M], None, "gelu", want_pre=True)
    H, ZZ = g.gpic_gated(X, W, want_pre=True)
    back = g.gpic_linear_backward(dY, X, W[:M], pre, "gelu")
    keep = torch.arange(N, device=DEV) != 1
    cols = torch.arange(K, device=DEV) != 37
    outs = torch.arange(M, device=DEV) != 5
    for bad in (float("nan"), float("inf"), -float("inf")):
        print(f"non-finite {dtype} {bad}", flush=True)
        x = X.clone()
        x[1, 37] = bad
        y = g.gpic_linear(x, W[:M])
        assert not bool(torch.isfinite(y[1]).any()) and bool(torch.isfinite(y[keep]).all())
        # the other rows keep their bits
        assert torch.equal(g.gpic_linear(x, W[:M], None, "gelu")[keep], clean[keep])
        assert torch.equal(g.gpic_gated(x, W)[keep], H[keep])
        gr = g.gpic_linear_backward(dY, x, W[:M], pre, "gelu")
        assert torch.equal(gr.dX, back.dX) and torch.equal(gr.db, back.db)
        assert not bool(torch.isfinite(gr.dW[:, 37]).any())
        assert torch.equal(gr.dW[:, cols], back.dW[:, cols])
        # a weight: its column of the result
        w = W.clone()
        w[5, 37] = bad
        y = g.gpic_linear(X, w[:M], None, "gelu")
        assert torch.equal(y[:, outs], clean[:, outs])
        assert torch.equal(g.gpic_gated(X, w)[:, outs], H[:, outs])
        gr = g.gpic_linear_backward(dY, X, w[:M], pre, "gelu")
        assert not bool(torch.isfinite(gr.dX[:, 37]).any())
        assert torch.equal(gr.dX[:, cols], back.dX[:, cols]) and torch.equal(gr.dW, back.dW)
        # an entry of the gradient: its row of dX, its row of dW
        dy = dY.clone()
        dy[1, 5] = bad
        gr = g.gpic_linear_backward(dy, X, W[:M], pre, "gelu")
        assert torch.equal(gr.dX[keep], back.dX[keep]) and torch.equal(gr.dW[outs], back.dW[outs])
        assert not bool(torch.isfinite(gr.dX[1]).any() | torch.isfinite(gr.dW[5]).any())
        assert torch.equal(gr.db[outs], back.db[outs]) and not bool(torch.isfinite(gr.db[5]))


def test_infinite_and_large_arguments(g):
    """Z of a wide layer at large arguments: activations at their limits."""
    z = torch.tensor([0.0, 5.0, -5.0, 13.9, -13.9, 14.1, -14.1, 90.0, -90.0, 120.0, -120.0, 1e4,
                      -1e4], device=DEV)
    X = torch.zeros((N, K), device=DEV)
    X[:, 0] = z.repeat(-(-N // len(z)))[:N]
    W = torch.zeros((M, K), device=DEV)
    W[:, 0] = 1.0
    _tiled(g, "linear", N, K, M, "f32")
    ref = X[:, :1].double().expand(N, M)
    for act in ("relu", "gelu", "silu"):
        a = _act(ref, act)[0]
        y = g.gpic_linear(X, W, None, act).double()
        tol = 3e-7 * (a.abs() + ref.abs().clamp(max=20)) + 2.0 ** -21 * ref.abs() * (a != 0)
        assert bool(((y - a).abs() <= tol).all()), act


def _everything(g, dtype, X=None):
    n, k, m = N, K, M
    X = _randn((n, k), dtype, 1) if X is None else X
    W, V = _randn((m, k), dtype, 2, 0.2), _randn((k, m), dtype, 3, 0.1)
    W2 = _randn((2 * m, k), dtype, 4, 0.2)
    Y, Z = g.gpic_linear(X, W, _randn((m,), dtype, 5), "gelu", want_pre=True)
    out = g.gpic_linear(Y, V, None, "none", X)
    gr = g.gpic_linear_backward(Y, X, W, Z, "gelu")
    H, ZZ = g.gpic_gated(X, W2, want_pre=True)
    gg = g.gpic_gated_backward(H, X, W2, ZZ)
    lin = g.gpic_linear_backward(Y, X, W)
    O = g.gpic_orthogonalize(gg.dW)
    mom, weights = torch.ones_like(W2, dtype=torch.float32), W2.clone()
    g.gpic_muon_step(weights, gg.dW, mom, 0.1)
    return [Y, Z, out, gr.dX, gr.dW, gr.db, H, ZZ, gg.dX, gg.dW, lin.dX, lin.dW, lin.db, O,
            weights, mom]


@pytest.mark.parametrize("dtype", list(T))
def test_results_do_not_depend_on_the_buffers(g, monkeypatch, dtype):
    from gpu_helpers import Filled
    _all_tiled(g, N, K, M, dtype)
    runs = []
    for x in (0.0, 1e300):
        print(f"scratch {x} {dtype}", flush=True)
        with monkeypatch.context() as mp:
            mp.setattr(g, "torch", Filled(x))
            runs.append(_everything(g, dtype))
        torch.cuda.synchronize()
    for a, b in zip(*runs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", list(T))
def test_another_stream_and_graph_replays(g, dtype):
    eager = [t.clone() for t in _everything(g, dtype)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        on = _everything(g, dtype)
    s.synchronize()
    for a, b in zip(on, eager):
        assert torch.equal(a, b)
    X = _randn((N, K), dtype, 1)
    W, W2 = _randn((M, K), dtype, 2, 0.2), _randn((2 * M, K), dtype, 4, 0.2)

    def step():
        Y, Z = g.gpic_linear(X, W, None, "gelu", want_pre=True)
        gr = g.gpic_linear_backward(Y, X, W, Z, "gelu")
        H, ZZ = g.gpic_gated(X, W2, want_pre=True)
        return [Y, gr.dX, gr.dW, gr.db, H, g.gpic_gated_backward(H, X, W2, ZZ).dW,
                g.gpic_orthogonalize(gr.dW)]

    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step()
    for i in range(4):
        X.copy_(_randn((N, K), dtype, 20 + i))
        want = step()
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_offsets_beyond_32_bits(g):
    """n m > 2^32 values of Y, Z and the residual through the tiles."""
    n, k, m = 525000, 72, 8200
    _tiled(g, "linear", n, k, m, "bf16")
    print(f"linear n={n} k={k} m={m} ({n * m} values)", flush=True)
    X, W, b = _randn((n, k), "bf16", 1), _randn((m, k), "bf16", 2, k ** -0.5), _randn((m,), "bf16", 3)
    R = torch.zeros((n, m), dtype=torch.bfloat16, device=DEV)
    rows = sorted({r for p in range(30, 33) for d in (-1, 0, 1) for r in [2 ** p // m + d] if r < n}
                  | {0, 1, n - 2, n - 1})
    R[rows] = _randn((len(rows), m), "bf16", 4)
    Y, Z = g.gpic_linear(X, W, b, "gelu", R, want_pre=True)
    z = X[rows].double() @ W.double().t() + b.double()
    pe = _product_error(X[rows].double(), W.double(), "bf16") + 2 * E * z.abs()
    a = _act(z, "gelu")[0]
    ref = a + R[rows].double()
    _close(Z[rows], z, pe, "bf16", "Z")
    _close(Y[rows], ref, 1.13 * pe + 2e-7 * z.abs() + 4 * E * (a.abs() + ref.abs()), "bf16", "Y")
    # every row was written: none is left at what the allocator held
    assert bool(torch.isfinite(Y.view(-1)[::4097]).all())


@pytest.mark.parametrize("x, w", [(1e34, 1e-30), (1e-30, 1e34), (1e-36, 1e36), (1e30, 1e-20)],
                         ids=str)
def test_magnitudes_at_the_ends_of_float32(g, x, w):
    """Operands whose powers of two, one after the other, would leave
    float32's range on the way to a result inside it."""
    X, W = _randn((N, K), "f32", 1) * x, _randn((2 * M, K), "f32", 2, 0.1) * w
    dY = _randn((N, M), "f32", 3) * (1.0 if x < 1 else 1e-10)
    _all_tiled(g, N, K, M, "f32")
    a, b, d = X.double(), W.double(), dY.double()
    _close(g.gpic_linear(X, W[:M]), a @ b[:M].t(), _product_error(a, b[:M], "f32"), "f32", "Y")
    z = a @ b.t()
    pe = _product_error(a, b, "f32")
    H, Z = g.gpic_gated(X, W, "none", want_pre=True)
    _close(Z, z, pe, "f32", "gated Z")
    _close(H, z[:, :M] * z[:, M:], pe[:, :M] * (z[:, M:].abs() + pe[:, M:])
           + z[:, :M].abs() * pe[:, M:] + 4 * E * (z[:, :M] * z[:, M:]).abs(), "f32", "H")
    gr = g.gpic_linear_backward(dY, X, W[:M])
    _close(gr.dX, d @ b[:M], _product_error(d, b[:M].t(), "f32"), "f32", "dX")
    _close(gr.dW, d.t() @ a, _product_error(d.t(), a.t(), "f32"), "f32", "dW")


def _forward_bound(x, w, dtype="f32"):
    """As _product_error, with each row's own largest entry: what a row of X
    (of W) loses does not depend on the others."""
    b = ((x.shape[1] + 16) * E + 2.0 ** -21) * (x.abs() @ w.abs().t())
    return b + 2.0 ** -38 * (x.abs().amax(1)[:, None] * w.abs().sum(1)[None, :]
                             + w.abs().amax(1)[None, :] * x.abs().sum(1)[:, None])


@pytest.mark.parametrize("k", [K, 2500, 17000])
@pytest.mark.parametrize("size", [1e6, 1e13, 1e30])
def test_outlier_leaves_the_other_rows_alone(g, size, k):
    """One huge finite entry in X (in W): the other points (outputs) keep
    the bits that they have without it."""
    X, W = _randn((N, k), "f32", 1), _randn((2 * M, k), "f32", 2, k ** -0.5)
    for op in ("linear", "gated"):
        _tiled(g, op, N, k, M, "f32")
    Y, H = g.gpic_linear(X, W[:M]), g.gpic_gated(X, W)
    x, w = X.clone(), W.clone()
    x[17, 3] = size
    keep = torch.arange(N, device=DEV) != 17
    assert torch.equal(g.gpic_linear(x, W[:M])[keep], Y[keep])
    assert torch.equal(g.gpic_gated(x, W)[keep], H[keep])
    xd, wd = x.double(), W.double()
    _close(g.gpic_linear(x, W[:M]), xd @ wd[:M].t(), _forward_bound(xd, wd[:M]), "f32", "Y")
    w[17, 3] = size
    outs = torch.arange(M, device=DEV) != 17
    assert torch.equal(g.gpic_linear(X, w[:M])[:, outs], Y[:, outs])
    assert torch.equal(g.gpic_gated(X, w)[:, outs], H[:, outs])


@pytest.mark.parametrize("size", [1e6, 1e13, 1e28])
def test_outlier_leaves_the_other_gradients_alone(g, size):
    """One huge finite entry of dY, X, W or Z: the rows and columns of the
    gradients that do not sum over it keep their bits."""
    _all_tiled(g, N, K, M, "f32")
    X, W = _randn((N, K), "f32", 1), _randn((2 * M, K), "f32", 2, K ** -0.5)
    dY, Z = _randn((N, M), "f32", 3, 0.01), _randn((N, 2 * M), "f32", 4)
    rows = torch.arange(N, device=DEV) != 17
    ins = torch.arange(K, device=DEV) != 3
    outs = torch.arange(M, device=DEV) != 5
    both = torch.cat([outs, outs])

    def lin(dy, x, w):
        return g.gpic_linear_backward(dy, x, w[:M], Z[:, :M], "gelu")

    def gat(dy, x, w, z=Z):
        return g.gpic_gated_backward(dy, x, w, z)

    dy, x, w = dY.clone(), X.clone(), W.clone()
    dy[17, 5] = x[17, 3] = w[5, 3] = size
    for f, keep in ((lin, outs), (gat, both)):
        want = f(dY, X, W)
        got = f(dy, X, W)
        assert torch.equal(got.dX[rows], want.dX[rows])
        assert torch.equal(got.dW[keep], want.dW[keep])
        got = f(dY, x, W)
        assert torch.equal(got.dX, want.dX) and torch.equal(got.dW[:, ins], want.dW[:, ins])
        got = f(dY, X, w)
        assert torch.equal(got.dX[:, ins], want.dX[:, ins]) and torch.equal(got.dW, want.dW)
    # what does sum over it, to the bound of its own rows and columns
    dz = dy.double() * _act(Z[:, :M].double(), "gelu")[1]
    off = 1e-6 * dy.double().abs() * (1 + Z[:, :M].double().abs())
    xd, wd = x.double(), W[:M].double()
    gr = lin(dy, x, W)
    for got, ref, bound, what in (
            (gr.dX, dz @ wd, off @ wd.abs() + _forward_bound(dz, wd.t()), "dX"),
            (gr.dW, dz.t() @ xd, off.t() @ xd.abs() + _forward_bound(dz.t(), xd.t()), "dW")):
        over = ref.abs() > torch.finfo(torch.float32).max        # infinite in float32
        assert torch.equal(got[over], ref[over].float()), what
        _close(got[~over], ref[~over], bound[~over], "f32", what)
    # a point with a huge Z that no gradient reaches
    dy, z = dY.clone(), Z.clone()
    dy[17] = 0.0
    want = gat(dy, X, W)
    z[17] = size
    got = gat(dy, X, W, z)
    assert torch.equal(got.dX, want.dX) and torch.equal(got.dW, want.dW)


@pytest.mark.parametrize("shape", [(2100, 70, 270), (5000, 300, 66), (40, 1100, 4300),
                                   (70000, 33, 20)], ids=str)
def test_float32_gradients_of_uneven_shapes(g, shape):
    """Every strip and part of the maxima: a scale that is off by a row or a
    column shows where rows and columns differ by powers of two."""
    n, k, m = shape
    _tiled(g, "linear_backward", n, k, m, "f32")
    _tiled(g, "gated_backward", n, k, m, "f32")
    up = lambda s, i: 2.0 ** (_randn((s,), "f32", i, 8.0).round())  # noqa: E731
    X, W = _randn((n, k), "f32", 1) * up(k, 10), _randn((2 * m, k), "f32", 2, k ** -0.5) * up(k, 11)
    dY = _randn((n, m), "f32", 3) * up(n, 12)[:, None]
    Z = _randn((n, 2 * m), "f32", 4)
    x, w, dy, zz = X.double(), W.double(), dY.double(), Z.double()
    gr = g.gpic_linear_backward(dY, X, W[:m], Z[:, :m], "silu")
    dz = dy * _act(zz[:, :m], "silu")[1]
    off = 1e-6 * dy.abs() * (1 + zz[:, :m].abs())
    _close(gr.dX, dz @ w[:m], off @ w[:m].abs() + _forward_bound(dz, w[:m].t()), "f32", "dX")
    _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _forward_bound(dz.t(), x.t()), "f32", "dW")
    gr = g.gpic_gated_backward(dY, X, W, Z)
    a, da = _act(zz[:, :m], "silu")
    dz = torch.cat([dy * zz[:, m:] * da, dy * a], 1)
    off = 1e-6 * torch.cat([(dy * zz[:, m:]).abs() * (1 + zz[:, :m].abs()),
                            (dy * zz[:, :m]).abs()], 1)
    _close(gr.dX, dz @ w, off @ w.abs() + _forward_bound(dz, w.t()), "f32", "gated dX")
    _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _forward_bound(dz.t(), x.t()), "f32", "gated dW")


@pytest.mark.parametrize("size", [1e6, 1e13, 1e30])
def test_float16_gradients_beside_a_huge_z(g, size):
    """A point with a huge Z that no gradient reaches takes no bits of dZ:
    its power of two comes from dZ itself, not from dH's and Z's largest."""
    _tiled(g, "gated_backward", N, K, M, "f16")
    X, W = _randn((N, K), "f16", 1), _randn((2 * M, K), "f16", 2, K ** -0.5)
    dH, Z = _randn((N, M), "f16", 3, 1e-3), _randn((N, 2 * M), "f32", 4)
    dH[17] = 0.0
    want = g.gpic_gated_backward(dH, X, W, Z)
    z = Z.clone()
    z[17] = size
    got = g.gpic_gated_backward(dH, X, W, z)
    assert torch.equal(got.dX, want.dX) and torch.equal(got.dW, want.dW)


def test_more_than_2_30_rows(g):
    """The gradients of a narrow layer at 2^30 + 77 rows, more than a launch
    of 64 rows a workgroup would take: zero but for rows at the ends of tiles
    and of powers of two, so that every sum is short."""
    n, k, m = 2 ** 30 + 77, 8, 8
    _tiled(g, "linear_backward", n, k, m, "bf16")
    print(f"linear backward n={n} k={k} m={m}", flush=True)
    X = torch.zeros((n, k), dtype=torch.bfloat16, device=DEV)
    dY = torch.zeros((n, m), dtype=torch.bfloat16, device=DEV)
    rows = sorted({0, 1, 63, 64, 255, 256, n - 1, n - 2, 2 ** 30, 2 ** 30 - 1, 2 ** 29, 2 ** 29 - 1,
                   2 ** 28 + 3, 3 * 2 ** 28 + 129})
    X[rows], dY[rows] = _randn((len(rows), k), "bf16", 1), _randn((len(rows), m), "bf16", 2)
    W = _randn((m, k), "bf16", 3)
    gr = g.gpic_linear_backward(dY, X, W)
    x, d, w = X[rows].double(), dY[rows].double(), W.double()
    _close(gr.dX[rows], d @ w, _product_error(d, w.t(), "bf16"), "bf16", "dX")
    _close(gr.dW, d.t() @ x, _product_error(d.t(), x.t(), "bf16"), "bf16", "dW")
    _close(gr.db, d.sum(0), 70 * E * d.abs().sum(0), "bf16", "db")
    gr.dX[rows] = 0
    for part in gr.dX.split(2 ** 27):           # no other row has a gradient
        assert not bool(part.any())


@pytest.mark.parametrize("n", [7, N])
def test_rows_far_apart_are_copied(g, n):
    """Rows further apart than a pitch may be (2^22 values): the binding
    copies them, and refuses results that would lie so."""
    pitch, k, m = 2 ** 22 + 8, 100, 20
    far = torch.zeros((n - 1) * pitch + k, dtype=torch.bfloat16, device=DEV).as_strided(
        (n, k), (pitch, 1))
    X, W = _randn((n, k), "bf16", 1), _randn((m, k), "bf16", 2)
    far.copy_(X)
    assert torch.equal(g.gpic_linear(far, W), g.gpic_linear(X, W))
    dY = _randn((n, m), "bf16", 3)
    got, want = g.gpic_linear_backward(dY, far, W), g.gpic_linear_backward(dY, X, W)
    assert torch.equal(got.dX, want.dX) and torch.equal(got.dW, want.dW)
    with pytest.raises(ValueError, match="apart"):
        g.gpic_linear(X, W, Y=far[:, :m])


@pytest.mark.parametrize("n", [10, N])
def test_results_beside_their_operands(g, n):
    """X, the residual and Y as columns of one table, and of tables of two
    pitches in one buffer: no byte is shared, so the calls run.  Where bytes
    are shared, and the call would race, it is refused."""
    k, m = 100, 60
    X, W, R = _randn((n, k), "f32", 1), _randn((m, k), "f32", 2, 0.1), _randn((n, m), "f32", 3)
    Y, H = g.gpic_linear(X, W, None, "silu", R), g.gpic_gated(X, W)
    table = torch.full((n, k + 2 * m + 3), float("nan"), device=DEV)
    x, r, y = table[:, :k], table[:, k:k + m], table[:, k + m + 2:k + 2 * m + 2]
    x.copy_(X), r.copy_(R)
    assert torch.equal(g.gpic_linear(x, W, None, "silu", r, Y=y), Y) and torch.equal(x, X)
    assert bool(table[:, k + m:k + m + 2].isnan().all() & table[:, k + 2 * m + 2].isnan().all())
    assert torch.equal(g.gpic_linear(x, W, None, "silu", r, Y=r), Y)          # in place
    assert torch.equal(g.gpic_gated(x, W, H=y[:, :m // 2]), H) and torch.equal(x, X)
    # rows of Y in the gaps of every second row of X's table
    buf = torch.full((2 * n, 400), float("nan"), device=DEV)
    x, y = buf.view(-1).as_strided((n, k), (400, 1)), buf.view(-1).as_strided((n, m), (800, 1), 200)
    x.copy_(X)
    assert torch.equal(g.gpic_linear(x, W, Y=y), g.gpic_linear(X, W)) and torch.equal(x, X)
    V = _randn((k, k), "f32", 4)
    table = torch.zeros((n, k + m), device=DEV)
    table[:, :k] = X
    for call in (lambda: g.gpic_linear(X, V, Y=X), lambda: g.gpic_linear(X, V, Y=V[:n]) if n <= k else
                 g.gpic_linear(X, V, Y=X), lambda: g.gpic_linear(table[:, :k], W, Y=table[:, k - 1:-1]),
                 lambda: g.gpic_linear(X, W, None, "none", table[:, k:], Y=table[:, k - 1:-1]),
                 lambda: g.gpic_gated(X, V, H=X[:, :k // 2])):
        with pytest.raises(g.GpicError, match="overlaps"):
            call()
    G = _randn((65, 300), "f32", 5)
    O = g.gpic_orthogonalize(G)
    big = torch.zeros(65 * 300 + 4, device=DEV)
    big[:65 * 300] = G.view(-1)
    with pytest.raises(g.GpicError, match="overlaps"):
        g.gpic_orthogonalize(big[:-4].view(65, 300), O=big[4:].view(65, 300))
    assert torch.equal(g.gpic_orthogonalize(G, O=G), O)
    w, M = _randn((65, 300), "f32", 6), torch.zeros((65, 300), device=DEV)
    w2, M2 = w.clone(), M.clone()
    g.gpic_muon_step(w, w.clone(), M, 0.1)
    g.gpic_muon_step(w2, w2, M2, 0.1)           # G is read before W is written
    assert torch.equal(w, w2) and torch.equal(M, M2)
    with pytest.raises(g.GpicError, match="overlaps"):
        g.gpic_muon_step(w, M, M, 0.1)
