"""Layers, their gradients and the orthogonalised update on the GPU against
plain float64 formulas, at sizes that cross every tile, padding and split of
the contraction, and where they can go wrong: single rows, no rows, odd
widths, views, misaligned buffers, outliers, infinities and NaN.

Tolerances (u: half a unit in the last place of the type, e = 2^-24).
Layers: a float32 accumulation of K products is off by at most (K + 16) e
sum |x||w|; float32 operands as two halves add 2^-21 sum |x||w|, and
entries below 2^-17 of their matrix's largest an absolute 2^-38 of it; Phi is
off by 1e-7; the result is rounded once, and so is dZ before its products.
Orthogonalised matrices: relative Frobenius norm, 4e-5 where X, A and the
polynomial are held to 22 bits (three products of 2^-22 a step, five steps,
an average growth of ten), 4.6e-3 for half-precision products (three
roundings of 2^-12 a step, five steps, slopes near one, and a quarter
more), plus the type's rounding."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
E = 2.0 ** -24
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return g


def _randn(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=gen) * scale).to(T[dtype])


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        c = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * c, c + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def _product_error(A, B, dtype):
    """Bound on a product A B^T of float64 copies, before the output's rounding."""
    K = A.shape[1]
    b = ((K + 16) * E + (2.0 ** -21 if dtype == "f32" else 0.0)) * (A.abs() @ B.abs().t())
    if dtype == "f32" and A.numel():
        # entries far below their matrix's largest are rounded absolutely
        b = b + 2.0 ** -38 * (A.abs().max() * B.abs().sum(1)[None, :]
                              + B.abs().max() * A.abs().sum(1)[:, None])
    return b


def _close(got, ref, bound, dtype, what):
    err = (got.double() - ref).abs()
    tol = bound + U[dtype] * (ref.abs() + bound) + (2.0 ** -24 if dtype == "f16" else 1e-37)
    assert got.shape == ref.shape
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, float((err / tol).nan_to_num(nan=9e9).max()),
                                 int(bad.sum()))


# one row; fewer than a tile; tile edges; odd widths; long contractions (split);
# the middle and the large tile
SHAPES = [(1, 8, 8), (1, 2048, 520), (3, 5, 7), (7, 1000, 777), (17, 64, 64), (64, 64, 64),
          (65, 33, 129), (40, 4099, 40), (130, 72, 200), (257, 136, 300), (2100, 96, 1800),
          (4100, 72, 3333),
          # whole and split tiles of the middle and the large size, in every operand order
          (4099, 1003, 4200), (2600, 2900, 1400), (6000, 3200, 2800), (4300, 4100, 4300)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_linear_and_gradients(g, shape, dtype):
    n, k, m = shape
    for i, act in enumerate(("none", "relu", "gelu", "silu")):
        if n * m > 10 ** 6 and act in ("relu", "silu"):
            continue
        print(f"linear n={n} k={k} m={m} {dtype} {act}", flush=True)
        X, W = _randn((n, k), dtype, 1), _randn((m, k), dtype, 2, k ** -0.5)
        b = _randn((m,), dtype, 3) if i % 2 == 0 or m == 7 else None
        R = _randn((n, m), dtype, 4) if i >= 1 else None
        Y, Z = g.gpic_linear(X, W, b, act, R, want_pre=True)
        assert torch.equal(Y, g.gpic_linear(X, W, b, act, R))
        x, w = X.double(), W.double()
        z = x @ w.t() + (b.double() if b is not None else 0.0)
        a, _ = _act(z, act)
        pe = _product_error(x, w, dtype) + 2 * E * z.abs()
        _close(Z, z, pe, dtype, "Z")
        ref = a + (R.double() if R is not None else 0.0)
        _close(Y, ref, 1.13 * pe + 2e-7 * z.abs() + 4 * E * (a.abs() + ref.abs()), dtype, "Y")

        dY = _randn((n, m), dtype, 5, 0.01)
        gr = g.gpic_linear_backward(dY, X, W, Z if act != "none" else None, act)
        _, da = _act(Z.double(), act)
        dz = dY.double() * da
        # dZ as the products read it: rounded to the type, act' to 3e-7
        off = (U[dtype] if act != "none" and dtype != "f32" else 0.0) * dz.abs() \
            + 1e-6 * dY.double().abs() * (1 + Z.double().abs() * (act != "none"))
        _close(gr.dX, dz @ w, off @ w.abs() + _product_error(dz, w.t(), dtype), dtype, "dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _product_error(dz.t(), x.t(), dtype),
               dtype, "dW")
        _close(gr.db, dz.sum(0), (1e-6 + 70 * E) * (dY.double().abs() * (1 + Z.double().abs())).sum(0),
               dtype, "db")


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated_and_gradients(g, shape, dtype):
    n, k, m = shape
    for act in ("silu", "gelu") if n * m < 10 ** 6 else ("silu",):
        print(f"gated n={n} k={k} m={m} {dtype} {act}", flush=True)
        X, W = _randn((n, k), dtype, 1), _randn((2 * m, k), dtype, 2, k ** -0.5)
        H, Z = g.gpic_gated(X, W, act, want_pre=True)
        assert torch.equal(H, g.gpic_gated(X, W, act))
        x, w = X.double(), W.double()
        z = x @ w.t()
        pe = _product_error(x, w, dtype)
        _close(Z, z, pe, dtype, "Z")
        a, _ = _act(z[:, :m], act)
        u = z[:, m:]
        bound = (1.13 * pe[:, :m] + 2e-7 * z[:, :m].abs()) * (u.abs() + pe[:, m:]) \
            + a.abs() * pe[:, m:] + 4 * E * (a * u).abs()
        _close(H, a * u, bound, dtype, "H")

        dH = _randn((n, m), dtype, 5, 0.01)
        gr = g.gpic_gated_backward(dH, X, W, Z, act)
        zz, dh = Z.double(), dH.double()
        a, da = _act(zz[:, :m], act)
        dz = torch.cat([dh * zz[:, m:] * da, dh * a], 1)
        r = U[dtype] if dtype != "f32" else 0.0
        off = r * dz.abs() + 1e-6 * torch.cat(
            [(dh * zz[:, m:]).abs() * (1 + zz[:, :m].abs()), (dh * zz[:, :m]).abs()], 1)
        if dtype == "f32":      # one scale for dZ, from the bound |dH| max(|Z|, 1)
            off = off + 2.0 ** -38 * dh.abs().max() * max(1.0, float(zz.abs().max()))
        _close(gr.dX, dz @ w, off @ w.abs() + _product_error(dz, w.t(), dtype), dtype, "dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + _product_error(dz.t(), x.t(), dtype),
               dtype, "dW")


# up to 64 values of k (read as they lie, in pieces of 16 bytes): every number
# of pieces, ends inside one, and k shorter than one
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("k", [1, 3, 4, 7, 8, 11, 16, 17, 31, 32, 33, 40, 47, 49, 63, 64])
def test_short_contractions(g, k, dtype):
    for n, m, act in ((33, 1, "silu"), (100, 5, "none"), (50, 70, "gelu"), (1000, 128, "relu"),
                      (70, 8200, "gelu"), (9000, 37, "silu")):
        print(f"short n={n} k={k} m={m} {dtype} {act}", flush=True)
        # rows of a wider matrix, starting anywhere
        X = _randn((n, k + 3), dtype, 1)[:, 2:k + 2]
        W = _randn((2 * m, k + 1), dtype, 2, k ** -0.5)[:, 1:]
        b, R = _randn((m,), dtype, 3), _randn((n, m), dtype, 4)
        x, w = X.double(), W.double()
        Y, Z = g.gpic_linear(X, W[:m], b, act, R, want_pre=True)
        assert torch.equal(Y, g.gpic_linear(X, W[:m], b, act, R, Y=R.clone()))
        z = x @ w[:m].t() + b.double()
        pe = _product_error(x, w[:m], dtype) + 2 * E * z.abs()
        a, _ = _act(z, act)
        ref = a + R.double()
        _close(Z, z, pe, dtype, "Z")
        _close(Y, ref, 1.13 * pe + 2e-7 * z.abs() + 4 * E * (a.abs() + ref.abs()), dtype, "Y")
        H, Z = g.gpic_gated(X, W, "silu", want_pre=True)
        assert torch.equal(H, g.gpic_gated(X, W, "silu"))
        z = x @ w.t()
        pe = _product_error(x, w, dtype)
        _close(Z, z, pe, dtype, "gated Z")
        a, _ = _act(z[:, :m], "silu")
        u = z[:, m:]
        _close(H, a * u, (1.13 * pe[:, :m] + 2e-7 * z[:, :m].abs()) * (u.abs() + pe[:, m:])
               + a.abs() * pe[:, m:] + 4 * E * (a * u).abs(), dtype, "H")


def test_short_contraction_of_a_large_float32_result(g):
    """Beyond 32 values of k and 2^23 results float32 goes through the tiles."""
    for n, k, m in ((4100, 48, 2100), (4100, 64, 2100)):
        X, W = _randn((n, k), "f32", 1), _randn((m, k), "f32", 2, k ** -0.5)
        x, w = X.double(), W.double()
        _close(g.gpic_linear(X, W), x @ w.t(), _product_error(x, w, "f32"), "f32", "Y")


@pytest.mark.parametrize("dtype", list(T))
def test_short_contractions_keep_non_finite_values(g, dtype):
    """What a fragment reads twice at the end of k is not counted twice."""
    for k in (5, 9, 33):
        X, W = _randn((40, k), dtype, 1), _randn((20, k), dtype, 2)
        X[3, k - 1], X[4, k - 2], X[5, 0] = math.inf, -math.inf, math.nan
        Y = g.gpic_linear(X, W).float()
        keep = torch.tensor([i for i in range(40) if i not in (3, 4, 5)], device=DEV)
        assert bool(torch.isfinite(Y[keep]).all())
        assert torch.equal(Y[3], W[:, k - 1].float() * math.inf)
        assert torch.equal(Y[4], W[:, k - 2].float() * -math.inf)
        assert bool(Y[5].isnan().all())


# small gradients (one launch, dZ unrounded): ends of tiles of 16 and 64, one row, one
# column, contractions of one turn and of many, waves with nothing to do
SMALL = [(1, 1, 1), (2, 58, 588), (3, 65, 17), (16, 64, 16), (33, 100, 5), (50, 512, 123),
         (100, 1, 130), (130, 7, 500), (257, 80, 33), (1000, 33, 16), (1024, 20, 300),
         (200, 300, 512)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", SMALL, ids=str)
def test_small_gradients(g, shape, dtype):
    n, k, m = shape
    X = _randn((n, k + 3), dtype, 1)[:, 2:k + 2]
    W = _randn((2 * m, k + 1), dtype, 2, k ** -0.5)[:, 1:]
    dY = _randn((n, m + 5), dtype, 3)[:, 3:m + 3]
    x, w, dy = X.double(), W.double(), dY.double()
    for act in ("none", "relu", "gelu", "silu"):
        print(f"small n={n} k={k} m={m} {dtype} {act}", flush=True)
        Z = g.gpic_linear(X, W[:m], None, act, want_pre=True)[1]
        gr = g.gpic_linear_backward(dY, X, W[:m], Z if act != "none" else None, act)
        da = _act(Z.double(), act)[1]
        dz = dy * da
        off = 1e-6 * dy.abs() * (1 + Z.double().abs() * (act != "none"))
        # sums in float32 of what is in hand, nothing else rounded
        _close(gr.dX, dz @ w[:m], off @ w[:m].abs() + (m + 16) * E * (dz.abs() @ w[:m].abs()),
               dtype, "dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + (n + 16) * E * (dz.abs().t() @ x.abs()),
               dtype, "dW")
        _close(gr.db, dz.sum(0), off.sum(0) + (n + 16) * E * dz.abs().sum(0), dtype, "db")
        for want in ((True, False, False), (False, True, False), (False, False, True)):
            one = g.gpic_linear_backward(dY, X, W[:m], Z if act != "none" else None, act, *want)
            for name, asked in zip(("dX", "dW", "db"), want):
                got = getattr(one, name)
                assert torch.equal(got, getattr(gr, name)) if asked else got is None
    for act in ("silu", "relu"):
        Z = g.gpic_gated(X, W, act, want_pre=True)[1]
        gr = g.gpic_gated_backward(dY, X, W, Z, act)
        z = Z.double()
        a, da = _act(z[:, :m], act)
        dz = torch.cat([dy * z[:, m:] * da, dy * a], 1)
        off = 1e-6 * torch.cat([dy * z[:, m:], dy * z[:, :m]], 1).abs() \
            * (1 + torch.cat([z[:, :m], z[:, :m]], 1).abs())
        _close(gr.dX, dz @ w, off @ w.abs() + (2 * m + 16) * E * (dz.abs() @ w.abs()), dtype,
               "gated dX")
        _close(gr.dW, dz.t() @ x, off.t() @ x.abs() + (n + 16) * E * (dz.abs().t() @ x.abs()),
               dtype, "gated dW")


@pytest.mark.parametrize("dtype", list(T))
def test_small_forward_of_many_rows(g, dtype):
    """Rows in blocks of 32 through the few-row kernel."""
    for n, k, m in ((33, 100, 17), (64, 65, 33), (500, 300, 100), (2048, 129, 70)):
        X = _randn((n, k + 3), dtype, 1)[:, 2:k + 2]
        W = _randn((2 * m, k + 1), dtype, 2, k ** -0.5)[:, 1:]
        x, w = X.double(), W.double()
        _close(g.gpic_linear(X, W), x @ w.t(), _product_error(x, w, dtype), dtype, "Y")
        H, Z = g.gpic_gated(X, W, "relu", want_pre=True)
        z = x @ w.t()
        pe = _product_error(x, w, dtype)
        _close(Z, z, pe, dtype, "Z")
        a, u = z[:, :m].clamp(min=0), z[:, m:]
        _close(H, a * u, pe[:, :m] * (u.abs() + pe[:, m:]) + a * pe[:, m:] + 4 * E * (a * u).abs(),
               dtype, "H")


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradients_against_differences(g, act):
    """Directional derivatives of sum(c * Y) by central differences of the
    float32 operators: step 2^-6, so the difference is off by h^2 / 6 times
    the third derivative (below 2e-4 of the terms' size) and by 2^-20 / h of
    their rounding; 2e-3 of the root of the summed squares covers both."""
    n, k, m, h = 33, 20, 27, 2.0 ** -6
    X, c = _randn((n, k), "f32", 1), _randn((n, m), "f32", 3)
    D = _randn((n, k), "f32", 5, k ** -0.5)
    for rows, f, back in (
            (m, lambda x, w: g.gpic_linear(x, w, None, act, want_pre=True),
             lambda x, w, z: g.gpic_linear_backward(c, x, w, z, act)),
            (2 * m, lambda x, w: g.gpic_gated(x, w, act, want_pre=True),
             lambda x, w, z: g.gpic_gated_backward(c, x, w, z, act))):
        W = _randn((rows, k), "f32", 2, k ** -0.5)
        V = _randn((rows, k), "f32", 6, 1.0 / k)
        gr = back(X, W, f(X, W)[1])
        for got, lo, hi in (
                (gr.dX, (X - h * D, W), (X + h * D, W)),
                (gr.dW, (X, W - h * V), (X, W + h * V))):
            terms = c.double() * (f(*hi)[0].double() - f(*lo)[0].double()) / (2 * h)
            d = D if got is gr.dX else V
            ref = float((got.double() * d.double()).sum())
            size = float(terms.square().sum().sqrt())
            assert abs(float(terms.sum()) - ref) <= 2e-3 * size, act


@pytest.mark.parametrize("dtype", list(T))
def test_views_and_alignment(g, dtype):
    """Column and row slices, a transposed operand, buffers that start one
    value late: the same bits as the contiguous tensors."""
    n, k, m = 150, 96, 136
    X, W, b, R = (_randn(s, dtype, i) for i, s in enumerate(((n, k), (m, k), (m,), (n, m))))
    Y, Z = g.gpic_linear(X, W, b, "gelu", R, want_pre=True)
    gr = g.gpic_linear_backward(R, X, W, Z, "gelu")

    def wide(t, pad, first):
        big = torch.full((t.shape[0] + 2, t.shape[1] + pad), float("nan"), dtype=t.dtype,
                         device=DEV)
        v = big[1:1 + t.shape[0], first:first + t.shape[1]]
        v.copy_(t)
        return v

    def late(t):
        flat = torch.full((t.numel() + 1,), float("nan"), dtype=t.dtype, device=DEV)
        v = flat[1:].view(t.shape)
        v.copy_(t)
        return v

    for make in (lambda t: wide(t, 24, 8), lambda t: wide(t, 5, 3), late,
                 lambda t: t.t().contiguous().t()):
        x, w, r, z = make(X), make(W), make(R), make(Z)
        out = torch.empty_like(R)
        assert torch.equal(g.gpic_linear(x, w, late(b[None])[0], "gelu", r, Y=out), Y)
        got = g.gpic_linear_backward(r, x, w, z, "gelu")
        for a, e in zip((got.dX, got.dW, got.db), (gr.dX, gr.dW, gr.db)):
            assert torch.equal(a, e)
    # strided and in-place outputs
    out = wide(R, 7, 3)
    assert torch.equal(g.gpic_linear(X, W, b, "gelu", out, Y=out), Y)
    H = g.gpic_gated(X, W)
    assert torch.equal(g.gpic_gated(wide(X, 5, 3), late(W), H=wide(H, 3, 1)), H)


@pytest.mark.parametrize("dtype", list(T))
def test_no_rows(g, dtype):
    X, W = _randn((0, 40), dtype, 1), _randn((24, 40), dtype, 2)
    Y, Z = g.gpic_linear(X, W, _randn((24,), dtype, 3), "gelu", want_pre=True)
    assert Y.shape == (0, 24)
    gr = g.gpic_linear_backward(Y, X, W, Z, "gelu")
    assert gr.dX.shape == (0, 40)
    assert not bool(gr.dW.any()) and not bool(gr.db.any())
    H, Z = g.gpic_gated(X, W, want_pre=True)
    gr = g.gpic_gated_backward(H, X, W, Z)
    assert H.shape == (0, 12) and not bool(gr.dW.any())
    assert g.gpic_orthogonalize(torch.empty((0, 5, 7), dtype=T[dtype], device=DEV)).shape == (0, 5, 7)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [3, 200])
def test_non_finite_values_stay_in_their_rows(g, dtype, n):
    X, W = _randn((n, 100), dtype, 1), _randn((140, 100), dtype, 2, 0.1)
    clean = g.gpic_linear(X, W, None, "gelu")
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = X.clone()
        x[1, 37] = bad
        y = g.gpic_linear(x, W)
        keep = torch.arange(n, device=DEV) != 1
        assert not bool(torch.isfinite(y[1]).any())
        assert bool(torch.isfinite(y[keep]).all())
        y = g.gpic_linear(x, W, None, "gelu")
        # the operands' scale comes from the finite values, so the rest keeps its bits
        if not bool((X.abs().max() == X[1, 37].abs())):
            assert torch.equal(y[keep], clean[keep])
        h, z = g.gpic_gated(x, W, want_pre=True)
        assert bool(torch.isfinite(h[keep]).all())
        gr = g.gpic_gated_backward(h.nan_to_num(0, 0, 0), x, W, z)
        assert bool(torch.isfinite(gr.dX[keep]).all())


def test_activation_limits(g):
    """Z = X through the identity: large, infinite and tiny arguments."""
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5.0, -5.0, 13.9, -13.9, 14.1, -14.1, 90.0, -90.0,
                      120.0, -120.0, 1e4, -1e4], device=DEV)
    X, W = z[:, None].contiguous(), torch.ones((1, 1), device=DEV)
    for act in ("relu", "gelu", "silu"):
        a, da = _act(z.double(), act)
        y = g.gpic_linear(X, W, None, act)[:, 0].double()
        # the split parts hold 2^-38 of the largest entry, 10^4
        tol = 3e-7 * (a.abs() + z.double().abs().clamp(max=20)) + 2.0 ** -38 * 1e4
        assert bool(((y - a).abs() <= tol).all()), act
        d = g.gpic_linear_backward(torch.ones_like(X), X, W, X, act).dX[:, 0].double()
        assert bool(((d - da).abs() <= 2e-6).all()), act


def test_outlier_row_float32(g):
    """One point 10^6 away: the other rows keep 2^-38 of the largest entry."""
    X, W = _randn((300, 64), "f32", 1), _randn((96, 64), "f32", 2, 0.125)
    X[17] *= 1e6
    _close(g.gpic_linear(X, W), X.double() @ W.double().t(),
           _product_error(X.double(), W.double(), "f32"), "f32", "Y")


def test_offsets_beyond_32_bits(g):
    """n m > 2^32 values of Y, Z, dY and dZ: the rows on both sides of every
    power of two, and the gradients of the weights and the bias in chunks."""
    n, k, m = 525000, 24, 8200
    print(f"linear n={n} m={m} ({n * m} values)", flush=True)
    X, W, b = _randn((n, k), "bf16", 1), _randn((m, k), "bf16", 2, k ** -0.5), _randn((m,), "bf16", 3)
    Y, Z = g.gpic_linear(X, W, b, "gelu", want_pre=True)
    gr = g.gpic_linear_backward(Y, X, W, Z, "gelu")
    w = W.double()
    rows = sorted({r for p in range(30, 33) for d in (-1, 0, 1) for r in [2 ** p // m + d] if r < n}
                  | {0, 1, n - 2, n - 1})
    x = X[rows].double()
    z = x @ w.t() + b.double()
    pe = _product_error(x, w, "bf16") + 2 * E * z.abs()
    _close(Z[rows], z, pe, "bf16", "Z")
    _close(Y[rows], _act(z, "gelu")[0], 1.13 * pe + 2e-7 * z.abs(), "bf16", "Y")
    dy, zz = Y[rows].double(), Z[rows].double()
    dz = dy * _act(zz, "gelu")[1]
    off = U["bf16"] * dz.abs() + 1e-6 * dy.abs() * (1 + zz.abs())
    _close(gr.dX[rows], dz @ w, off @ w.abs() + _product_error(dz, w.t(), "bf16"), "bf16", "dX")
    dW = torch.zeros((m, k), dtype=torch.float64, device=DEV)
    size, off, db, dba = torch.zeros_like(dW), torch.zeros_like(dW), 0.0, 0.0
    for r in range(0, n, 35000):
        zz, dy, x = Z[r:r + 35000].double(), Y[r:r + 35000].double(), X[r:r + 35000].double()
        dz = dy * _act(zz, "gelu")[1]
        dW += dz.t() @ x
        size += dz.abs().t() @ x.abs()
        db, dba = db + dz.sum(0), dba + (dy.abs() * (1 + zz.abs())).sum(0)
        del zz, dy, dz, x
    # sums of n values in float32: rounding errors of n partial sums, of
    # random sign, 4 sqrt(n) of them at the most likely worst
    _close(gr.dW, dW, (U["bf16"] + 1e-6 + 4 * math.sqrt(n) * E) * size, "bf16", "dW")
    _close(gr.db, db, (1e-6 + 70 * E) * dba, "bf16", "db")


def test_binding_refusals(g):
    x = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)  # noqa: E731
    X, W = x(5, 8), x(6, 8)
    bad = [
        (ValueError, lambda: g.gpic_linear(X, x(6, 7))),
        (ValueError, lambda: g.gpic_linear(x(8), W)),
        (ValueError, lambda: g.gpic_linear(X, W, activation="tanh")),
        (ValueError, lambda: g.gpic_linear(X, W, x(5))),
        (ValueError, lambda: g.gpic_linear(X, W, residual=x(5, 7))),
        (ValueError, lambda: g.gpic_linear(X, W, Y=x(6, 5).t())),
        (ValueError, lambda: g.gpic_linear(X, W.cpu().to(DEV), Y=x(4, 6))),
        (TypeError, lambda: g.gpic_linear(X, W.half())),
        (TypeError, lambda: g.gpic_linear(X.double(), W.double())),
        (TypeError, lambda: g.gpic_linear(X, W, x(6, dt=torch.float16))),
        (ValueError, lambda: g.gpic_gated(X, x(7, 8))),
        (ValueError, lambda: g.gpic_linear_backward(x(5, 6), X, W, None, "gelu")),
        (ValueError, lambda: g.gpic_linear_backward(x(5, 5), X, W)),
        (TypeError, lambda: g.gpic_gated_backward(x(5, 3).half(), X.half(), W.half(), x(5, 6).half())),
        (ValueError, lambda: g.gpic_gated_backward(x(5, 3), X, W, x(5, 5))),
        (ValueError, lambda: g.gpic_orthogonalize(x(5))),
        (TypeError, lambda: g.gpic_orthogonalize(x(5, 4).double())),
        (ValueError, lambda: g.gpic_orthogonalize(x(5, 4), O=x(4, 5).t())),
        (ValueError, lambda: g.gpic_muon_step(W, x(6, 7), x(6, 8), 0.1)),
        (TypeError, lambda: g.gpic_muon_step(W.half(), W.half(), W.half(), 0.1)),
        (ValueError, lambda: g.gpic_muon_step(x(8, 6).t(), W, x(6, 8), 0.1)),
        (g.GpicError, lambda: g.gpic_orthogonalize(x(5, 4), steps=0)),
        (g.GpicError, lambda: g.gpic_orthogonalize(x(5, 4), coefficients=(20.0, 0.0, 0.0))),
        (g.GpicError, lambda: g.gpic_muon_step(W, W.clone(), x(6, 8), float("nan"))),
    ]
    for i, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"case {i} was accepted")


# ------------------------------------------------- orthogonalised updates
COEF = (3.4445, -4.7750, 2.0315)


def _polar(G, steps=5, coef=COEF, eps=1e-7):
    a, b, c = coef
    X = G.double()
    X = X / (X.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        if X.shape[-2] <= X.shape[-1]:
            A = X @ X.transpose(-2, -1).contiguous()
            X = a * X + (b * A + c * A @ A) @ X
        else:
            A = X.transpose(-2, -1).contiguous() @ X
            X = a * X + X @ (b * A + c * A @ A)
    return X


def _gradient(shape, seed, floor=0.5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    b, m, n = shape
    r = max(1, min(m, n) // 4)
    s = torch.arange(1, r + 1, device=DEV).rsqrt()
    u = torch.randn((b, m, r), device=DEV, generator=gen) * s
    v = torch.randn((b, r, n), device=DEV, generator=gen)
    return torch.bmm(u, v) + floor * torch.randn((b, m, n), device=DEV, generator=gen)


def _polar_tolerance(dtype):
    return {"f32": 4e-5, "f16": 4e-5 + U["f16"], "bf16": 4.6e-3 + U["bf16"]}[dtype]


def _rel(got, ref):
    d = (got.double() - ref).square().sum((-2, -1)).sqrt()
    return float((d / ref.square().sum((-2, -1)).sqrt()).max())


STACKS = [(1, 1, 1), (2, 1, 7), (2, 9, 1), (1, 16, 16), (12, 64, 256), (3, 256, 64), (5, 100, 300),
          (2, 513, 129), (3, 65, 65), (1, 300, 1000), (2, 20, 4100), (1, 2000, 33),
          (1, 1100, 1500), (1, 2500, 1025), (1, 30, 1024), (4, 64, 448), (2, 448, 63), (1, 65, 448),
          (3, 1500, 2100), (1, 4100, 2300), (1, 4000, 4100), (1, 5900, 6100)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", STACKS, ids=str)
def test_orthogonalize(g, shape, dtype):
    print(f"orthogonalize {shape} {dtype}", flush=True)
    G = _gradient(shape, 3).to(T[dtype])
    O = g.gpic_orthogonalize(G)
    assert _rel(O, _polar(G)) <= _polar_tolerance(dtype)
    again = G.clone()
    g.gpic_orthogonalize(again, O=again)
    assert torch.equal(again, O)
    if shape[0] > 1:                       # a stack is its matrices
        assert _rel(g.gpic_orthogonalize(G[1])[None], _polar(G[1:2])) <= _polar_tolerance(dtype)


@pytest.mark.parametrize("shape", [(2, 58, 45), (3, 64, 256), (2, 31, 1000), (2, 2489, 31),
                                   (1, 64, 4000)], ids=str)
def test_orthogonalize_few_directions_bf16(g, shape):
    """A smaller side of up to 64: split operands, so the result's own rounding
    (at most 2^-9 of an entry) and float32's 4e-5 are all."""
    G = _gradient(shape, 11).to(torch.bfloat16)
    assert _rel(g.gpic_orthogonalize(G), _polar(G)) <= 2.0 ** -9 + 4e-5


@pytest.mark.parametrize("dtype", list(T))
def test_orthogonalize_other_polynomials_and_ranks(g, dtype):
    G = _gradient((2, 96, 160), 5, floor=0.02).to(T[dtype])
    for steps, coef in ((1, COEF), (2, COEF), (12, (15 / 8, -10 / 8, 3 / 8)), (7, (1.5, -0.5, 0.0))):
        # the slower polynomials grow what is rounded off by a^steps at most
        tol = _polar_tolerance(dtype) * (1 if steps < 5 else 4)
        assert _rel(g.gpic_orthogonalize(G, steps, coef), _polar(G, steps, coef)) <= tol
    # rank one over nothing: the singular vectors of the one direction
    u, v = _randn((60, 1), "f32", 1), _randn((1, 90), "f32", 2)
    G = (u @ v).to(T[dtype])
    if dtype == "f32":
        assert _rel(g.gpic_orthogonalize(G)[None], _polar(G[None])) <= 1e-3
    Z = g.gpic_orthogonalize(torch.zeros((2, 70, 90), dtype=T[dtype], device=DEV))
    assert not bool(Z.any())


def test_orthogonalize_magnitudes_and_non_finite(g):
    G = _gradient((3, 70, 130), 7)
    ref = _polar(G, eps=0.0)
    for s in (1e30, 1e-30, 1e-3):
        assert _rel(g.gpic_orthogonalize(G * s, eps=0.0), ref) <= 4e-5
    O = g.gpic_orthogonalize(G)
    G[1, 3, 5] = float("nan")
    P = g.gpic_orthogonalize(G)
    assert torch.equal(P[0], O[0]) and torch.equal(P[2], O[2])
    assert not bool(torch.isfinite(P[1]).any())


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(1, 40, 70), (3, 65, 33), (2, 128, 256), (1, 700, 300)], ids=str)
def test_muon_step(g, shape, nesterov, dtype):
    b, m, n = shape
    W = _randn(shape, dtype, 1, n ** -0.5)
    M = _gradient(shape, 2) * 0.01
    w, mo = W.double(), M.double()
    for step in range(3):
        G = (_gradient(shape, 10 + step) * 0.01).to(T[dtype])
        before = w if step == 0 else W.double()
        mo = 0.9 * mo + G.double()
        U_ = G.double() + 0.9 * mo if nesterov else mo
        s = max(1.0, m / n) ** 0.5
        ref = (1 - 0.05 * 0.1) * before - 0.05 * s * _polar(U_)
        g.gpic_muon_step(W, G, M, 0.05, 0.9, nesterov, 0.1)
        assert float((M.double() - mo).abs().max()) <= 16 * E * float(mo.abs().max())
        tol = 0.05 * s * _polar_tolerance("f32" if dtype == "f16" else dtype) \
            * float(_polar(U_).square().sum().sqrt()) + U[dtype] * float(ref.square().sum().sqrt()) * 1.01
        assert float((W.double() - ref).square().sum().sqrt()) <= tol
    # a scale of its own, on a single matrix
    W1, M1, G1 = W[0].clone(), M[0].clone(), G[0].clone()
    g.gpic_muon_step(W1, G1, M1, 0.0, 0.9, nesterov, 0.0, scale=2.0)
    assert torch.equal(W1, W[0])


# ------------------------------------------------------------ how they run
def _everything(g, dtype):
    n, k, m = 70, 50, 90
    X, W, V = _randn((n, k), dtype, 1), _randn((m, k), dtype, 2, 0.2), _randn((k, m), dtype, 3, 0.1)
    W2 = _randn((2 * m, k), dtype, 4, 0.2)
    Y, Z = g.gpic_linear(X, W, _randn((m,), dtype, 5), "gelu", want_pre=True)
    out = g.gpic_linear(Y, V, None, "none", X)
    gr = g.gpic_linear_backward(Y, X, W, Z, "gelu")
    H, ZZ = g.gpic_gated(X, W2, want_pre=True)
    gg = g.gpic_gated_backward(H, X, W2, ZZ)
    K = g.gpic_linear(_randn((30, 3000), dtype, 6), _randn((40, 3000), dtype, 7, 0.02))
    O = g.gpic_orthogonalize(gr.dW)
    P = g.gpic_orthogonalize(_gradient((2, 33, 2000), 8).to(T[dtype]))
    M = torch.ones_like(W, dtype=torch.float32)
    W = W.clone()
    g.gpic_muon_step(W, gr.dW, M, 0.1)
    return [Y, Z, out, gr.dX, gr.dW, gr.db, H, ZZ, gg.dX, gg.dW, K, O, P, W, M]


@pytest.mark.parametrize("dtype", list(T))
def test_results_do_not_depend_on_the_buffers(g, monkeypatch, dtype):
    from gpu_helpers import Filled
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
    """The operators on a stream of the caller's, and captured into a graph
    that is replayed between eager work: the same bits every time."""
    eager = [t.clone() for t in _everything(g, dtype)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        on = _everything(g, dtype)
    s.synchronize()
    for a, b in zip(on, eager):
        assert torch.equal(a, b)
    n, k, m = 70, 50, 90
    X, W, W2 = _randn((n, k), dtype, 1), _randn((m, k), dtype, 2, 0.2), _randn((2 * m, k), dtype, 4, 0.2)

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
        X.copy_(_randn((n, k), dtype, 20 + i))
        want = step()
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i
