"""Cross entropy without logits on the GPU against plain float64 formulas, at
sizes that cross every tile, padding and piece of the vocabulary, and where it
can go wrong: one entry, one row, no rows, padding, entries that a bias takes
out, targets that are all but certain, infinities and NaN, tiny and huge
gradients.

Tolerances (u: half a unit in the last place of the type, e = 2^-24).  A logit
is off by dz = (K + 16) e sum |x||w| + 2 e |z|, float32 operands as two halves
add 2^-21 sum |x||w| and 2^-38 of each side's largest times the other's sum.
An exponential is off by the error of its argument, 2 e of it and 4 e; sums of
them pass through at most v / 256 + 40 joins of 4 e; so the others' lse is off
by dl = max over their probabilities of dz, weighted, and that.  The loss
softplus(lse' - z_t) has the slope 1 - p_t.  dZ then is off by that times p,
and is rounded as the products' operand: to the type, float16 and float32 no
finer than 2^-39 of the row's |dloss|, float32 to 2^-22.  dW's other operand is X
times dloss over its largest, rounded to the type where that is not 1."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
E = 2.0 ** -24
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return g


def _randn(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=gen) * scale).to(T[dtype])


def _within(got, ref, tol, what):
    assert got.shape == ref.shape
    err = (got.double() - ref).abs()
    bad = ~((err <= tol) | (got.double() == ref))
    assert not bool(bad.any()), (what, float((err / tol).nan_to_num(nan=9e9).max()),
                                 int(bad.sum()))


def _close(got, ref, bound, dtype, what):
    assert got.dtype == T[dtype]
    tol = bound + U[dtype] * (ref.abs() + bound) + TINY[dtype]
    if dtype == "f16":
        # float16's largest value is 2^16 - 2^5, the next would be 2^16: what is 2^16 -
        # 2^4 = 65,520 or more in magnitude rounds to infinity (the tie to the even 2^16),
        # so an exact value is infinite if it is that far out less its bound, and may
        # be if it is that far out with it
        edge, inf = 65520.0, torch.copysign(torch.full_like(ref, math.inf), ref)
        must, may = ref.abs() - bound >= edge, ref.abs() + bound >= edge
        ref = torch.where(must | (may & got.isinf()), inf, ref)
    _within(got, ref, tol, what)


def _inputs(n, k, v, dtype, seed=1, bias=True, spread=3.0):
    X, W = _randn((n, k), dtype, seed), _randn((v, k), dtype, seed + 1, spread * k ** -0.5)
    b = _randn((v,), dtype, seed + 2, 0.5) if bias else None
    gen = torch.Generator(device=DEV).manual_seed(seed + 3)
    t = torch.randint(v, (n,), device=DEV, generator=gen)
    if n > 2:
        t[n // 3] = -100
        t[n // 2] = v
    if n > 8:                  # rows that all but know their target
        some = torch.arange(0, n, 3, device=DEV)
        w = W[t[some].clamp(0, v - 1)].float()
        X[some] += (w * (7.0 / w.norm(dim=1, keepdim=True).clamp(min=1e-3))).to(T[dtype])
    return X, W, b, t


def _check(g, X, W, b, t, dloss, dtype, what):
    (n, k), v = X.shape, W.shape[0]
    print(f"loss n={n} k={k} v={v} {dtype} {what}", flush=True)
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    assert torch.equal(loss, g.gpic_cross_entropy(X, W, t, b))
    gr = g.gpic_cross_entropy_backward(dloss, X, W, t, loss, lse, b)
    again = g.gpic_cross_entropy_backward(dloss, X, W, t, loss, lse, b)
    for name in ("dX", "dW", "db"):
        assert torch.equal(getattr(gr, name), getattr(again, name))
    x, w = X.double(), W.double()
    real = (t >= 0) & (t < v)
    at = t.clamp(0, v - 1).long()[:, None]
    z = x @ w.t()
    if b is not None:
        z += b.double()
    dz = (k + 16) * E * (x.abs() @ w.abs().t()) + 2 * E * z.abs().nan_to_num(posinf=0.0)
    if dtype == "f32":
        dz += 2.0 ** -21 * (x.abs() @ w.abs().t())
        dz += 2.0 ** -38 * (x.abs().amax(1)[:, None] * w.abs().sum(1)
                            + w.abs().amax(1) * x.abs().sum(1)[:, None])
    full = z.logsumexp(1)
    p = (z - full[:, None]).exp()
    one = torch.zeros_like(p).scatter_(1, at, real.double()[:, None])
    others = z.masked_fill(one > 0, -math.inf).logsumexp(1)
    q = (z - others[:, None]).exp().masked_fill(one > 0, 0.0).nan_to_num(nan=0.0)   # of the others
    joins = 4 * (v / 256 + 40) * E
    far = (z - z.amax(1, keepdim=True)).abs().nan_to_num(posinf=0.0)
    dl = (q * (dz + 2 * E * far + 4 * E)).sum(1) + joins + 2 * E * others.abs().nan_to_num(posinf=0.0)
    zt, dzt = z.gather(1, at)[:, 0], dz.gather(1, at)[:, 0]
    pt = (p * one).sum(1)
    ref = torch.where(real, torch.nn.functional.softplus(others - zt, threshold=1e9), 0.0)
    rest = -torch.expm1(-ref)                      # 1 - p_t
    # (the slope along the error is at most e^error times that)
    dloss_err = rest * 1.01 * (dl + dzt) + 6 * E * ref
    _within(loss, ref, torch.where(real, dloss_err, 0.0), "loss")
    assert not loss[~real].any()
    lse_err = (p * (dz + 2 * E * far + 4 * E)).sum(1) + joins + 4 * E * full.abs()
    _within(lse, full, lse_err, "lse")

    gl = torch.where(real, dloss.double(), 0.0)[:, None]
    d = gl * (p - one)
    d = torch.where(one > 0, -gl * rest[:, None], d)
    rel = dz + lse_err[:, None] + 2 * E * (z - full[:, None]).abs().nan_to_num(posinf=0.0) + 6 * E
    off = gl.abs() * torch.where(one > 0, (pt * dloss_err)[:, None] + 6 * E * rest[:, None], p * rel)
    _close(gr.db, d.sum(0), off.sum(0) + (n / 64 + 32) * E * d.abs().sum(0), dtype, "db")
    if dtype == "f32":
        off = off + 2.0 ** -22 * d.abs() + 2.0 ** -39 * gl.abs()
    else:
        off = off + U[dtype] * d.abs() + (2.0 ** -39 * gl.abs() if dtype == "f16" else 0.0)
    ex = off @ w.abs() + (v + 48) * E * (d.abs() @ w.abs())
    ew = off.t() @ x.abs() + (n + 16) * E * (d.abs().t() @ x.abs())
    # X times its share of the largest dloss, as dW's operand: a float32 division and
    # product, rounded to the type (float16: 2^-25 of the largest dloss at least)
    unlike = bool((gl[gl != 0].abs() != gl.abs().max()).any()) if bool(gl.any()) else False
    ew += (3 * E + (U[dtype] if unlike else 0.0)) * (d.abs().t() @ x.abs())
    if dtype == "f16" and unlike:
        ew += 2.0 ** -25 * gl.abs().max() * (d.abs() / gl.abs().clamp(min=1e-300)).sum(0)[:, None]
    if dtype == "f32":
        ex += 2.0 ** -21 * (d.abs() @ w.abs()) + 2.0 ** -38 * d.abs().sum(1)[:, None] * w.abs().amax(0)
        share = (d.abs() / gl.abs().clamp(min=1e-300)).sum(0)
        ew += 2.0 ** -21 * (d.abs().t() @ x.abs()) + 2.0 ** -38 * share[:, None] * (gl.abs() * x.abs()).amax(0)
    _close(gr.dX, d @ w, ex, dtype, "dX")
    _close(gr.dW, d.t() @ x, ew, dtype, "dW")
    assert not gr.dX[~real].any()
    return loss, lse, gr


SHAPES = [(1, 8, 1), (1, 2048, 500), (3, 5, 7), (17, 64, 300), (33, 40, 1000), (64, 64, 64),
          (130, 72, 257), (52, 512, 1013), (300, 136, 5000), (1003, 700, 10007), (2100, 96, 3001),
          (4100, 72, 5001), (2049, 520, 4099), (700, 1, 33), (20, 3001, 100), (5000, 24, 2),
          # few float32 rows over a large vocabulary, odd widths and partial blocks
          (1, 130, 5000), (16, 63, 3001), (17, 65, 2049), (33, 700, 4007), (64, 1, 2500), (48, 4099, 3000),
          (65, 200, 3000), (64, 300, 5003), (8, 203, 5001), (32, 129, 900),
          # tiles of the large size in every product
          (6000, 1100, 9000),
          # a handful of classes; rows beyond what 128 workgroups take at once
          (64, 20000, 5), (40, 5000, 20), (600000, 8, 3)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_loss_and_gradients(g, shape, dtype):
    n, k, v = shape
    X, W, b, t = _inputs(n, k, v, dtype)
    scale = 64.0 if dtype == "f16" else 1.0 / n
    _check(g, X, W, b, t, torch.full((n,), scale, device=DEV), dtype, "mean")
    if n * v < 3 * 10 ** 7:
        weight = _randn((n,), "f32", 9, scale)
        _check(g, X, W, None, t.int(), weight, dtype, "weighted")


@pytest.mark.parametrize("dtype", list(T))
def test_pieces_of_the_vocabulary(g, dtype):
    """dZ beyond 512 MB: several pieces, the last of them short."""
    n, k, v = (9001, 72, 33003)
    X, W, b, t = _inputs(n, k, v, dtype)
    _check(g, X, W, b, t, torch.full((n,), 1.0 if dtype == "f16" else 1.0 / n, device=DEV), dtype,
           "pieces")


def test_rows_of_unlike_gradients_float32(g):
    """Rows keep their bits whatever the other rows' gradients are, and the
    columns' sums theirs; rows without a gradient take none."""
    n, k, v = 2500, 40, 700
    X, W, b, t = _inputs(n, k, v, "f32")
    dloss = torch.exp2(-torch.arange(n, device=DEV) % 90 * 1.0)
    dloss[5::7] = 0.0
    _check(g, X, W, b, t, dloss, "f32", "unlike")
    _check(g, X, W, b, t, dloss * 1e-30, "f32", "tiny")
    _check(g, X, W, b, t, dloss * 1e9, "f32", "huge")        # up to 6e35
    # an infinite gradient stays in its row of dX
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    ref = g.gpic_cross_entropy_backward(dloss, X, W, t, loss, lse, b).dX
    some = dloss.clone()
    some[7] = math.inf
    dX = g.gpic_cross_entropy_backward(some, X, W, t, loss, lse, b).dX
    keep = torch.arange(n, device=DEV) != 7
    assert not bool(dX[7].isfinite().any()) and torch.equal(dX[keep], ref[keep])
    zero = torch.zeros_like(dloss)
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    gr = g.gpic_cross_entropy_backward(zero, X, W, t, loss, lse, b)
    assert not gr.dX.any() and not gr.dW.any() and not gr.db.any()


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [5, 300])
def test_entries_taken_out(g, n, dtype):
    """A bias of -inf takes entries out; a target among them is impossible."""
    X, W, b, t = _inputs(n, 48, 5000 if n == 300 else 130, dtype)
    v = W.shape[0]
    out = torch.rand(v, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.5
    b = b.masked_fill(out, -math.inf)
    live = (~out).nonzero()[:, 0]
    t = torch.where((t >= 0) & (t < v), live[t.clamp(0, v - 1) % len(live)], t)
    _check(g, X, W, b, t, torch.ones(n, device=DEV), dtype, "out")
    t[1] = out.nonzero()[0, 0]
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    assert float(loss[1]) == math.inf and bool(lse.isfinite().all())
    gr = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), X, W, t, loss, lse, b)
    assert bool(gr.dX.isfinite().all() and gr.dW.isfinite().all())
    assert not gr.dW[out & (torch.arange(v, device=DEV) != t[1])].any()
    # nothing left
    loss = g.gpic_cross_entropy(X, W, t, torch.full_like(b, -math.inf))
    real = (t >= 0) & (t < v)
    assert bool(loss[real].isnan().all()) and not loss[~real].any()


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [5, 300, 2100])
def test_masks_of_the_lowest_value(g, n, dtype):
    """Entries at the type's lowest value weigh nothing beside others, and as
    much as each other where nothing else is left."""
    X, W, b, t = _inputs(n, 48, 130 if n == 5 else 5000, dtype)
    v = W.shape[0]
    out = torch.rand(v, generator=torch.Generator().manual_seed(2)).to(DEV) < 0.5
    live = (~out).nonzero()[:, 0]
    t = torch.where((t >= 0) & (t < v), live[t.clamp(0, v - 1) % len(live)], t)
    low = torch.finfo(T[dtype]).min
    one = torch.ones(n, device=DEV)
    got = []
    for mask in (low, -math.inf):
        loss, lse = g.gpic_cross_entropy(X, W, t, b.masked_fill(out, mask), want_lse=True)
        gr = g.gpic_cross_entropy_backward(one, X, W, t, loss, lse, b.masked_fill(out, mask))
        got.append((loss, lse, gr.dX, gr.dW, gr.db))
    for a, c in zip(*got):
        assert torch.equal(a, c)
    # all of them: the products vanish beside 3.4e38 (not beside float16's lowest,
    # whose share cancels), and every entry weighs the same
    mask = torch.full_like(b, low)
    loss, lse = g.gpic_cross_entropy(X, W, t, mask, want_lse=True)
    gr = g.gpic_cross_entropy_backward(one, X, W, t, loss, lse, mask)
    real = (t >= 0) & (t < v)
    z = X.double() @ W.double().t() if dtype == "f16" else torch.zeros((n, v), device=DEV).double()
    ref = z.logsumexp(1) - z.gather(1, t.clamp(0, v - 1)[:, None])[:, 0]
    # float16: logits beside 65504 are off by 2^-8 in float32
    tol = 2.0 ** -6 if dtype == "f16" else 4 * (v / 256 + 40) * E + 1e-6
    assert float((loss.double() - ref)[real].abs().max()) <= tol and not loss[~real].any()
    d = (z - z.logsumexp(1, keepdim=True)).exp()
    d[torch.arange(n, device=DEV), t.clamp(0, v - 1)] -= 1.0
    d = torch.where(real[:, None], d, 0.0)
    size = d.abs() @ W.double().abs()
    _close(gr.dX, d @ W.double(), (2 * tol + U[dtype] + (v + 48) * E) * size, dtype, "dX")


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [6, 300])
def test_non_finite_rows_and_certain_targets(g, n, dtype):
    X, W, b, t = _inputs(n, 48, 900 if n == 6 else 5000, dtype)
    v = W.shape[0]
    t = t.clamp(0, v - 1)
    ref = g.gpic_cross_entropy(X, W, t, b)
    bad = X.clone()
    bad[1, 3], bad[4, 0] = math.nan, math.inf
    loss, lse = g.gpic_cross_entropy(bad, W, t, b, want_lse=True)
    keep = [i for i in range(n) if i not in (1, 4)]
    assert bool(loss[[1, 4]].isnan().all()) and torch.equal(loss[keep], ref[keep])
    dX = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), bad, W, t, loss, lse, b).dX
    clean = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), X, W, t,
                                          *g.gpic_cross_entropy(X, W, t, b, want_lse=True), b).dX
    assert bool(dX[[1, 4]].isnan().all()) and torch.equal(dX[keep], clean[keep])
    # padding rows may hold anything
    pad = t.clone()
    pad[[1, 4]] = -1
    loss, lse = g.gpic_cross_entropy(bad, W, pad, b, want_lse=True)
    assert not loss[[1, 4]].any()
    gr = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), bad, W, pad, loss, lse, b)
    assert not gr.dX[[1, 4]].any() and torch.equal(gr.dX[keep], clean[keep])
    few = g.gpic_cross_entropy(X, W, pad, b, want_lse=True)
    want = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), X, W, pad, *few, b)
    assert torch.equal(gr.dW, want.dW) and torch.equal(gr.db, want.db)
    # so may rows whose dloss is 0
    some = torch.ones(n, device=DEV)
    some[[1, 4]] = 0.0
    loss, lse = g.gpic_cross_entropy(bad, W, t, b, want_lse=True)
    gr = g.gpic_cross_entropy_backward(some, bad, W, t, loss, lse, b)
    assert not gr.dX[[1, 4]].any() and torch.equal(gr.dX[keep], clean[keep])
    assert torch.equal(gr.dW, want.dW) and torch.equal(gr.db, want.db)
    # a loss far below a float32 rounding of its logits
    b2 = torch.zeros_like(b)
    b2[7] = 60.0
    sure = torch.full_like(t, 7)
    _check(g, X, W, b2, sure, torch.ones(n, device=DEV), dtype, "sure")


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", [(9, 100, 60), (1100, 104, 3000), (1100, 99, 3000),
                                   (7, 99, 3000)], ids=str)
def test_views_alignment_and_wanted_gradients(g, shape, dtype):
    n, k, v = shape
    X, W, b, t = _inputs(n, k, v, dtype)
    d = torch.full((n,), 1.0, device=DEV)
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    ref = g.gpic_cross_entropy_backward(d, X, W, t, loss, lse, b)
    table = _randn((n, k + 24), dtype, 5)
    table[:, 8:8 + k] = X
    off = torch.zeros(v * k + 1, dtype=T[dtype], device=DEV)[1:].view(v, k)
    off.copy_(W)
    wide = _randn((v, k + 3), dtype, 6)
    wide[:, :k] = W
    for x in (X, table[:, 8:8 + k], X.t().contiguous().t()):
        for w in (W, off, wide[:, :k]):
            a, c = g.gpic_cross_entropy(x, w, t, b, want_lse=True)
            assert torch.equal(a, loss) and torch.equal(c, lse)
            gr = g.gpic_cross_entropy_backward(d, x, w, t, loss, lse, b)
            for name in ("dX", "dW", "db"):
                assert torch.equal(getattr(gr, name), getattr(ref, name))
    for kw in (dict(want_x=False), dict(want_w=False), dict(want_bias=False),
               dict(want_x=False, want_w=False), dict(want_w=False, want_bias=False),
               dict(want_x=False, want_w=False, want_bias=False)):
        part = g.gpic_cross_entropy_backward(d, X, W, t, loss, lse, b, **kw)
        for name, want in (("dX", "want_x"), ("dW", "want_w"), ("db", "want_bias")):
            if kw.get(want, True):
                assert torch.equal(getattr(part, name), getattr(ref, name))
            else:
                assert getattr(part, name) is None


@pytest.mark.parametrize("dtype", list(T))
def test_no_rows_and_padding_alone(g, dtype):
    X, W, b, t = _inputs(40, 24, 500, dtype)
    loss, lse = g.gpic_cross_entropy(X[:0], W, t[:0], b, want_lse=True)
    gr = g.gpic_cross_entropy_backward(loss, X[:0], W, t[:0], loss, lse, b)
    assert loss.shape == (0,) and gr.dX.shape == (0, 24)
    assert not gr.dW.any() and not gr.db.any()
    pad = torch.full_like(t, -100)
    loss, lse = g.gpic_cross_entropy(X, W, pad, b, want_lse=True)
    gr = g.gpic_cross_entropy_backward(torch.ones(40, device=DEV), X, W, pad, loss, lse, b)
    assert not loss.any() and not gr.dX.any() and not gr.dW.any() and not gr.db.any()


def test_targets_beyond_32_bits_are_padding(g):
    X, W, b, _ = _inputs(40, 24, 500, "f32")
    t = torch.arange(40, device=DEV) + 2 ** 32
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    assert not loss.any()
    gr = g.gpic_cross_entropy_backward(torch.ones(40, device=DEV), X, W, t, loss, lse, b)
    assert not gr.dX.any() and not gr.dW.any()


def test_gradients_against_differences(g):
    """float32: the loss moves as its gradients say along random directions."""
    n, k, v = 60, 40, 300
    X, W, b, t = _inputs(n, k, v, "f32")
    dloss = _randn((n,), "f32", 8)
    loss, lse = g.gpic_cross_entropy(X, W, t, b, want_lse=True)
    gr = g.gpic_cross_entropy_backward(dloss, X, W, t, loss, lse, b)
    h = 2.0 ** -7
    for which, (tensor, grad) in enumerate(((X, gr.dX), (W, gr.dW), (b, gr.db))):
        D = _randn(tuple(tensor.shape), "f32", 20 + which)
        D /= D.norm()
        values = []
        for s in (h, -h):
            a = [X, W, b]
            a[which] = tensor + s * D
            values.append((g.gpic_cross_entropy(a[0], a[1], t, a[2]).double() * dloss).sum())
        slope = float((values[0] - values[1]) / (2 * h))
        want = float((grad.double() * D).sum())
        # central differences: h^2 / 6 of a third derivative of a few units a row at
        # most, and the losses' float32 error (2e-6 each) over 2 h
        tol = h * h * float(dloss.abs().sum()) + 2e-6 * float(dloss.abs().sum()) / h
        assert abs(slope - want) <= tol, (which, slope, want, tol)


@pytest.mark.parametrize("n", [2, 40])
def test_weights_beyond_32_bits(g, n):
    """v k > 2^32 values of W and dW."""
    v, k = 1 << 20, 4120
    print(f"loss n={n} k={k} v={v}", flush=True)
    W = torch.empty((v, k), dtype=T["bf16"], device=DEV)
    for i in range(0, v, 65536):
        W[i:i + 65536] = _randn((65536, k), "bf16", i, k ** -0.5)
    X = _randn((n, k), "bf16", 1)
    t = torch.tensor([v - 1, 2 ** 32 // k + 1] * (n // 2), device=DEV)
    loss, lse = g.gpic_cross_entropy(X, W, t, want_lse=True)
    z = torch.cat([X.double() @ W[i:i + 65536].double().t() for i in range(0, v, 65536)], 1)
    full = z.logsumexp(1)
    # logits of size one: (K + 16) e of sum |x||w| (at most 70) each, weighted; 8,192 joins of
    # strips by 256 lanes (n = 2: 256 a lane) or 16 lanes, 4 e each
    tol = (k + 16) * E * 70 + 4 * (v / 256 / 16 + 40) * E + 4 * E * float(full.abs().max())
    _within(lse, full, torch.full_like(full, tol), "lse")
    _within(loss, full - z.gather(1, t[:, None])[:, 0], torch.full_like(full, 2 * tol), "loss")
    gr = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), X, W, t, loss, lse)
    rows = torch.tensor([0, 1, 2 ** 31 // k, 2 ** 32 // k - 1, 2 ** 32 // k, 2 ** 32 // k + 1, v - 2,
                         v - 1], device=DEV)
    d = (z - full[:, None]).exp()
    d[torch.arange(n, device=DEV), t] -= 1.0
    x = X.double()
    off = (U["bf16"] + 2 * tol) * d.abs()
    _close(gr.dW[rows], d[:, rows].t() @ x, (off[:, rows].t() + 60 * E * d[:, rows].abs().t()) @ x.abs(),
           "bf16", "dW")
    dX, size = torch.zeros((n, k), dtype=torch.float64, device=DEV), 0.0
    for i in range(0, v, 65536):
        w = W[i:i + 65536].double()
        dX += d[:, i:i + 65536] @ w
        size = size + d[:, i:i + 65536].abs() @ w.abs()
    # float32 sums of v products, of random sign: 4 sqrt(v) of their roundings at the most
    # likely worst, and one rounding of dZ each
    _close(gr.dX, dX, (U["bf16"] + 2 * tol + 4 * math.sqrt(v) * E) * size, "bf16", "dX")
    del W, gr, z, d
    torch.cuda.empty_cache()


def test_gradients_of_logits_beyond_32_bits(g):
    """A piece's dZ of more than 2^32 values: the rows on both sides of 2^31 and
    2^32, and the weights' gradient in chunks."""
    n, k, v = 2 ** 21 + 300, 24, 2100
    print(f"loss n={n} k={k} v={v}", flush=True)
    X, W = _randn((n, k), "bf16", 1), _randn((v, k), "bf16", 2, k ** -0.5)
    t = torch.arange(n, device=DEV) % v
    loss, lse = g.gpic_cross_entropy(X, W, t, want_lse=True)
    gr = g.gpic_cross_entropy_backward(torch.ones(n, device=DEV), X, W, t, loss, lse)
    w = W.double()
    rows = sorted({2 ** p // 2304 + d for p in (31, 32) for d in (-1, 0, 1)}
                  | {2 ** p // 2112 + d for p in (31, 32) for d in (-1, 0, 1) if 2 ** p // 2112 + d < n}
                  | {0, 1, n - 2, n - 1})
    z = X[rows].double() @ w.t()
    d = (z - z.logsumexp(1, keepdim=True)).exp()
    d[torch.arange(len(rows), device=DEV), t[rows]] -= 1.0
    _close(gr.dX[rows], d @ w, (U["bf16"] + 1e-5 + (v + 48) * E) * (d.abs() @ w.abs()), "bf16", "dX")
    dW, size = torch.zeros((v, k), dtype=torch.float64, device=DEV), 0.0
    for i in range(0, n, 100000):
        x = X[i:i + 100000].double()
        z = x @ w.t()
        d = (z - z.logsumexp(1, keepdim=True)).exp()
        d[torch.arange(len(x), device=DEV), t[i:i + 100000]] -= 1.0
        dW += d.t() @ x
        size = size + d.abs().t() @ x.abs()
    _close(gr.dW, dW, (U["bf16"] + 1e-5 + 4 * math.sqrt(n) * E) * size, "bf16", "dW")
