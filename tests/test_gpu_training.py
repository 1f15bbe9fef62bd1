"""Layer norm, embedding table and dropout on the GPU against plain float64
formulas, where they can go wrong: no rows, one row, one column, odd widths,
rows longer than a workgroup holds, views, non-finite rows, padding, tokens
of every frequency.

Tolerances (u: half a unit in the last place of the type, e = 2^-24): a
float32 sum of which no term passes through more than D additions is off by
at most D e sum|terms|.  Norm: a lane adds at least every sixteenth value of
a row, so D <= k / 16 + 32 with the lanes' join and the roundings of the
terms; the mean is kept in float32 (2 e |mean|).  Column sums: at most n / 64
+ 32 rows one after another.  Table: at most 256 + 32 rows one after another,
or 64 and a sixteenth of the cuts.  Results are rounded once."""
import math

import numpy as np
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


def _close(got, ref, bound, dtype, what):
    assert got.shape == ref.shape and got.dtype == T[dtype]
    err = (got.double() - ref).abs()
    tol = bound + U[dtype] * (ref.abs() + bound) + TINY[dtype]
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, float((err / tol).nan_to_num(nan=9e9).max()),
                                 int(bad.sum()))


# ------------------------------------------------------------------- norm
def _norm_check(g, X, w, b, dY, dtype, what, eps=1e-5):
    n, k = X.shape
    Y, stats = g.gpic_layer_norm(X, w, b, eps, want_stats=True)
    assert torch.equal(Y, g.gpic_layer_norm(X, w, b, eps))
    x, dy = X.double(), dY.double()
    wd = w.double() if w is not None else torch.ones(k, device=DEV, dtype=torch.float64)
    bd = b.double() if b is not None else torch.zeros(k, device=DEV, dtype=torch.float64)
    mean = x.mean(1, keepdim=True)
    r = 1.0 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    h = (x - mean) * r
    D = (k / 16 + 32) * E
    # What the mean's error moves h by.  The mean is m0 + fl(sum d) / k with d = fl(x - m0):
    # each d is off by E |d|, their float32 sum by at most D sum |d|, so the mean of d by
    # (D + E) mean |d| <= (D + E) / r (the mean of |h| is at most 1), and m0 plus it, times
    # fl(1 / k), is rounded to 2 E |mean|.
    off = 2 * E * mean.abs() + (D + E) / r
    hm = r * off
    _close(Y, h * wd + bd, (D * h.abs() + hm) * wd.abs() + 2 * E * bd.abs(), dtype, what + " Y")
    assert bool(((stats[:, 0:1].double() - mean).abs() <= off).all())
    assert float(((stats[:, 1:2].double() - r).abs() / r).max()) <= D

    gr = g.gpic_layer_norm_backward(dY, X, w, stats)
    G = dy * wd
    s1, s2 = G.mean(1, keepdim=True), (G * h).mean(1, keepdim=True)
    a1, a2 = G.abs().mean(1, keepdim=True), (G * h).abs().mean(1, keepdim=True)
    bound = r * (2 * D * (G.abs() + a1 + h.abs() * a2 * 2) + hm * a2 + h.abs() * hm * a1)
    _close(gr.dX, r * (G - s1 - h * s2), bound, dtype, what + " dX")
    Dn = (n / 64 + 32) * E
    _close(gr.dW, (dy * h).sum(0),
           Dn * (dy * h).abs().sum(0) + (dy.abs() * (D * h.abs() + hm)).sum(0), dtype, what + " dW")
    _close(gr.db, dy.sum(0), Dn * dy.abs().sum(0), dtype, what + " db")
    for kw in (dict(want_x=False), dict(want_w=False), dict(want_bias=False),
               dict(want_x=False, want_w=False)):
        part = g.gpic_layer_norm_backward(dY, X, w, stats, **kw)
        for name, want in (("dX", "want_x"), ("dW", "want_w"), ("db", "want_bias")):
            if kw.get(want, True):
                assert torch.equal(getattr(part, name), getattr(gr, name))
            else:
                assert getattr(part, name) is None


NORMS = [(1, 1), (1, 2048), (3, 7), (5, 64), (1, 8192), (17, 129), (300, 8), (1003, 300),
         (4100, 512), (5000, 40), (2100, 1000), (1030, 2048), (777, 2049), (513, 4100), (70, 8200),
         (9, 33000), (3, 100001), (40000, 24),
         (140000, 30), (9001, 3), (70001, 33), (300, 64)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_norm_and_gradients(g, shape, dtype):
    n, k = shape
    print(f"norm n={n} k={k} {dtype}", flush=True)
    X = (_randn((n, k), dtype, 1).float() * (1 + _randn((n, 1), "f32", 2).abs())
         + 3 * _randn((n, 1), "f32", 3)).to(T[dtype])
    w = (1 + _randn((k,), "f32", 4, 0.3)).to(T[dtype])
    b = _randn((k,), dtype, 5)
    dY = _randn((n, k), dtype, 6, 0.01)
    _norm_check(g, X, w, b, dY, dtype, "norm")
    if n < 2000:
        _norm_check(g, X, None, None, dY, dtype, "plain norm", eps=1e-3)
        _norm_check(g, X, w, None, dY, dtype, "norm without bias")


@pytest.mark.parametrize("dtype", list(T))
def test_norm_far_from_zero(g, dtype):
    """Rows whose mean is 2^7 times their spread keep their digits."""
    X = (128 + _randn((65, 1000), "f32", 1)).to(T[dtype])
    w, b, dY = _randn((1000,), dtype, 2), _randn((1000,), dtype, 3), _randn((65, 1000), dtype, 4)
    _norm_check(g, X, w, b, dY, dtype, "far")


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("k", [24, 1000, 2048, 4104])
def test_norm_views_in_place_and_alignment(g, k, dtype):
    n = 70
    table = _randn((n, k + 24), dtype, 1)
    X = table[:, 8:8 + k]
    w, b, dY = _randn((k,), dtype, 2), _randn((k,), dtype, 3), _randn((n, k + 5), dtype, 4)[:, 3:3 + k]
    ref, stats = g.gpic_layer_norm(X.contiguous(), w, b, want_stats=True)
    assert torch.equal(g.gpic_layer_norm(X, w, b), ref)
    off = torch.empty(n * k + 1, dtype=T[dtype], device=DEV)[1:].view(n, k)
    off.copy_(X)
    assert torch.equal(g.gpic_layer_norm(off, w, b), ref)
    assert torch.equal(g.gpic_layer_norm(X.t().contiguous().t(), w, b), ref)
    a = g.gpic_layer_norm_backward(dY, X, w, stats)
    c = g.gpic_layer_norm_backward(dY.contiguous(), X.contiguous(), w, stats)
    assert torch.equal(a.dX, c.dX) and torch.equal(a.dW, c.dW) and torch.equal(a.db, c.db)
    before = table.clone()
    assert g.gpic_layer_norm(X, w, b, Y=X) is X
    assert torch.equal(X, ref)
    assert torch.equal(table[:, :8], before[:, :8]) and torch.equal(table[:, 8 + k:], before[:, 8 + k:])


@pytest.mark.parametrize("dtype", list(T))
def test_norm_non_finite_rows_and_no_rows(g, dtype):
    X, w, b = _randn((40, 300), dtype, 1), _randn((300,), dtype, 2), _randn((300,), dtype, 3)
    ref = g.gpic_layer_norm(X, w, b)
    bad = X.clone()
    bad[3, 7], bad[20, 299] = math.inf, math.nan
    Y = g.gpic_layer_norm(bad, w, b)
    assert bool(Y[[3, 20]].isnan().all())
    keep = [i for i in range(40) if i not in (3, 20)]
    assert torch.equal(Y[keep], ref[keep])
    # a constant row is all deviation zero: the bias
    same = torch.full((2, 300), 5.0, dtype=T[dtype], device=DEV)
    assert torch.equal(g.gpic_layer_norm(same, w, b), b.expand(2, 300))
    none = X[:0]
    Y, stats = g.gpic_layer_norm(none, w, b, want_stats=True)
    assert Y.shape == (0, 300)
    gr = g.gpic_layer_norm_backward(none, none, w, stats)
    assert gr.dX.shape == (0, 300) and not gr.dW.any() and not gr.db.any()


# -------------------------------------------------------------- embedding
def _table_check(g, n, k, rows, ids, dtype, scale, what):
    Tb, dY = _randn((rows, k), dtype, 1), _randn((n, k), dtype, 2)
    real = (ids >= 0) & (ids < rows)
    at = ids.clamp(0, rows - 1).long()
    Y = g.gpic_embedding(ids, Tb, scale)
    y = torch.where(real[:, None], Tb.double()[at] * scale, 0.0)
    _close(Y, y, 2 * E * y.abs(), dtype, what + " Y")
    wide = _randn((n, k + 4), dtype, 4)
    kept = wide.clone()
    table = torch.cat([Tb, Tb], 1)[:, :k] if k < 2000 else Tb          # a pitch of 2 k
    g.gpic_embedding(ids, table, scale, Y=wide[:, 3:3 + k])
    assert torch.equal(wide[:, 3:3 + k], Y) and torch.equal(wide[:, :3], kept[:, :3])
    assert torch.equal(wide[:, 3 + k:], kept[:, 3 + k:])
    dT = g.gpic_embedding_backward(dY, ids, rows, scale)
    d = torch.where(real[:, None], dY.double(), 0.0)
    zero = torch.zeros((rows, k), device=DEV, dtype=torch.float64)
    ref, size = zero.index_add(0, at, d), zero.index_add(0, at, d.abs())
    count = torch.bincount(at[real], minlength=rows).double()[:, None]
    bound = (count.clamp(max=256) + count / 1024 + 32) * E * size * abs(scale)
    _close(dT, ref * scale, bound, dtype, what + " dT")
    assert not bool(dT[(count == 0).squeeze(1)].any())
    assert torch.equal(dT, g.gpic_embedding_backward(dY, ids, rows, scale))
    old = _randn((rows, k + 3), dtype, 3)
    acc = old.clone()
    view = acc[:, 2:2 + k]
    assert g.gpic_embedding_backward(dY, ids, rows, scale, dT=view, accumulate=True) is view
    total = old[:, 2:2 + k].double() + ref * scale
    _close(view, total, bound + 2 * E * (total.abs() + (ref * scale).abs()), dtype, what + " sum")
    empty = (count == 0).squeeze(1)
    assert torch.equal(acc[empty], old[empty])
    into = old.clone()                       # every row written, nothing beside them
    g.gpic_embedding_backward(dY, ids, rows, scale, dT=into[:, 1:1 + k])
    assert torch.equal(into[:, 1:1 + k], dT)
    assert torch.equal(into[:, :1], old[:, :1]) and torch.equal(into[:, 1 + k:], old[:, 1 + k:])
    assert torch.equal(acc[:, :2], old[:, :2]) and torch.equal(acc[:, 2 + k:], old[:, 2 + k:])


TABLES = [(1, 1, 1), (1, 2048, 50), (3, 7, 5), (64, 64, 3), (65, 8, 1000), (1000, 300, 77),
          (1024, 40, 30000), (1025, 40, 30000), (1100, 1, 2), (4096, 9, 255), (4097, 513, 256),
          (5000, 1030, 700), (70000, 72, 9), (40000, 16, 70000), (70001, 520, 3001),
          (20000, 100, 2), (9000, 257, 3), (30000, 3, 4)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", TABLES, ids=str)
def test_embedding_and_gradient(g, shape, dtype):
    n, k, rows = shape
    print(f"embedding n={n} k={k} rows={rows} {dtype}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(n)
    u = torch.rand(n, device=DEV, generator=gen, dtype=torch.float64)
    zipf = (torch.exp(u * math.log(rows + 1.0)).long() - 1).clamp(0, rows - 1)
    _table_check(g, n, k, rows, zipf, dtype, 1.0, "zipf")
    uniform = (u * rows).long()
    uniform[torch.rand(n, device=DEV, generator=gen) < 0.1] = -100
    uniform[n // 2] = rows                               # just outside
    _table_check(g, n, k, rows, uniform.int(), dtype, -2.5, "uniform")
    _table_check(g, n, k, rows, torch.full((n,), rows // 2, device=DEV), dtype, 0.5, "one")
    _table_check(g, n, k, rows, torch.full((n,), -1, device=DEV), dtype, 1.0, "padding")


@pytest.mark.parametrize("n", [1500, 9000])
@pytest.mark.parametrize("lengths", [(64,), (65,), (63, 65, 64, 128, 129), (1, 200, 64, 1)], ids=str)
def test_embedding_runs_at_chunk_edges(g, n, lengths):
    """Runs that start and end on, before and after multiples of 64."""
    ids, v = [], 0
    while len(ids) < n:
        for m in lengths:
            ids += [v] * m
            v += 2
    ids = torch.tensor(ids[:n], device=DEV)
    perm = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(DEV)
    _table_check(g, n, 33, v + 1, ids, "f32", 1.0, "in order")
    _table_check(g, n, 33, v + 1, ids[perm], "bf16", 1.0, "shuffled")


def test_embedding_ids_beyond_32_bits_are_padding(g):
    Tb = _randn((5, 8), "f32", 1)
    ids = torch.tensor([2 ** 32 + 1, -2 ** 32, 4, 2 ** 62, -2 ** 63], device=DEV)
    Y = g.gpic_embedding(ids, Tb)
    assert torch.equal(Y[2], Tb[4]) and not Y[[0, 1, 3, 4]].any()
    for n in (5, 2000):
        many = ids.repeat(n // 5)
        dT = g.gpic_embedding_backward(torch.ones((n, 8), device=DEV), many, 5)
        assert not dT[:4].any() and bool((dT[4] == n // 5).all())


def test_embedding_keeps_non_finite_rows_apart(g):
    dY = _randn((3000, 24), "f32", 1)
    ids = torch.arange(3000, device=DEV) % 30
    ref = g.gpic_embedding_backward(dY, ids, 40)
    dY[31] = math.nan
    dT = g.gpic_embedding_backward(dY, ids, 40)
    assert bool(dT[1].isnan().all())
    keep = [i for i in range(40) if i != 1]
    assert torch.equal(dT[keep], ref[keep])


# ---------------------------------------------------------------- dropout
def _philox(counter, key):
    c, (k0, k1) = list(counter), key
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k0, b & 0xffffffff, (a >> 32) ^ c[3] ^ k1, a & 0xffffffff]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return c


def _bits(first, count, seed, offset):
    """The 16 bits of values first .. first + count - 1."""
    out = []
    block = None
    for i in range(first, first + count):
        if block is None or i % 8 == 0:
            b = i // 8
            block = _philox((b & 0xffffffff, b >> 32, offset & 0xffffffff, offset >> 32),
                            (seed & 0xffffffff, seed >> 32))
        out.append(block[i % 8 // 2] >> (16 * (i % 2)) & 0xffff)
    return np.array(out)


def test_philox_of_the_paper():
    """The published answers of Philox4x32-10."""
    assert _philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 0xffffffff
    assert _philox((f, f, f, f), (f, f)) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (1, 2048), (3, 5), (9, 11), (40, 24), (33, 129),
                                   (2, 1000)], ids=str)
def test_dropout(g, shape, dtype):
    n, m = shape
    X, R = _randn((n, m), dtype, 1), _randn((n, m), dtype, 2)
    wide = _randn((n, m + 9), dtype, 1)
    for p, seed, offset in ((0.0, 0, 0), (0.1, 5, 7), (0.5, 2 ** 64 - 1, 2 ** 64 - 1),
                            (0.9, 2 ** 33 + 1, 2 ** 40)):
        limit = round(p * 65536)
        keep = torch.from_numpy(_bits(0, n * m, seed, offset) >= limit).view(n, m).to(DEV)
        scale = 65536.0 / (65536 - limit)
        for x in (X, wide[:, 4:4 + m]):
            for r in (None, R):
                y = torch.where(keep, x.double() * scale, 0.0) + (0 if r is None else r.double())
                Y = g.gpic_dropout(x, p, seed, offset, residual=r)
                bound = 3 * E * (x.double().abs() * scale + y.abs())
                _close(Y, y, bound, dtype, f"dropout {p}")
                assert torch.equal((Y == 0) & (x != 0), ~keep) or r is not None
    assert torch.equal(g.gpic_dropout(X, 0.0, 3), X)
    # in place, over X and over the residual
    ref = g.gpic_dropout(X, 0.3, 3, 4, residual=R)
    x, r = X.clone(), R.clone()
    assert g.gpic_dropout(X, 0.3, 3, 4, residual=r, Y=r) is r and torch.equal(r, ref)
    assert g.gpic_dropout(x, 0.3, 3, 4, residual=R, Y=x) is x and torch.equal(x, ref)


def test_dropout_mask_depends_on_the_index_alone(g):
    """One mask for every type, pitch and shape of a run of values; another
    for another seed, offset or step; a share of p of it dropped."""
    n, m, p = 1003, 777, 0.1
    one = torch.ones((n, m), device=DEV)
    base = g.gpic_dropout(one, p, 11, 3)
    for x in (one.half(), one.bfloat16(), torch.ones((n, m + 3), device=DEV)[:, 1:1 + m],
              torch.ones((n, m + 3), device=DEV).bfloat16()[:, :m]):
        assert torch.equal(g.gpic_dropout(x, p, 11, 3) != 0, base != 0)
    flat = g.gpic_dropout(one.view(1, n * m), p, 11, 3)
    assert torch.equal(flat.view(n, m), base)
    step = torch.tensor([2], device=DEV)
    assert torch.equal(g.gpic_dropout(one, p, 11, 1, step=step), base)
    for seed, offset in ((12, 3), (11, 4), (11 + 2 ** 32, 3), (11, 3 + 2 ** 32)):
        other = g.gpic_dropout(one, p, seed, offset)
        both = float(((other == 0) & (base == 0)).double().mean())
        # two independent masks: p^2, within six deviations
        assert abs(both - p * p) <= 6 * math.sqrt(p * p / (n * m))
    share = float((base == 0).double().mean())
    assert abs(share - p) <= 6 * math.sqrt(p * (1 - p) / (n * m)) + 2.0 ** -17
    assert abs(float(base.double().mean()) - 1.0) <= 6 * math.sqrt(p / (1 - p) / (n * m))


def test_dropout_drops_non_finite_values(g):
    x = torch.full((5, 100), math.nan, device=DEV)
    x[1::2] = math.inf
    y = g.gpic_dropout(x, 0.5, 1)
    keep = torch.from_numpy(_bits(0, 500, 1, 0) >= 32768).view(5, 100).to(DEV)
    assert not y[~keep].any() and not bool(y[keep].isfinite().any())
    assert g.gpic_dropout(x[:0], 0.5, 1).shape == (0, 100)


@pytest.mark.parametrize("pitched", [False, True])
def test_dropout_beyond_32_bits(g, pitched):
    """The last values of 2^32 + 4,099: counters and offsets past 32 bits."""
    n, m = 65536, 65537
    if pitched:
        X = torch.ones((n, m + 7), dtype=torch.bfloat16, device=DEV)[:, 3:3 + m]
    else:
        X = torch.ones((n, m), dtype=torch.bfloat16, device=DEV)
    Y = g.gpic_dropout(X, 0.5, 9, 1)
    tail = Y[-1, -4000:].cpu()
    want = _bits(n * m - 4000, 4000, 9, 1) >= 32768
    assert np.array_equal((tail != 0).numpy(), want)
    assert bool((tail[torch.from_numpy(want)] == 2).all())
    del X, Y
    torch.cuda.empty_cache()


# ------------------------------------------------- beyond 32 bits of values
def _filled(shape, dtype, seed):
    t = torch.empty(shape, dtype=T[dtype], device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    for i in range(0, shape[0], 16384):
        t[i:i + 16384] = torch.randn((min(16384, shape[0] - i), shape[1]), device=DEV,
                                     generator=gen).to(t.dtype)
    return t


def test_norm_beyond_32_bits(g):
    """n k > 2^32: the rows on both sides of 2^31 and 2^32 values, and the last."""
    n, k = 1050000, 4100
    print(f"norm n={n} k={k}", flush=True)
    X, dY = _filled((n, k), "bf16", 1), _filled((n, k), "bf16", 2)
    w, b = (1 + _randn((k,), "f32", 3, 0.2)).to(T["bf16"]), _randn((k,), "bf16", 4)
    Y, stats = g.gpic_layer_norm(X, w, b, want_stats=True)
    gr = g.gpic_layer_norm_backward(dY, X, w, stats)
    rows = [0, 1, 2 ** 31 // k - 1, 2 ** 31 // k, 2 ** 31 // k + 1, 2 ** 32 // k - 1, 2 ** 32 // k,
            2 ** 32 // k + 1, n - 2, n - 1]
    x, dy = X[rows].contiguous(), dY[rows].contiguous()
    ref, s = g.gpic_layer_norm(x, w, b, want_stats=True)
    assert torch.equal(Y[rows], ref) and torch.equal(stats[rows], s)
    assert torch.equal(gr.dX[rows], g.gpic_layer_norm_backward(dy, x, w, s).dX)
    db, size = (torch.zeros(k, dtype=torch.float64, device=DEV) for _ in range(2))
    for i in range(0, n, 50000):
        d = dY[i:i + 50000].double()
        db, size = db + d.sum(0), size + d.abs().sum(0)
    # (rows of a wave: n / 512 one after another at most)
    _close(gr.db, db, (n / 512 + 32) * E * size, "bf16", "db")
    del X, dY, Y, gr
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [100, 5000])
def test_embedding_beyond_32_bits(g, n):
    """A table and its gradient of more than 2^32 values."""
    rows, k = 140000, 32768
    print(f"embedding n={n} rows={rows} k={k}", flush=True)
    Tb = torch.zeros((rows, k), dtype=T["bf16"], device=DEV)
    some = torch.tensor([0, 1, 2 ** 31 // k - 1, 2 ** 31 // k, 2 ** 32 // k - 1, 2 ** 32 // k,
                         2 ** 32 // k + 1, rows - 2, rows - 1], device=DEV)
    Tb[some] = _randn((len(some), k), "bf16", 1)
    ids = some[torch.arange(n, device=DEV) % len(some)]
    assert torch.equal(g.gpic_embedding(ids[:20], Tb), Tb[ids[:20]])
    dY = _randn((n, k), "bf16", 2)
    dT = Tb                            # every row is written
    dT.fill_(5.0)
    g.gpic_embedding_backward(dY, ids, rows, dT=dT)
    for i, v in enumerate(some.tolist()):
        d = dY[i::len(some)].double()
        _close(dT[v], d.sum(0), (min(len(d), 512) + 64) * E * d.abs().sum(0), "bf16", f"row {v}")
    total = sum(float(dT[i:i + 10000].abs().sum(dtype=torch.float64)) for i in range(0, rows, 10000))
    kept = float(dT[some].abs().sum(dtype=torch.float64))
    assert abs(total - kept) <= 1e-9 * kept          # the other rows are zeros
    del Tb, dT
    torch.cuda.empty_cache()


def test_embedding_of_many_ids_beyond_32_bits(g):
    """n k > 2^32 values of Y and dY."""
    n, k, rows = 2 ** 23 + 4099, 512, 3000
    print(f"embedding n={n} k={k}", flush=True)
    Tb = _randn((rows, k), "bf16", 1)
    ids = torch.arange(n, device=DEV, dtype=torch.int32) % rows
    Y = g.gpic_embedding(ids, Tb)
    at = [0, 2 ** 22 - 1, 2 ** 22, 2 ** 23 - 1, 2 ** 23, n - 1]
    assert torch.equal(Y[at], Tb[[i % rows for i in at]])
    # every row of dY one value: sums of up to 2,798 whole numbers are exact
    Y.copy_(((torch.arange(n, device=DEV) // rows) % 2).to(Y.dtype)[:, None].expand(n, k))
    dT = g.gpic_embedding_backward(Y, ids, rows)
    count = torch.bincount(ids.long(), weights=((torch.arange(n, device=DEV) // rows) % 2).double(),
                           minlength=rows)
    assert torch.equal(dT.double(), count.to(T["bf16"]).double()[:, None].expand(rows, k))
    del Y
    torch.cuda.empty_cache()
