"""The calls around an encoder's layers together with the layers, as a training
step uses them: a table that is both the input's and the loss's, norms, a gated
block with dropout before its residual, the loss and every gradient; on another
stream, in replayed graphs, with scratch memory of any contents, and beside
autograd."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
P, SEED = 0.2, 77


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return g


def _randn(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=gen) * scale).to(T[dtype])


def _weights(dtype, v=301, k=96, m=136):
    return {"table": _randn((v, k), dtype, 1, 0.3), "n1": (1 + _randn((k,), "f32", 2, 0.2)).to(T[dtype]),
            "b1": _randn((k,), dtype, 3, 0.1), "gate": _randn((2 * m, k), dtype, 4, k ** -0.5),
            "down": _randn((k, m), dtype, 5, m ** -0.5),
            "n2": (1 + _randn((k,), "f32", 6, 0.2)).to(T[dtype]), "b2": _randn((k,), dtype, 7, 0.1),
            "bias": _randn((v,), dtype, 8, 0.2)}


def _tokens(n=130, v=301):
    gen = torch.Generator(device=DEV).manual_seed(9)
    u = torch.rand((2, n), device=DEV, generator=gen, dtype=torch.float64)
    ids, targets = ((torch.exp(u * math.log(v + 1.0)).long() - 1).clamp(0, v - 1)).unbind(0)
    ids, targets = ids.clone(), targets.clone()
    ids[5] = targets[11] = targets[12] = -100
    return ids, targets


def _step(g, w, ids, targets, scale=1.0, step=None):
    """Losses and the gradients of their sum times `scale`, with the package."""
    x = g.gpic_embedding(ids, w["table"], 2.0)
    h, s1 = g.gpic_layer_norm(x, w["n1"], w["b1"], want_stats=True)
    a, z = g.gpic_gated(h, w["gate"], want_pre=True)
    d = g.gpic_linear(a, w["down"])
    y = g.gpic_dropout(d, P, SEED, 3, residual=x, step=step)
    f, s2 = g.gpic_layer_norm(y, w["n2"], w["b2"], want_stats=True)
    loss, lse = g.gpic_cross_entropy(f, w["table"], targets, w["bias"], want_lse=True)
    dloss = torch.full_like(loss, scale)
    gl = g.gpic_cross_entropy_backward(dloss, f, w["table"], targets, loss, lse, w["bias"])
    g2 = g.gpic_layer_norm_backward(gl.dX, y, w["n2"], s2)
    dd = g.gpic_dropout(g2.dX, P, SEED, 3, step=step)
    gd = g.gpic_linear_backward(dd, a, w["down"], want_bias=False)
    gg = g.gpic_gated_backward(gd.dX, h, w["gate"], z)
    g1 = g.gpic_layer_norm_backward(gg.dX, x, w["n1"], s1)
    dx = g1.dX + g2.dX
    g.gpic_embedding_backward(dx, ids, w["table"].shape[0], 2.0, dT=gl.dW, accumulate=True)
    return {"loss": loss, "table": gl.dW, "bias": gl.db, "n2": g2.dW, "b2": g2.db, "down": gd.dW,
            "gate": gg.dW, "n1": g1.dW, "b1": g1.db}


def _reference(w, ids, targets, keep):
    """The same in float64 with torch's autograd."""
    w = {k: v.detach().double().requires_grad_() for k, v in w.items()}

    def norm(x, weight, bias):
        m = x.mean(1, keepdim=True)
        return (x - m) / ((x - m).square().mean(1, keepdim=True) + 1e-5).sqrt() * weight + bias

    real = (ids >= 0)[:, None]
    x = torch.where(real, w["table"][ids.clamp(min=0)] * 2.0, 0.0)
    h = norm(x, w["n1"], w["b1"])
    m = w["gate"].shape[0] // 2
    zg, zu = h @ w["gate"][:m].t(), h @ w["gate"][m:].t()
    d = (zg * torch.sigmoid(zg) * zu) @ w["down"].t()
    y = x + torch.where(keep, d * (65536.0 / (65536 - round(P * 65536))), 0.0)
    f = norm(y, w["n2"], w["b2"])
    z = f @ w["table"].t() + w["bias"]
    loss = z.logsumexp(1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    loss = torch.where(targets >= 0, loss, 0.0)
    loss.sum().backward()
    out = {k: v.grad for k, v in w.items()}
    out["loss"] = loss.detach()
    return out


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [130, 2500])
def test_a_training_step(g, n, dtype):
    """float32: a chain of twenty products and sums of up to 301 terms, each off
    by (301 + 32) 2^-24 of its terms at most: 4e-4 of the 2-norm; 16 bits: about
    twenty roundings of 2^-9 (2^-12) on average, of random sign, on the way to a
    gradient: 4.5 of them, and as much again for the slopes."""
    w = _weights(dtype)
    ids, targets = _tokens(n)
    print(f"training step n={n} {dtype}", flush=True)
    got = _step(g, w, ids, targets)
    keep = g.gpic_dropout(torch.ones((n, 96), device=DEV), P, SEED, 3) != 0
    ref = _reference(w, ids, targets, keep)
    tol = {"f32": 4e-4, "f16": 9 * 2.0 ** -12, "bf16": 9 * 2.0 ** -9}[dtype]
    for name, r in ref.items():
        err = float((got[name].double() - r).norm() / r.norm())
        assert err <= tol, (name, err)


def test_step_against_differences(g):
    """The sum of the losses moves as the gradients say."""
    w = _weights("f32")
    ids, targets = _tokens()
    grads = _step(g, w, ids, targets)
    h = 2.0 ** -9
    for i, name in enumerate(w):
        D = _randn(tuple(w[name].shape), "f32", 30 + i)
        D /= D.norm()
        value = [_step(g, {**w, name: w[name] + s * D}, ids, targets)["loss"].double().sum()
                 for s in (h, -h)]
        slope, want = float((value[0] - value[1]) / (2 * h)), float((grads[name].double() * D).sum())
        # 130 losses, each off by 2e-6 at most, over 2 h; central differences: h^2
        # times a third derivative, for which the norms' stand: 1e3 a gradient's size
        tol = 130 * 2e-6 / h + 1e3 * h * h * float(grads[name].norm())
        assert abs(slope - want) <= tol, (name, slope, want, tol)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [130, 2500])
def test_results_do_not_depend_on_the_buffers(g, monkeypatch, n, dtype):
    from gpu_helpers import Filled
    w = _weights(dtype)
    ids, targets = _tokens(n)
    runs = []
    for x in (0.0, 1e300):
        print(f"scratch {x} n={n} {dtype}", flush=True)
        with monkeypatch.context() as mp:
            mp.setattr(g, "torch", Filled(x))
            runs.append(_step(g, w, ids, targets))
        torch.cuda.synchronize()
    for name in runs[0]:
        assert torch.equal(runs[0][name], runs[1][name]), name


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("n", [130, 2500])
def test_streams_and_graph_replays(g, n, dtype):
    w = _weights(dtype)
    ids, targets = _tokens(n)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    eager = {k: v.clone() for k, v in _step(g, w, ids, targets, step=step).items()}
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    both = []
    for s in (a, b):                       # two calls at once
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            both.append(_step(g, w, ids, targets, step=step))
    torch.cuda.synchronize()
    for one in both:
        for name in eager:
            assert torch.equal(one[name], eager[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        out = _step(g, w, ids, targets, step=step)
        step.add_(1)
    step.zero_()
    for i in range(4):
        ids.copy_(ids.roll(3))
        w["gate"].mul_(0.9)
        now = torch.full_like(step, i)
        want = _step(g, w, ids, targets, step=now)
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == i + 1
        for name in want:
            assert torch.equal(out[name], want[name]), (i, name)


def _t(*shape, dtype=torch.float32):
    return torch.ones(shape, device=DEV, dtype=dtype)


def _calls(g):
    """name of the operand -> a call that takes the tensor there"""
    X, v, ids, s = _t(5, 8), _t(8), torch.zeros(5, dtype=torch.int64, device=DEV), _t(5, 2)
    one = _t(5)
    return {
        "X": ((5, 8), lambda t: g.gpic_layer_norm(t)), "weight": ((8,), lambda t: g.gpic_layer_norm(X, t)),
        "bias": ((8,), lambda t: g.gpic_layer_norm(X, None, t)),
        "Y": ((5, 8), lambda t: g.gpic_layer_norm(X, Y=t)),
        "dY": ((5, 8), lambda t: g.gpic_layer_norm_backward(t, X, v, s)),
        "drop X": ((5, 8), lambda t: g.gpic_dropout(t, 0.1, 1)),
        "residual": ((5, 8), lambda t: g.gpic_dropout(X, 0.1, 1, residual=t)),
        "T": ((5, 8), lambda t: g.gpic_embedding(ids, t)),
        "table dY": ((5, 8), lambda t: g.gpic_embedding_backward(t, ids, 5)),
        "dT": ((5, 8), lambda t: g.gpic_embedding_backward(X, ids, 5, dT=t)),
        "loss X": ((5, 8), lambda t: g.gpic_cross_entropy(t, X, ids)),
        "W": ((5, 8), lambda t: g.gpic_cross_entropy(X, t, ids)),
        "dloss": ((5,), lambda t: g.gpic_cross_entropy_backward(t, X, X, ids, one, one)),
    }


def test_tensors_that_require_gradients_are_refused(g):
    for name, (shape, call) in _calls(g).items():
        with pytest.raises(ValueError, match="requires gradients"):
            call(_t(*shape).requires_grad_())
        with torch.no_grad():
            call(_t(*shape).requires_grad_())
        call(_t(*shape))


def test_writes_in_place_are_counted(g):
    X, ids = _t(5, 8), torch.zeros(5, dtype=torch.int64, device=DEV)
    for call in (lambda t: g.gpic_layer_norm(X, Y=t), lambda t: g.gpic_dropout(X, 0.1, 1, Y=t),
                 lambda t: g.gpic_embedding(ids, X, Y=t),
                 lambda t: g.gpic_embedding_backward(X, ids, 5, dT=t)):
        t = _t(5, 8)
        before = t._version
        call(t)
        assert t._version > before


def test_binding_refusals(g):
    X, ids, s = _t(5, 8), torch.zeros(5, dtype=torch.int64, device=DEV), _t(5, 2)
    one = _t(5)
    bad = [
        (ValueError, lambda: g.gpic_layer_norm(_t(8))),
        (TypeError, lambda: g.gpic_layer_norm(X.double())),
        (ValueError, lambda: g.gpic_layer_norm(X, _t(7))),
        (TypeError, lambda: g.gpic_layer_norm(X, _t(8).half())),
        (ValueError, lambda: g.gpic_layer_norm(X, Y=_t(8, 5).t())),
        (g.GpicError, lambda: g.gpic_layer_norm(X, eps=-1.0)),
        (ValueError, lambda: g.gpic_layer_norm_backward(X, X, None, _t(5, 3))),
        (TypeError, lambda: g.gpic_layer_norm_backward(X, X, None, s.double())),
        (ValueError, lambda: g.gpic_layer_norm_backward(_t(5, 7), X, None, s)),
        (g.GpicError, lambda: g.gpic_dropout(X, 1.0, 1)),
        (g.GpicError, lambda: g.gpic_dropout(X, -0.1, 1)),
        (ValueError, lambda: g.gpic_dropout(X, 0.1, -1)),
        (ValueError, lambda: g.gpic_dropout(X, 0.1, 1, 1 << 64)),
        (ValueError, lambda: g.gpic_dropout(X, 0.1, 1, residual=_t(5, 7))),
        (TypeError, lambda: g.gpic_dropout(X, 0.1, 1, step=_t(1))),
        (ValueError, lambda: g.gpic_dropout(X, 0.1, 1, step=ids)),
        (g.GpicError, lambda: g.gpic_dropout(X[:4], 0.1, 1, Y=X[1:])),
        (TypeError, lambda: g.gpic_embedding(one, X)),
        (ValueError, lambda: g.gpic_embedding(ids.view(5, 1), X)),
        (TypeError, lambda: g.gpic_embedding(ids, ids.view(1, 5))),
        (g.GpicError, lambda: g.gpic_embedding(ids, X, float("nan"))),
        (ValueError, lambda: g.gpic_embedding_backward(X, ids[:4], 5)),
        (ValueError, lambda: g.gpic_embedding_backward(X, ids, 5, accumulate=True)),
        (ValueError, lambda: g.gpic_embedding_backward(X, ids, 5, dT=_t(4, 8))),
        (g.GpicError, lambda: g.gpic_embedding_backward(X, ids, 0)),
        (g.GpicError, lambda: g.gpic_embedding_backward(X, ids, 5, dT=X)),
        (ValueError, lambda: g.gpic_cross_entropy(X, _t(5, 7), ids)),
        (TypeError, lambda: g.gpic_cross_entropy(X, X.half(), ids)),
        (ValueError, lambda: g.gpic_cross_entropy(X, X, ids[:3])),
        (ValueError, lambda: g.gpic_cross_entropy(X, X, ids, _t(4))),
        (ValueError, lambda: g.gpic_cross_entropy_backward(_t(4), X, X, ids, one, one)),
        (TypeError, lambda: g.gpic_cross_entropy_backward(one.half(), X, X, ids, one, one)),
        (ValueError, lambda: g.gpic_cross_entropy_backward(one, X, X, ids, one, _t(6))),
    ]
    for i, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"case {i} was accepted")
