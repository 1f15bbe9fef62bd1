"""The encoder's operators beside autograd: they record no gradients, so a
tensor that would expect them is refused instead of its graph being cut, and
what they write in place is known to autograd, which refuses a backward pass
over values that are no longer there."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    return g


def _t(*shape):
    return torch.ones(shape, device=DEV)


def _calls(g):
    """name of the operand -> a call that takes the tensor there"""
    X, W, W2, V = _t(5, 8), _t(6, 8), _t(12, 8), _t(5, 6)
    return {
        "X": lambda t: g.gpic_linear(t, W), "W": lambda t: g.gpic_linear(X, t),
        "bias": lambda t: g.gpic_linear(X, W, t), "residual": lambda t: g.gpic_linear(X, W, residual=t),
        "dY": lambda t: g.gpic_linear_backward(t, X, W),
        "Z": lambda t: g.gpic_linear_backward(V, X, W, t, "gelu"),
        "H": lambda t: g.gpic_gated(X, W2, H=t), "dH": lambda t: g.gpic_gated_backward(t, X, W2, _t(5, 12)),
        "G": g.gpic_orthogonalize, "O": lambda t: g.gpic_orthogonalize(V, O=t),
        "step": lambda t: g.gpic_muon_step(t, W.clone(), _t(6, 8), 0.1),
    }


SHAPES = {"X": (5, 8), "W": (6, 8), "bias": (6,), "residual": (5, 6), "dY": (5, 6), "Z": (5, 6),
          "H": (5, 6), "dH": (5, 6), "G": (5, 6), "O": (5, 6), "step": (6, 8)}


@pytest.mark.parametrize("name", list(SHAPES))
def test_operands_that_require_gradients_are_refused(g, name):
    call, t = _calls(g)[name], _t(*SHAPES[name]).requires_grad_()
    with pytest.raises(ValueError, match="requires gradients"):
        call(t)
    assert bool((t == 1).all())
    call(t.detach())
    with torch.no_grad():
        call(t)
    with torch.inference_mode():
        call(_t(*SHAPES[name]))


def test_writes_in_place_are_counted(g):
    X, W, V = _t(5, 8), _t(6, 8), _t(12, 8)
    for n, f in (((5, 6), lambda t: g.gpic_linear(X, W, Y=t)),
                 ((5, 6), lambda t: g.gpic_gated(X, V, H=t)),
                 ((5, 6), lambda t: g.gpic_orthogonalize(_t(5, 6), O=t)),
                 ((6, 8), lambda t: g.gpic_muon_step(t, W.clone(), _t(6, 8), 0.1)),
                 ((6, 8), lambda t: g.gpic_muon_step(W.clone(), W.clone(), t, 0.1))):
        t = _t(*n)
        before = t._version
        f(t)
        assert t._version > before
        assert X._version == 0                  # what is read is not
    # a graph over weights that the step has replaced is refused
    w = torch.nn.Parameter(_t(6, 8))
    y = (w * w).sum()
    with torch.no_grad():
        g.gpic_muon_step(w, _t(6, 8), _t(6, 8), 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
