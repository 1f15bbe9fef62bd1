"""Orthogonalised updates at the ends of what the polynomial may do: the
iterates are held in half precision, so what the entry points accept must
stay finite and right there, and the rest must be refused."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_encoder import DEV, T, U, _gradient, _polar, _polar_tolerance, _rel  # noqa: E402


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    return g


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("shape", [(60, 90), (300, 200), (130, 520)], ids=str)
def test_growing_singular_values(g, shape, dtype):
    """A matrix of rank one has the singular value 1 at the start.  1.9 x takes
    it to 1.9^3 = 6.9 before the fourth step, where A's entries reach 47; 6 x -
    3 x^3 to 3, where b A is 27; x + 15 x^3 - 15 x^5 cancels to 1.  Halves are
    off by 2^-12, A by 2^-11; the steepest of the three, the last, takes that
    to 15 (2^-11) of the result, twice that with the other roundings."""
    m, n = shape
    u = torch.where(torch.arange(m, device=DEV) % 3 == 0, -1.0, 1.0)[:, None]
    v = torch.zeros((1, n), device=DEV)
    v[0, 5] = 1.0                                   # one column: A's entries are 1 / m ..
    one = torch.zeros((m, n), device=DEV)
    one[3, 5] = 1.0                                 # .. and one entry: A has a 1
    for G in ((u @ v).to(T[dtype]), one.to(T[dtype])):
        for steps, coef in ((4, (1.9, 0.0, 0.0)), (1, (1.0, 15.0, -15.0)), (2, (6.0, -3.0, 0.0))):
            print(f"polar {shape} {dtype} {steps} {coef}", flush=True)
            O = g.gpic_orthogonalize(G, steps, coef)
            assert bool(torch.isfinite(O).all())
            ref = _polar(G[None], steps, coef)
            assert _rel(O[None], ref) <= 2.0 ** -6 + U[dtype]
    with pytest.raises(g.GpicError, match="singular values"):
        g.gpic_orthogonalize(one.to(T[dtype]), 5, (1.9, 0.0, 0.0))


def test_a_refused_step_changes_nothing(g):
    W, G = _gradient((1, 130, 520), 1), _gradient((1, 130, 520), 2)
    M = torch.ones_like(W)
    w = W.clone()
    with pytest.raises(g.GpicError, match="singular values"):
        g.gpic_muon_step(W, G, M, 0.1, coefficients=(1.9, 0.0, 0.0))
    assert torch.equal(W, w) and bool((M == 1).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 60, 90), (2, 130, 520)], ids=str)
def test_magnitudes_at_the_ends_of_the_type(g, shape, dtype):
    """1 / |G|_F is no float32 below 2.9e-39 and above 3.4e38, and times 1,024
    from 3.0e-36 on; the matrices are.  With eps = 0 only the direction counts."""
    for s in (1e-39, 1e-37, 1e-35, 1e34, 1e37):
        G = (_gradient(shape, 7) * s).to(T[dtype])
        assert bool(torch.isfinite(G).all() & (G != 0).any())
        O = g.gpic_orthogonalize(G, eps=0.0)
        assert _rel(O, _polar(G, eps=0.0)) <= _polar_tolerance(dtype), s
    # the zero matrix of a stack stays what it was, 0 / 0
    G[1] = 0
    O = g.gpic_orthogonalize(G, eps=0.0)
    assert bool(O[1].isnan().all()) and bool(torch.isfinite(O[0]).all())
    assert not bool(g.gpic_orthogonalize(torch.zeros_like(G)).any())


# The rounding of the result to 8 bits: half a unit, uniform, of values of which
# all mantissas are as likely, 2^-7 / sqrt(12) / 1.35 = 1.7e-3 in the 2-norm.  Each
# of five steps rounds X, A and b A + c A^2 to 11 bits, 1.7e-3 / 8 of them each,
# against terms three times the result's size, and p'(1) = -0.7 takes half of
# the square of it on to the next: sqrt(3) 3 (2.1e-4) sqrt(2) = 1.6e-3, a quarter more
# for entries that are not independent.  Two bits less in the iterates would be
# 6e-3 and more.
@pytest.mark.parametrize("shape", [(1, 65, 300), (2, 100, 1000), (1, 300, 300), (1, 1500, 513),
                                   (1, 1024, 4096)], ids=str)
def test_bf16_iterates_keep_eleven_bits(g, shape):
    gen = torch.Generator(device=DEV).manual_seed(5)
    for G in (torch.randn(shape, device=DEV, generator=gen), _gradient(shape, 9)):
        G = G.to(torch.bfloat16)
        assert _rel(g.gpic_orthogonalize(G), _polar(G)) <= (1.7e-3 ** 2 + 2.0e-3 ** 2) ** 0.5
