"""Host-side checks at the edges of the calls around an encoder's layers (no GPU
needed)."""
import pytest

from test_training_host import _embed, _loss, _norm


@pytest.fixture(scope="module")
def g():
    import paper_1604_02700_amd as g
    g.lib()
    return g


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("sides", [dict(), dict(v=50000, k=4096, ldx=4096, ldw=4096),
                                   dict(v=1 << 20, k=1 << 20, ldx=1 << 20, ldw=1 << 20, aligned16=0)],
                         ids=str)
def test_an_empty_batch_needs_no_workspace(g, dtype, sides):
    L = g.lib()
    for back in (0, 1):
        assert L.gpic_cross_entropy_workspace_bytes(back, _loss(g, n=0, dtype=dtype, **sides)) == 0
    assert L.gpic_layer_norm_workspace_bytes(_norm(g, n=0, dtype=dtype)) == 0
    assert L.gpic_embedding_workspace_bytes(_embed(g, n=0, dtype=dtype)) == 0
