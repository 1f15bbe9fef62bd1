"""The example that learns an embedding and clusters it, at a small size:
the loss falls, single points embed as the batch does, and the clustering
of the embedded points is the oracle's."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_learned_embedding(orc, dtype):
    from gpu_helpers import check_labels, rel_l1
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import learned_embedding
    finally:
        sys.path.pop(0)
    n = 2000
    print(f"learned embedding n={n} {dtype}", flush=True)
    r = learned_embedding.run(n, 40, getattr(torch, dtype))
    assert all(np.isfinite(r["losses"])) and r["losses"][-1] < 0.3 * r["losses"][0]
    E = r["embedding"]
    assert E.shape == (n, 16) and bool(torch.isfinite(E).all())
    # rows of one point and of the batch differ by their sums' order and, in
    # 16 bits, by a rounding of each of four layers
    size = float(E.square().mean().sqrt())
    tol = 1e-4 if dtype == "float32" else 4 * 4 * 2.0 ** -8
    assert float((r["one"] - E[:8]).abs().max()) <= tol * size
    X = E.cpu().numpy()
    ref = orc.pic_dense(X, r["sigma"], r["k"], "converge", 1000, 1e-5 / n)
    out = r["clusters"]
    assert out.pi.converged and abs(out.pi.iterations - ref.pi.iterations) <= 1
    if out.pi.iterations == ref.pi.iterations:
        v = out.pi.v.cpu().numpy()
        assert rel_l1(v, ref.pi.v) <= 1e-4
        check_labels(orc, f"learned embedding {dtype}", ref.pi.v, ref.km.labels, v, out.km, r["k"])
