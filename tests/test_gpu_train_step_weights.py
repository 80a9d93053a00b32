"""The router weights' gradients of a training step, slot by slot as the routing has
them: every used slot has its gradient, an unused one has none."""
import pytest
import torch

from test_gpu_train_step import SMOOTH, THROUGH_RELU, exact, make, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [1, 4])
def test_gradients_of_router_weights(seed):
    m = make(seed)
    got, ref = step(m), exact(m)
    used = m["ids"] >= 0
    assert bool(used.any()) and not bool(used.all())
    for name, tol in (("alpha0", THROUGH_RELU), ("alpha1", SMOOTH)):
        g, r = got[name], ref[name]
        assert not g[~used].any() and not r[~used].any()
        # a token without a target has none; no other slot is lost
        assert int((r != 0).sum()) > used.sum() // 3 and torch.equal(g != 0, r != 0), name
        assert float((g.double() - r).norm() / r.norm()) <= tol, name
