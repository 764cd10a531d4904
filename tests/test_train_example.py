"""The example's factor of the gradients, on the CPU: a norm that is not finite gives one that is not, so that the step is
skipped (an infinite norm would otherwise give 0, which is finite)."""

import math
import os
import sys

import pytest

from conftest import ROOT

pytest.importorskip("paper_2606_23087_amd.training", reason="libflowpool.so not built (run __graft_entry__.build())")
torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 1e30])
def test_clip_factor_of_gradients_that_are_not_finite(bad):
    from train_head import clip_factor
    grads = [torch.ones(3, 5), torch.zeros(7)]
    grads[1][2] = bad                                   # the square of 1e30 is infinite
    assert not math.isfinite(float(clip_factor(grads, 1.0)))


@pytest.mark.parametrize("size,want", [(0.0, 1.0), (1e-3, 1.0), (0.25, 1.0), (0.5, 0.5), (1.0, 0.25)])
def test_clip_factor(size, want):
    from train_head import clip_factor
    factor = clip_factor([torch.full((4, 2), size), torch.full((8,), size)], 1.0)     # of norm 4 size
    assert factor.shape == (1,) and abs(float(factor) - want) <= 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 1e30])
def test_step_is_skipped(bad):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from train_head import Trainer
    t = Trainer()
    try:
        t.step()
        m = t.model
        held = [*m.params.values(), *m.bf16.values(), *m.states]
        before = [x.clone() for x in held]
        m.grads["adapter"][3, 5] = bad
        t.update(3e-3, 1.0)
        assert all(torch.equal(a, b) for a, b in zip(held, before))
        m.grads["adapter"][3, 5] = 0.0
        t.update(3e-3, 1.0)
        assert all(bool(torch.isfinite(x).all()) for x in held) and not torch.equal(held[0], before[0])
    finally:
        t.close()
