"""The example that runs the 4-bit products, the block norms and the optimizer step together."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_example_learns_and_serves_single_tokens():
    import mx4_blocks
    model, x, losses = mx4_blocks.train(steps=100, verbose=False)
    # the target's mean square is about 1/2, and a model that learns nothing cannot go below it; twice the first loss means divergence
    assert losses[-1] < 0.5 * losses[0] and all(loss < 2 * losses[0] for loss in losses)
    batch = model.forward(x, keep=False)
    for row in (0, 7, 511):
        token = model.forward(x[row:row + 1].contiguous(), keep=False)
        # the same function: sums in another order, whose last bits can move a value to the neighbouring one of four bits
        assert float((token - batch[row:row + 1]).float().abs().max()) < 0.25


def test_the_example_is_the_same_every_time():
    import mx4_blocks
    one, two = (mx4_blocks.train(steps=5, verbose=False)[0] for _ in range(2))
    for a, b in zip(one.params.buffers, two.params.buffers):
        assert torch.equal(a.param, b.param) and torch.equal(a.rho, b.rho) and torch.equal(a.m_q, b.m_q) and torch.equal(a.v_q, b.v_q)
