"""Steps that take a clipping factor of any scale, where test_gpu_clip_steps.py has powers of two or none: the default AdamW step, and what the step saves over gradients clipped in place."""
import gc

import pytest
import torch

from test_gpu_clip_steps import buffers, expected, factor_of, same, step
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()


def weights(b):
    out = torch.empty(b.numel, device="cuda")
    fo.reconstruct_weights(b.param, b.rho, out)
    return out


@pytest.mark.parametrize("sizes", [[4097], [33, 70_001, 32], [3_000_001]])
def test_the_default_adamw_step_at_any_scale(sizes):
    # its division is faithful, not exactly rounded: weights differ in their last code on at most 1e-5 of the elements, as without a factor; the states are the same bits
    bufs = buffers(sizes, "adamw")
    tensors = fo.TensorList(bufs)
    for t, scale in ((1, 0.3137), (2, 1e-3), (200, 0.99999)):
        f = factor_of(scale)
        want = [expected("adamw_exact", b, f.scale.cpu(), t) for b in bufs]
        before = [weights(b) for b in bufs]
        step("adamw", tensors, t, clip=f)
        differ = 0
        for b, w, old in zip(bufs, want, before):
            for name in ("m_q", "v_q", "m_scale", "v_scale"):
                assert torch.equal(getattr(b, name).view(torch.uint8), getattr(w, name).view(torch.uint8)), name
            got, exact = weights(b), weights(w)
            differ += int((got != exact).sum())
            # a code is 2^-8 / 127 of the weight or less, and the weight may be on the other side of one's border; the update itself is off by some
            # units of 2^-23 of its own
            assert bool(((got - exact).abs() <= 2.0 ** -14 * exact.abs() + 2.0 ** -20 * (old - exact).abs()).all())
            b.grad.mul_(1.5)
        assert differ <= 1 + 1e-5 * sum(sizes)


def test_a_step_with_the_factor_rounds_once_less_than_clipping():
    # beside the step with the factor one on gradients that were clipped in place: each the algorithm on its own gradients
    for kind in ("sgd", "lion", "adamw_exact"):
        a, b = buffers([4099], kind), buffers([4099], kind)
        f, one = factor_of(0.3), factor_of(1.0)
        clipped = fo.TensorList(b)
        fo.clip_gradients(fo.GradList.of(clipped), f)
        exact = a[0].grad.float() * f.scale
        assert torch.equal(b[0].grad, exact.to(torch.bfloat16)) and not torch.equal(b[0].grad.float(), exact)
        want = [[expected(kind, x[0], g.scale.cpu(), 1)] for x, g in ((a, f), (b, one))]
        step(kind, fo.TensorList(a), clip=f)
        step(kind, clipped)
        same(a, want[0])
        same(b, want[1])
        assert kind == "lion" or not torch.equal(a[0].m_q, b[0].m_q) or not torch.equal(a[0].m_scale, b[0].m_scale)
