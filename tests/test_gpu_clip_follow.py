"""Gradients that get new memory from step to step: the list of a model's gradients reads and clips those that the step takes."""
import gc

import pytest
import torch

from test_gpu_clip_steps import buffers, same, step
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

SIZES = [4097, 1, 70_001, 32]


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()


@pytest.mark.parametrize("in_step", [False, True])
def test_new_gradients_every_step(in_step):
    a, b = buffers(SIZES, "adamw_exact"), buffers(SIZES, "adamw_exact")
    ta, tb = fo.TensorList(a), fo.TensorList(b)
    followed, factor, twin = fo.GradList.of(ta), fo.ClipFactor(), fo.ClipFactor()
    first = [x.grad.clone() for x in a]
    ws = torch.empty(fo.grad_norm_workspace(followed), dtype=torch.uint8, device="cuda")
    for t in (1, 2, 3):
        new = [torch.randn(n, device="cuda").mul_(10.0 ** t).to(torch.bfloat16) for n in SIZES]
        for i, g in enumerate(new):
            ta.set_grad(i, g)
            b[i].grad.copy_(g)
        fo.grad_norm(followed, 0.5, factor, workspace=ws)
        fo.grad_norm(fo.GradList([x.grad for x in b]), 0.5, twin, workspace=ws)
        assert torch.equal(factor.data.view(torch.int64), twin.data.view(torch.int64)) and float(factor.scale) < 1
        if in_step:
            step("adamw_exact", ta, t, clip=factor)
            step("adamw_exact", tb, t, clip=twin)
        else:
            fo.clip_gradients(followed, factor)
            fo.clip_gradients(fo.GradList([x.grad for x in b]), twin)
            assert all(torch.equal(g, x.grad) for g, x in zip(new, b))
            step("adamw_exact", ta, t)
            step("adamw_exact", tb, t)
        same(a, b)
    assert all(torch.equal(x.grad, g) for x, g in zip(a, first))       # what the list began with has not been written
