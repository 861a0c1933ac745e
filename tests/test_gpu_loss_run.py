"""From logits to the step and back: the losses, the norm and clipping of gradients and the steps as a training program strings them together.

The parameters are the logits themselves, a table [rows, vocab] in the compressed layout, so that the loss's gradient is the parameter's and the whole
loop is made of these calls.  Losses and gradients are held to their formulas in 64 bits with the bounds of loss_reference.py, the clipped gradients to
the two roundings of their product, the step to the same step of gradients clipped by torch."""
import gc
import os
import sys

import pytest
import torch

import loss_reference as ref
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

BF16, FP32, FP64 = torch.bfloat16, torch.float32, torch.float64
SHAPES = [(24, 1000), (6, 40_003), (300, 333)]


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()


def gpu(*shape, dtype=FP32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


class Table:
    """A table of logits as a parameter, its gradient, and what the calls on it need."""

    def __init__(self, rows, vocab, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.rows, self.vocab = rows, vocab
        self.params, self.logits, self.grad = [], [], []
        # beside the table a parameter of odd size, whose gradient is not a loss's
        for n in (rows * vocab, 1003):
            b = fo.ParamBuffers(n, "adamw")
            fo.split_weights(torch.randn(n, generator=g, device="cuda"), b.param, b.rho)
            b.lr, b.weight_decay = 1e-2, 0.01
            self.params.append(b)
        self.other = torch.randn(1003, generator=g, device="cuda").to(BF16)
        self.logits, self.grad = self.params[0].param.view(rows, vocab), self.params[0].grad.view(rows, vocab)
        self.list = fo.TensorList(self.params)
        self.grads, self.factor = fo.GradList.of(self.list), fo.ClipFactor()
        self.tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        self.tokens[rows // 2] = -1
        self.advantages, self.old, self.ref = (torch.randn(rows, generator=g, device="cuda") for _ in range(3))
        self.weights = torch.rand(rows, generator=g, device="cuda") / rows
        self.old.copy_(-7 + 0.1 * self.old)
        self.ref.copy_(-7 + 0.1 * self.ref)
        n = self.rows - self.rows % 4
        self.offsets = torch.tensor([0, n // 4, n // 2 + 1, n // 2 + 1 + n // 8, n], device="cuda")
        size = max(fo.policy_loss_workspace(self.logits), fo.token_logprob_workspace(self.logits), fo.grad_norm_workspace(self.grads))
        self.workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.stats, self.loss, self.logprob, self.lse, self.slope = gpu(4), gpu(1), gpu(rows), gpu(rows), gpu(rows)
        self.wide = gpu(rows, dtype=FP64)
        torch.cuda.synchronize()

    def loss_of(self, how):
        self.params[1].grad.copy_(self.other)
        if how == "policy":
            fo.policy_loss(fo.PolicyLoss(kl_weight=0.1), self.logits, self.tokens, self.advantages, self.stats, old_logprob=self.old,
                           ref_logprob=self.ref, weights=self.weights, logprob=self.logprob, dlogits=self.grad, workspace=self.workspace)
            return
        fo.token_logprob(self.logits, self.tokens, logprob=self.logprob, logprob64=self.wide, lse=self.lse, workspace=self.workspace)
        fo.preference_loss(fo.PreferenceLoss(beta=0.2), self.wide, self.offsets, self.loss, ref_logprob=self.ref, dlogprob=self.slope)
        fo.token_logprob_backward(self.logits, self.tokens, self.lse, self.slope, self.grad)

    def clip(self):
        fo.grad_norm(self.grads, 0.05, self.factor, workspace=self.workspace)
        fo.clip_gradients(self.grads, self.factor)

    def update(self, step):
        fo.adamw_step_exact(self.list, 0.9, 0.99, 1e-8, step)

    def everything(self):
        return [t for b in self.params for t in (b.param, b.rho, b.grad, b.m_q, b.v_q, b.m_scale, b.v_scale)] + \
               [self.stats, self.loss, self.factor.data.view(torch.int64)]


@pytest.mark.parametrize("how", ["policy", "preference"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logits_to_step(rows, vocab, how):
    table, twin = Table(rows, vocab), Table(rows, vocab)
    for step in (1, 2, 3):
        table.loss_of(how)
        at = ref.Rows(table.logits, table.tokens)
        if how == "policy":
            want = ref.Policy(at, table.advantages, old=table.old, ref=table.ref, weights=table.weights, kl_weight=0.1)
            ref.close(table.stats, want.stats, want.stats_err, "stats")
            g, err = at.gradient(want.slope, want.slope_err, from_lse=False)
        else:
            # with the log-probabilities and the slopes that the calls themselves handed on: each has a test of its own
            loss, _, slope = ref.preference(table.wide, table.offsets, ref=table.ref, beta=0.2)
            assert abs(float(table.loss) - loss) <= ref.U * abs(loss) + 1e-12
            ref.close(table.wide, torch.where(at.counted, at.logprob, 0.0), at.err, "logprob")
            ref.close(table.slope, slope, ref.U * slope.abs() + 1e-12, "slope")
            g, err = at.gradient(slope, ref.U * slope.abs() + 1e-12, from_lse=True)
        ref.close(table.grad, g, err, "gradient")
        whole = [b.grad.clone() for b in table.params]
        table.clip()
        norm = torch.cat([t.double() for t in whole]).norm()
        assert abs(float(table.factor.norm) - float(norm)) <= 2.0 ** -23 * float(norm)
        clipped = [(t.float() * table.factor.scale).to(BF16) for t in whole]
        assert float(norm) > 0.05 and all(torch.equal(b.grad, t) for b, t in zip(table.params, clipped))
        table.update(step)
        for b, t in zip(twin.params, clipped):
            b.grad.copy_(t)
        twin.update(step)
        for a, b in zip(table.params, twin.params):
            for name in ("param", "rho", "m_q", "v_q", "m_scale", "v_scale"):
                assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("how", ["policy", "preference"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_a_captured_loop_goes_where_the_eager_one_goes(rows, vocab, how):
    captured, eager = Table(rows, vocab), Table(rows, vocab)
    for t in (captured, eager):                        # (one step outside the graph, so that the library has its tables)
        t.loss_of(how)
        t.clip()
        t.update(5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.loss_of(how)
        captured.clip()
        captured.update(5)
    for replay in range(4):
        graph.replay()
        eager.loss_of(how)
        eager.clip()
        eager.update(5)
        torch.cuda.synchronize()
        for a, b in zip(captured.everything(), eager.everything()):
            assert torch.equal(a, b), replay
        captured.workspace.fill_(0xFF)
        captured.grad.fill_(float("nan"))


def test_gradients_accumulated_in_fp32():
    table, g = Table(24, 1000), torch.Generator("cuda").manual_seed(5)
    sums = [torch.zeros(b.numel, device="cuda") for b in table.params]
    grads = fo.GradList(sums, [b.grad for b in table.params])
    workspace = torch.empty(fo.grad_norm_workspace(grads), dtype=torch.uint8, device="cuda")
    for micro in range(3):
        table.advantages.copy_(torch.randn(24, generator=g, device="cuda"))
        table.loss_of("policy")
        for s, b in zip(sums, table.params):
            s += b.grad
    fo.grad_norm(grads, 0.05, table.factor, workspace=workspace)
    fo.clip_gradients(grads, table.factor)
    norm = float(torch.cat([s.double() for s in sums]).norm())
    assert abs(float(table.factor.norm) - norm) <= 2.0 ** -23 * norm
    for s, b in zip(sums, table.params):
        assert torch.equal(b.grad, (s * table.factor.scale).to(BF16))


@pytest.mark.parametrize("how", ["policy", "preference"])
def test_the_example_aligns_a_policy(how):
    import mx4_blocks
    aligned, course = mx4_blocks.align(how, steps=3, verbose=False)
    model = aligned.model
    assert len(course) == 3 and all(0 <= v < 10 for v in course)
    norm, scale = float(model.factor.norm), float(model.factor.scale)
    assert 0 < norm < float("inf") and scale == (1.0 if norm <= 1 else pytest.approx(1 / norm, rel=1e-6))
    after = float(torch.cat([b.grad.double() for b in model.params.buffers]).norm())
    assert after <= 1 + 2.0 ** -8                      # (each gradient is rounded to BF16 once more)
    again, _ = mx4_blocks.align(how, steps=3, verbose=False)
    for a, b in zip(model.params.buffers, again.model.params.buffers):
        assert torch.equal(a.param, b.param) and torch.equal(a.rho, b.rho) and torch.equal(a.m_q, b.m_q) and torch.equal(a.v_q, b.v_q)


def test_the_examples_gradient_of_the_logits():
    import mx4_blocks
    aligned = mx4_blocks.Aligned()
    logits = aligned.model.logits(aligned.x)
    tokens = torch.arange(aligned.rows, device="cuda") % aligned.vocab
    old, adv = aligned.logprob(logits, tokens), aligned.right(tokens) - 0.5
    before, stats = logits.clone(), gpu(4)
    fo.policy_loss(fo.PolicyLoss(), logits, tokens, adv, stats, old_logprob=old, dlogits=logits, workspace=aligned.workspace)
    at = ref.Rows(before, tokens)
    want = ref.Policy(at, adv, old=old)
    ref.close(logits, *at.gradient(want.slope, want.slope_err, from_lse=False), "gradient")
    aligned.model.backward_from_logits(logits)
    assert all(bool(torch.isfinite(b.grad).all()) for b in aligned.model.params.buffers)
    assert float(aligned.model.head.weight.grad.float().norm()) > 0
