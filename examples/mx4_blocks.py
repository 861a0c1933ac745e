"""A stack of residual blocks trained on 4-bit weights: the whole step around the optimizer, and single tokens afterwards.  With a head
on top, the same stack is a policy over tokens, aligned by a clipped policy loss or by a preference loss with clipped gradients.

Each block is  h <- h + gate * norm(W_out silu(W_in norm(h))).  The weights live in the compressed layout that the optimizer
steps (BF16 with an 8-bit correction); the products run on their 4-bit copies, made anew from the corrected weights after
every step, and leave the BF16 gradients that the next step takes.

    python examples/mx4_blocks.py [--steps 100] [--align policy|preference]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_23349_amd as fo  # noqa: E402

BF16 = torch.bfloat16


def empty(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


class Param:
    """A parameter in the compressed layout, seen in its shape."""

    def __init__(self, value, weight_decay=0.0):
        self.shape = value.shape
        self.buffers = fo.ParamBuffers(value.numel(), "adamw")
        fo.split_weights(value.reshape(-1).contiguous(), self.buffers.param, self.buffers.rho)
        self.buffers.lr, self.buffers.weight_decay = 2e-3, weight_decay
        self.value, self.rho, self.grad = (t.view(self.shape) for t in (self.buffers.param, self.buffers.rho, self.buffers.grad))


class Linear:
    """A weight [n, k] with its 4-bit copies in both directions."""

    def __init__(self, n, k, g):
        self.n, self.k = n, k
        self.weight = Param(torch.randn(n, k, generator=g, device="cuda") * k ** -0.5, weight_decay=0.01)
        self.w, self.wt = fo.Mx4Tensor(n, k), fo.Mx4Tensor(k, n)
        self.xt = None                    # x transposed, for the backward pass; the same memory in every step
        self.refresh()

    def refresh(self):
        fo.mx4_quantize(self.weight.value, self.w, self.wt, rho=self.weight.rho)

    def forward(self, x, workspace, keep):
        y = empty(x.shape[0], self.n)
        if keep and (self.xt is None or self.xt.cols != x.shape[0]):
            self.xt = fo.Mx4Tensor(self.k, x.shape[0])
        fo.mx4_linear(x, self.w, y, xt=self.xt if keep else None, workspace=workspace)
        return y

    def backward(self, dy, workspace, rand):
        dx = empty(dy.shape[0], self.k)
        fo.mx4_linear_backward(dy, self.wt, self.xt, dx, self.weight.grad, rand=rand, workspace=workspace)
        return dx


class Model:
    def __init__(self, blocks=3, width=256, hidden=640, rows=512, seed=0, vocab=None, max_norm=None):
        g = torch.Generator("cuda").manual_seed(seed)
        self.generator, self.rows, self.width, self.hidden = g, rows, width, hidden
        self.up = [Linear(hidden, width, g) for _ in range(blocks)]
        self.down = [Linear(width, hidden, g) for _ in range(blocks)]
        one = torch.ones(width, device="cuda")
        self.pre = [Param(one) for _ in range(blocks + 1)]           # in front of each block, and of the output
        self.post = [Param(one) for _ in range(blocks)]
        self.gate = [Param(0.5 * one.view(1, -1)) for _ in range(blocks)]
        # boundary i lies between block i - 1 and block i: the norm behind the one, the gate, the residual, the norm in front of the other
        self.boundary = [fo.BlockNorm(width, post_norm=i > 0, post_weight=self.post[i - 1].value if i else None,
                                      pre_weight=self.pre[i].value) for i in range(blocks + 1)]
        self.head = Linear(vocab, width, g) if vocab else None
        self.linears = linears = self.up + self.down + ([self.head] if vocab else [])
        self.params = fo.TensorList([p.buffers for p in [l.weight for l in linears] + self.pre + self.post + self.gate])
        self.grads, self.max_norm, self.factor = fo.GradList.of(self.params), max_norm, fo.ClipFactor()
        sizes = [fo.mx4_linear_backward_workspace(rows, l.n, l.k) for l in linears] + \
                [fo.mx4_linear_workspace(rows, l.n, l.k) for l in linears] + \
                [fo.block_norm_backward_workspace(b, rows) for b in self.boundary] + [fo.grad_norm_workspace(self.grads)]
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
        self.step = 0

    def forward(self, x, keep=True):
        """The output, and with `keep` what the backward pass reads."""
        rows = x.shape[0]
        self.saved = []
        h, f = x, None
        for i, boundary in enumerate(self.boundary):
            y, stats = empty(rows, self.width), torch.empty(4, rows, device="cuda") if keep else None
            new = None if f is None else torch.empty_like(h)
            fo.block_norm(boundary, h, f=f, gate=self.gate[i - 1].value if i else None, h=new, y=y, stats=stats)
            h = h if f is None else new
            saved = [h, f, stats]
            if i < len(self.up):
                u = self.up[i].forward(y, self.workspace, keep)
                f = self.down[i].forward(torch.nn.functional.silu(u), self.workspace, keep)
                saved.append(u)
            if keep:
                self.saved.append(saved)
        return y

    def random(self, n):
        return torch.randint(0, 256, (self.rows, n), generator=self.generator, dtype=torch.uint8, device="cuda")

    def backward(self, dy):
        dh = df = None
        for i in reversed(range(len(self.boundary))):
            h, f, stats = self.saved[i][:3]
            if i < len(self.up):
                u = self.saved[i][3].float()
                s = torch.sigmoid(u)
                da = self.down[i].backward(df, self.workspace, self.random(self.width))
                dy = self.up[i].backward((da.float() * s * (1 + u * (1 - s))).to(BF16), self.workspace, self.random(self.hidden))
            grads = dict(dx=torch.empty_like(h), dpre_weight=self.pre[i].grad)
            if i:
                grads.update(df=torch.empty_like(f), dgate=self.gate[i - 1].grad, dpost_weight=self.post[i - 1].grad)
            fo.block_norm_backward(self.boundary[i], h, stats, f=f, gate=self.gate[i - 1].value if i else None, dy=dy, dh=dh,
                                   workspace=self.workspace, **grads)
            dh, df = grads["dx"], grads.get("df")

    def logits(self, x, keep=True):
        return self.head.forward(self.forward(x, keep), self.workspace, keep)

    def backward_from_logits(self, dlogits):
        self.backward(self.head.backward(dlogits, self.workspace, self.random(self.head.n)))

    def update(self):
        self.step += 1
        if self.max_norm is not None:
            fo.grad_norm(self.grads, self.max_norm, self.factor, workspace=self.workspace)
            fo.clip_gradients(self.grads, self.factor)
        fo.adamw_step_exact(self.params, 0.9, 0.99, 1e-8, self.step)
        for linear in self.linears:
            linear.refresh()


def train(steps=100, verbose=True):
    """Fits the model to a fixed random function; returns the model, its inputs and the losses."""
    model = Model()
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(model.rows, model.width, generator=g, device="cuda").to(BF16)
    teacher = torch.randn(model.width, model.width, generator=g, device="cuda") * model.width ** -0.5
    target = torch.sin(2 * x.float() @ teacher)
    losses = []
    for step in range(steps):
        off = model.forward(x).float() - target
        losses.append(float(off.square().mean()))
        if verbose and step % 20 == 0:
            print(f"step {step:4d}  loss {losses[-1]:.4f}", flush=True)
        model.backward((2 * off / off.numel() * 64).to(BF16))        # (scaled: AdamW does not see it)
        model.update()
    return model, x, losses


class Aligned:
    """A policy over `vocab` tokens whose answer to a context is right if it is of the context's kind, one of four."""

    def __init__(self, vocab=64, rows=512):
        self.model = Model(blocks=2, rows=rows, vocab=vocab, max_norm=1.0)
        self.g = torch.Generator("cuda").manual_seed(2)
        self.x = torch.randn(rows, self.model.width, generator=self.g, device="cuda").to(BF16)
        self.kind = torch.randint(0, 4, (rows,), generator=self.g, device="cuda")
        self.start = self.model.logits(self.x, keep=False)           # of the reference policy: the model as it began
        self.workspace = torch.empty(max(fo.token_logprob_workspace(self.start), fo.policy_loss_workspace(self.start)), dtype=torch.uint8,
                                     device="cuda")
        self.rows, self.vocab = rows, vocab

    def of_rows(self, dtype=torch.float32):
        return torch.empty(self.rows, dtype=dtype, device="cuda")

    def logprob(self, logits, tokens, **also):
        out = self.of_rows()
        fo.token_logprob(logits, tokens, logprob=out, workspace=self.workspace, **also)
        return out

    def right(self, tokens):
        return (tokens % 4 == self.kind).float()

    def policy_step(self, epochs=2):
        """One answer to each context, and `epochs` updates on them.  Returns the share of right answers."""
        spec = fo.PolicyLoss(clip_low=0.2, clip_high=0.28, kl_weight=0.02)
        logits = self.model.logits(self.x, keep=False)
        tokens = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=self.g)[:, 0]
        old, ref, reward = self.logprob(logits, tokens), self.logprob(self.start, tokens), self.right(tokens)
        advantages = (reward - reward.mean()) / (reward.std() + 1e-6)
        weights, self.stats = torch.full_like(reward, 1 / self.rows), empty(4, dtype=torch.float32)
        for _ in range(epochs):
            logits = self.model.logits(self.x)
            fo.policy_loss(spec, logits, tokens, advantages, self.stats, old_logprob=old, ref_logprob=ref, weights=weights, dlogits=logits,
                           workspace=self.workspace)                 # (the gradient takes the logits' place)
            self.model.backward_from_logits(logits)
            self.model.update()
        return float(reward.mean())

    def preference_step(self, length=8):
        """One update on pairs of sequences of `length` answers, the chosen ones right, the rejected ones wrong.  Returns the loss."""
        spec = fo.PreferenceLoss(beta=0.1)
        offsets = torch.arange(0, self.rows + 1, length, device="cuda")
        chosen = torch.arange(self.rows, device="cuda") // length % 2 == 0
        wrong = torch.randint(1, 4, (self.rows,), generator=self.g, device="cuda")
        block = torch.randint(0, self.vocab // 4, (self.rows,), generator=self.g, device="cuda")
        tokens = 4 * block + (self.kind + torch.where(chosen, 0, wrong)) % 4
        ref, logits = self.logprob(self.start, tokens), self.model.logits(self.x)
        wide, lse, slope, loss = self.of_rows(torch.float64), self.of_rows(), self.of_rows(), empty(1, dtype=torch.float32)
        self.logprob(logits, tokens, logprob64=wide, lse=lse)
        fo.preference_loss(spec, wide, offsets, loss, ref_logprob=ref, dlogprob=slope)
        fo.token_logprob_backward(logits, tokens, lse, slope, logits)
        self.model.backward_from_logits(logits)
        self.model.update()
        return float(loss)


def align(how, steps=100, verbose=True):
    aligned = Aligned()
    course = []
    for step in range(steps):
        course.append(aligned.policy_step() if how == "policy" else aligned.preference_step())
        if verbose and step % 20 == 0:
            print(f"step {step:4d}  {'right answers' if how == 'policy' else 'loss'} {course[-1]:.4f}  gradients' norm "
                  f"{float(aligned.model.factor.norm):.3g}", flush=True)
    return aligned, course


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--align", choices=("policy", "preference"))
    args = ap.parse_args()
    if args.align:
        _, course = align(args.align, args.steps)
        print(f"{'right answers' if args.align == 'policy' else 'loss'} {course[0]:.4f} -> {course[-1]:.4f}")
        return
    model, x, losses = train(args.steps)
    batch = model.forward(x, keep=False)
    token = model.forward(x[7:8].contiguous(), keep=False)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f};  one token alone against the batch: off by {float((token - batch[7:8]).abs().max()):.3g}")


if __name__ == "__main__":
    main()
