"""A stack of residual blocks trained on 4-bit weights: the whole step around the optimizer, and single tokens afterwards.

Each block is  h <- h + gate * norm(W_out silu(W_in norm(h))).  The weights live in the compressed layout that the optimizer
steps (BF16 with an 8-bit correction); the products run on their 4-bit copies, made anew from the corrected weights after
every step, and leave the BF16 gradients that the next step takes.

    python examples/mx4_blocks.py [--steps 100]
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
    def __init__(self, blocks=3, width=256, hidden=640, rows=512, seed=0):
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
        linears = self.up + self.down
        self.params = fo.TensorList([p.buffers for p in [l.weight for l in linears] + self.pre + self.post + self.gate])
        sizes = [fo.mx4_linear_backward_workspace(rows, l.n, l.k) for l in linears] + \
                [fo.mx4_linear_workspace(rows, l.n, l.k) for l in linears] + \
                [fo.block_norm_backward_workspace(b, rows) for b in self.boundary]
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

    def update(self):
        self.step += 1
        fo.adamw_step_exact(self.params, 0.9, 0.99, 1e-8, self.step)
        for linear in self.up + self.down:
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


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    model, x, losses = train(ap.parse_args().steps)
    batch = model.forward(x, keep=False)
    token = model.forward(x[7:8].contiguous(), keep=False)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f};  one token alone against the batch: off by {float((token - batch[7:8]).abs().max()):.3g}")


if __name__ == "__main__":
    main()
