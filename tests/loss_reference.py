"""The losses on the logits from their definitions, in 64 bits on the CPU, and how far the kernels' FP32 arithmetic may be off.

Tolerances, with u = 2^-24.  A row's sum of exponentials: the argument (x - m) c is off by 3 u of itself (the difference, the rounding of
c, the product), the power of two by 2 u, and a lane adds up at most `adds` of them with an error of u each, rescales its sum at most
once per eight values, 4 u each time for the power and the product, and joins the others in FP64.  So log(sum) is off by
u (3 sum p |x - m| / T + 2 + 1.5 adds), and what is rounded to FP32 by u of itself in addition."""
import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def adds(vocab):
    """The most values that one lane adds up: a row is shared by 256 lanes or more, which take eight at a time."""
    return 8 * -(-vocab // 2048) + 1


class Rows:
    """log-probabilities of the rows of `logits` [rows, vocab] and their error bounds."""

    def __init__(self, logits, tokens, temperature=1.0):
        self.t = float(torch.tensor(temperature, dtype=torch.float32))
        self.x, self.tokens, self.dtype = logits.double().cpu(), tokens.cpu(), logits.dtype
        self.vocab = self.x.shape[1]
        self.counted = self.tokens >= 0
        self.out = self.tokens >= self.vocab
        self.most = self.x.max(1, keepdim=True).values
        e = torch.exp((self.x - self.most) / self.t)
        self.sum = e.sum(1)
        log_sum = torch.log(self.sum)
        self.log_sum = log_sum
        self.p = e / self.sum[:, None]
        self.lse = self.most[:, 0] / self.t + log_sum
        at = self.tokens.clamp(0, self.vocab - 1)[:, None]
        self.hit = torch.zeros_like(self.x).scatter_(1, at, 1.0)
        self.logprob = (self.x.gather(1, at) - self.most)[:, 0] / self.t - log_sum
        self.logprob[self.out] = float("nan")
        far = torch.nan_to_num(((self.most - self.x) / self.t).clamp(max=1e6) * self.p)
        self.err = U * (3 * far.sum(1) + 2 + 1.5 * adds(self.vocab))
        for v in (self.lse, self.logprob):
            v[~self.counted] = 0

    def gradient(self, d, d_err, from_lse):
        """(gradient of the logits, its error bound) for the slopes d [rows], themselves off by d_err.  from_lse: the probabilities come
        from lse in FP32, else from the largest value and the log of the sum."""
        d, d_err = (torch.where(self.counted, v, torch.zeros_like(v))[:, None] for v in (d, d_err))
        g = d / self.t * (self.hit - self.p)
        g[(d == 0)[:, 0]] = 0
        g[self.out & (d != 0)[:, 0]] = float("nan")
        # the exponent: c off by u of itself, a difference and a multiply-add, and a shift rounded three times
        shift = self.lse.abs() if from_lse else self.log_sum.abs()
        base = self.x.abs() if from_lse else (self.x - self.most).abs()
        e = U * (3 * (base / self.t).clamp(max=200) + 3 * shift[:, None] + 4) + self.err[:, None]
        err = (d.abs() / self.t) * (self.p * e + 3 * U * (self.hit + self.p)) + d_err / self.t * (self.hit - self.p).abs()
        return g, err + HALF[self.dtype] * (g.abs() + err) + 1e-45


def close(got, want, err, what=""):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = (got == want) | torch.isnan(want)
    off = torch.where(same, 0.0, (got - want).abs())
    assert bool((off <= torch.nan_to_num(err, nan=0.0)).all()), (what, float((off - err).nan_to_num(nan=-1).max()))


class Policy:
    """The policy loss: slopes, terms and statistics."""

    def __init__(self, rows, advantages, old=None, ref=None, weights=None, low=0.2, high=0.2, kl_weight=0.0, grad_scale=1.0):
        f = lambda v: None if v is None else v.double().cpu()        # noqa: E731
        low, high, kl_weight = (float(torch.tensor(v, dtype=torch.float32)) for v in (low, high, kl_weight))
        a, old, ref = f(advantages), f(old), f(ref)
        w = torch.ones_like(a) if weights is None else f(weights)
        rows.counted = rows.counted & (w != 0)
        z = torch.zeros_like(a)
        lp = rows.logprob
        self.ratio = r = torch.exp(lp - (lp if old is None else old))
        self.blocked = ((a > 0) & (r > 1 + high)) | ((a < 0) & (r < 1 - low))
        surrogate = -torch.minimum(r * a, torch.clamp(r, 1 - low, 1 + high) * a)
        d = -a * r * ~self.blocked
        size = (a * r).abs()
        kl, kl_slope = z, z
        if ref is not None:
            gap = ref - lp
            kl = torch.expm1(gap) - gap
            kl_slope = kl_weight * torch.exp(gap)
            d = d - kl_weight * torch.expm1(gap)
        pick = lambda v: torch.where(rows.counted, v, z)        # noqa: E731
        self.slope = pick(w * d) * grad_scale
        err = rows.err + 1e-15
        self.slope_err = pick(w.abs() * ((size + kl_slope) * err * 1.01 + 3 * U * d.abs())) * abs(grad_scale)
        parts = [pick(w * surrogate), pick(w * kl), pick(w * self.blocked)]
        errs = [pick(w.abs() * size * err * 1.01), pick(w.abs() * (torch.exp(gap) - 1).abs() * err * 1.01 + w.abs() * err ** 2) if ref is not None else z, z]
        s, e = [p.sum() for p in parts], [v.sum() for v in errs]
        self.stats = torch.stack([s[0] + kl_weight * s[1]] + s)
        self.stats_err = torch.stack([e[0] + kl_weight * e[1]] + e)
        self.stats_err = self.stats_err + U * self.stats.abs() + 1e-15 * sum(p.abs().sum() for p in parts)
        self.logprob = pick(lp)
        self.logprob_err = pick(rows.err) + U * self.logprob.abs()


def preference(logprob, offsets, ref=None, weights=None, kind="sigmoid", beta=0.1, smoothing=0.0, halves=False, grad_scale=1.0):
    """(loss, margins, gradient of logprob, sum of magnitudes behind each margin) in 64 bits."""
    beta, smoothing = (float(torch.tensor(v, dtype=torch.float32)) for v in (beta, smoothing))
    lp = logprob.double().cpu()
    n = lp.numel()
    w = torch.ones(n, dtype=torch.float64) if weights is None else weights.double().cpu()
    gap = lp - (0 if ref is None else ref.double().cpu())
    part = torch.where(w == 0, torch.zeros_like(lp), w * gap)
    cut = [min(max(int(v), 0), n) for v in offsets]
    pairs = (len(cut) - 1) // 2
    loss, margins, grad = 0.0, torch.zeros(pairs, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for p in range(pairs):
        of = (p, pairs + p) if halves else (2 * p, 2 * p + 1)
        gain = [part[cut[q]:cut[q + 1]].sum() for q in of]
        z = (beta * (gain[0] - gain[1])).requires_grad_()
        if kind == "sigmoid":
            soft = torch.nn.functional.softplus
            one = (1 - smoothing) * soft(-z) + (smoothing * soft(z) if smoothing else 0.0)
        elif kind == "hinge":
            one = torch.clamp(1 - z, min=0)
        else:
            one = (z / beta - 0.5 / beta) ** 2
        dz = torch.autograd.grad(one, z)[0]
        loss += float(one.detach()) / pairs
        margins[p] = z.detach()
        for q, sign in zip(of, (1, -1)):
            a, b = cut[q], cut[q + 1]
            grad[a:b] = torch.where(w[a:b] == 0, 0.0, sign * dz * beta * grad_scale / pairs * w[a:b])
    return loss, margins, grad
