"""The operators at both ends of a backward pass, as a training program calls them, each beside its plain form: the losses on
the logits with their gradients, and the global norm of the gradients with their clipping ahead of the optimizer step.

With `own` false, `run` computes an operator in elementary torch operations in 32 bits (64 for long sums and for what is
computed once per row), rounded once at the end; with `own` true it calls this package.  `exact` gives the same outputs
from the definitions in 64 bits.

A case is a dict of plain values:
  op   norm        the norm of all gradients of a list and the factor that brings it down to a limit, which a step takes
       clip        the same, and the gradients times that factor
       logprob     the log-probability of one token per row of logits, and the log of the row's sum of exponentials
       policy      the clipped policy loss with its KL term on rows of logits, and the gradient of the logits
       preference  the preference loss of pairs of sequences of rows, and the gradient of the logits
  list   gpt2 (the tensors of a GPT-2 124M), llama (embedding, head and `layers` layers of Llama-3.1-8B), flat (one tensor
         of `numel`) or mixed (`tensors` tensors of uneven, mostly odd sizes drawn from `shape`, `numel` in all)
  grads  type of the gradients;  what is clipped becomes BF16
  rows, vocab, dtype   the logits;  masked: how many rows do not count (prompt tokens, padding)
  kl     weight of the KL term, 0: no reference policy;  on_policy: the ratio is that of the policy to itself
  pairs  the rows are 2 `pairs` sequences of uneven lengths, a chosen and a rejected one by turns;  kind, smoothing: the loss
"""
import math
import random

import torch

own = False

BF16, FP32, FP64 = torch.bfloat16, torch.float32, torch.float64
TYPES = {"bf16": BF16, "fp32": FP32}
MAX_NORM = 1.0
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
BETA = 0.1
LARGEST = 4096 * 128256


def listed():
    return [
        # one flat buffer of 2^20 gradients, the smallest of the benchmark's lists
        dict(name="norm_flat_1m", op="norm", list="flat", numel=1 << 20, grads="bf16"),
        # embedding, head and two layers of Llama-3.1-8B: the norm that the fused step takes its factor from
        dict(name="norm_llama_2l", op="norm", list="llama", layers=2, grads="bf16"),
        # adapters, norms and biases: tensors of every awkward size, latency
        dict(name="clip_odd_sizes", op="clip", list="mixed", numel=250_000, tensors=25, shape=7, grads="bf16"),
        # gradients accumulated in FP32 over several batches, clipped into the BF16 ones that the step reads
        dict(name="clip_gpt2_accumulated", op="clip", list="gpt2", grads="fp32"),
        # one token that was just generated
        dict(name="logprob_1_token", op="logprob", rows=1, vocab=128256, dtype="bf16", masked=0, temperature=0.7),
        # the old or the reference policy over a batch of answers behind their prompts
        dict(name="logprob_8192_tokens", op="logprob", rows=8192, vocab=50257, dtype="bf16", masked=2500, temperature=1.0),
        # a handful of tokens over a small, odd vocabulary
        dict(name="policy_12_tokens", op="policy", rows=12, vocab=1001, dtype="fp32", masked=2, temperature=1.0, kl=0.02,
             on_policy=False),
        # a ragged micro-batch with FP32 logits
        dict(name="policy_gpt2_fp32", op="policy", rows=1001, vocab=50257, dtype="fp32", masked=0, temperature=0.9, kl=0.0,
             on_policy=False),
        # the largest: a batch of answers over Llama-3.1-8B's vocabulary, KL to the reference
        dict(name="policy_4096_tokens", op="policy", rows=4096, vocab=128256, dtype="bf16", masked=512, temperature=1.0, kl=0.05,
             on_policy=False),
        # one short pair
        dict(name="preference_1_pair", op="preference", rows=45, vocab=32000, dtype="bf16", masked=10, pairs=1, kind="sigmoid",
             smoothing=0.0),
        # a batch of pairs, a third of the rows prompts
        dict(name="preference_8_pairs", op="preference", rows=4100, vocab=50257, dtype="bf16", masked=1400, pairs=8,
             kind="sigmoid", smoothing=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "clip", "logprob", "policy", "policy", "preference"])
    if op in ("norm", "clip"):
        c = dict(op=op, numel=_log_int(rng, 1000, 700_000_000 if op == "norm" else 200_000_000),
                 grads=rng.choice(["bf16", "bf16", "fp32"]))
        if rng.random() < 0.25:
            c["list"] = "flat"
        else:
            c.update(list="mixed", tensors=_log_int(rng, 2, 400), shape=rng.randrange(1 << 20))
        return c
    vocab = _log_int(rng, 300, 131072)
    if rng.random() < 0.5:
        vocab = max(320, vocab // 64 * 64)
    rows = min(_log_int(rng, 1, 8192), LARGEST // vocab)
    c = dict(op=op, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if c["dtype"] == "fp32":
        rows = max(1, rows // 2)
    if op == "preference":
        c["pairs"] = _log_int(rng, 1, 64)
        rows = max(rows, 2 * c["pairs"] + 3)
        c.update(kind=rng.choice(["sigmoid", "sigmoid", "hinge", "squared"]), smoothing=0.0)
        if c["kind"] == "sigmoid":
            c["smoothing"] = rng.choice([0.0, 0.05, 0.2])
    else:
        c["temperature"] = rng.choice([1.0, 1.0, 0.6, 1.3])
    if op == "policy":
        c.update(kl=rng.choice([0.0, 0.01, 0.1]), on_policy=rng.random() < 0.3)
    c.update(rows=rows, masked=int(rows * rng.choice([0.0, 0.1, 0.4])))
    return c


def work(case):
    c = case
    if c["op"] in ("norm", "clip"):
        n, s = sum(_sizes(c)), 2 if c["grads"] == "bf16" else 4
        return {"bytes": n * (s + (2 if c["op"] == "clip" else 0)) + 16, "flops": n * (3 if c["op"] == "clip" else 2)}
    rows, vocab, s = c["rows"], c["vocab"], 2 if c["dtype"] == "bf16" else 4
    counted = rows - c["masked"]
    read = counted * vocab * s + 8 * rows
    if c["op"] == "logprob":
        return {"bytes": read + 8 * rows, "flops": 4 * counted * vocab}
    if c["op"] == "policy":
        given = 2 + (0 if c["on_policy"] else 1) + (1 if c["kl"] else 0)
        return {"bytes": read + rows * vocab * s + 4 * rows * (given + 1), "flops": 8 * counted * vocab}
    return {"bytes": read + rows * vocab * s + 4 * rows * 3 + 8 * (2 * c["pairs"] + 1), "flops": 8 * counted * vocab}


# --------------------------------------------------------------------------------------------------- inputs --

def _sizes(c):
    """The element counts of the case's list."""
    if c["list"] == "flat":
        return [c["numel"]]
    if c["list"] == "gpt2":
        d = 768
        layer = [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * 4 * d, 4 * d, 4 * d * d, d]
        return [50257 * d, 1024 * d] + 12 * layer + [d, d]
    if c["list"] == "llama":
        d, kv, f = 4096, 1024, 14336
        layer = [d * d, kv * d, kv * d, d * d, f * d, f * d, d * f, d, d]
        return [128256 * d] + c["layers"] * layer + [d, 128256 * d]
    r = random.Random(c["shape"])
    share = [math.exp(r.uniform(0.0, 9.0)) for _ in range(c["tensors"])]
    return [max(1, int(c["numel"] * x / sum(share))) for x in share]


def _layout(sizes):
    """First element of every tensor in one array that holds them all, each on a multiple of 256, and its length."""
    first, end = [], 0
    for n in sizes:
        first.append(end)
        end += (n + 255) // 256 * 256
    return first, end


def _rng(seed, what=0):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 8 + what)


def _gradients(c, seed):
    """All gradients in one array (zero between the tensors), each tensor of a size of its own, some values far out."""
    g, sizes = _rng(seed), _sizes(c)
    first, end = _layout(sizes)
    flat = torch.zeros(end, dtype=TYPES[c["grads"]], device="cuda")
    for f, n in zip(first, sizes):
        x = torch.randn(n, generator=g, device="cuda")
        size = torch.exp(torch.randn(1, generator=g, device="cuda")) * (8.0 / math.sqrt(end))
        flat[f:f + n] = x.mul_(size)
    return flat, first, sizes


def _chunks(rows, vocab):
    step = max(1, (1 << 26) // vocab)
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _logits(c, seed):
    """Logits whose rows have one more likely token of uneven height, and for each row a token drawn from them."""
    g, rows, vocab = _rng(seed), c["rows"], c["vocab"]
    t = c.get("temperature", 1.0)
    logits = torch.empty(rows, vocab, dtype=TYPES[c["dtype"]], device="cuda")
    tokens = torch.empty(rows, dtype=torch.int64, device="cuda")
    logp = torch.empty(rows, device="cuda")
    for a, b in _chunks(rows, vocab):
        x = torch.randn(b - a, vocab, generator=g, device="cuda").mul_(2.5)
        top = torch.randint(0, vocab, (b - a, 1), generator=g, device="cuda")
        x.scatter_add_(1, top, 4 + 14 * torch.rand(b - a, 1, generator=g, device="cuda"))
        logits[a:b] = x
        x = logits[a:b].float().div_(t)
        u = torch.rand(b - a, vocab, generator=g, device="cuda").clamp_(min=1e-30)
        tokens[a:b] = (x - u.log_().neg_().log_()).argmax(1)
        logp[a:b] = x.gather(1, tokens[a:b, None])[:, 0] - torch.logsumexp(x, 1)
    masked = torch.randperm(rows, generator=g, device="cuda")[:c["masked"]]
    return logits, tokens, logp, masked


def _lengths(c):
    """The bounds of the 2 `pairs` sequences among the rows, of uneven lengths, the last one at the end."""
    n = 2 * c["pairs"]
    r = random.Random(c["rows"] * 64 + c["pairs"])
    cuts = sorted(r.randrange(c["rows"] + 1) for _ in range(n - 1))
    return [0] + cuts + [c["rows"]]


def _inputs(c, seed):
    """What a loss is given."""
    s = {}
    s["logits"], s["tokens"], logp, masked = _logits(c, seed)
    g, rows = _rng(seed, 1), c["rows"]
    near = lambda size: logp + size * torch.randn(rows, generator=g, device="cuda")      # noqa: E731
    if c["op"] == "logprob":
        s["tokens"][masked] = -100
        return s
    s["weights"] = torch.ones(rows, device="cuda")
    s["weights"][masked] = 0
    if c["op"] == "policy":
        s["weights"] /= max(1, rows - c["masked"])
        s["advantages"] = torch.randn(rows, generator=g, device="cuda")
        s["old"] = None if c["on_policy"] else near(0.15)
        s["ref"] = near(0.2) if c["kl"] else None
    else:
        s["tokens"][masked] = -100
        s["ref"] = near(0.3)
        s["offsets"] = torch.tensor(_lengths(c), dtype=torch.int64, device="cuda")
    return s


def prepare(case, seed):
    c = dict(case)
    if c["op"] in ("norm", "clip"):
        flat, first, sizes = _gradients(c, seed)
        s = {"case": c, "grads": flat, "out": torch.zeros_like(flat, dtype=BF16) if c["op"] == "clip" else None}
        if own:
            import paper_2602_23349_amd as fo
            views = lambda x: [x[f:f + n] for f, n in zip(first, sizes)]      # noqa: E731
            s["list"] = fo.GradList(views(flat), None if s["out"] is None else views(s["out"]))
            s["clip"] = fo.ClipFactor()
            s["workspace"] = torch.empty(fo.grad_norm_workspace(s["list"]), dtype=torch.uint8, device="cuda")
        return s
    s = {"case": c, **_inputs(c, seed)}
    rows = c["rows"]
    s["logprob"] = torch.empty(rows, device="cuda")
    s["lse"] = torch.empty(rows, device="cuda")
    if c["op"] != "logprob":
        s["dlogits"] = torch.empty_like(s["logits"])
    if c["op"] == "policy":
        s["stats"] = torch.empty(4, device="cuda")
    if c["op"] == "preference":
        s["loss"], s["margins"] = torch.empty(1, device="cuda"), torch.empty(c["pairs"], device="cuda")
        s["dlogprob"] = torch.empty(rows, device="cuda")
    if own:
        import paper_2602_23349_amd as fo
        if c["op"] == "policy":
            s["spec"] = fo.PolicyLoss(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_weight=c["kl"], temperature=c["temperature"])
            size = fo.policy_loss_workspace(s["logits"])
        else:
            size = fo.token_logprob_workspace(s["logits"])
        if c["op"] == "preference":
            s["logprob64"] = torch.empty(rows, dtype=FP64, device="cuda")
            s["spec"] = fo.PreferenceLoss(beta=BETA, kind=c["kind"], label_smoothing=c["smoothing"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ run --

def run(state):
    return _own_run(state) if own else _plain_run(state)


def _own_run(s):
    import paper_2602_23349_amd as fo
    c = s["case"]
    if c["op"] in ("norm", "clip"):
        fo.grad_norm(s["list"], MAX_NORM, s["clip"], workspace=s["workspace"])
        out = {"norm": s["clip"].norm, "scale": s["clip"].scale}
        if c["op"] == "clip":
            fo.clip_gradients(s["list"], s["clip"])
            out["grads"] = s["out"]
        return out
    if c["op"] == "policy":
        fo.policy_loss(s["spec"], s["logits"], s["tokens"], s["advantages"], s["stats"], old_logprob=s["old"],
                       ref_logprob=s["ref"], weights=s["weights"], logprob=s["logprob"], dlogits=s["dlogits"],
                       workspace=s["workspace"])
        return {"stats": s["stats"], "logprob": s["logprob"], "dlogits": s["dlogits"]}
    fo.token_logprob(s["logits"], s["tokens"], s["logprob"], s["lse"], temperature=c.get("temperature", 1.0),
                     logprob64=s.get("logprob64"), workspace=s["workspace"])
    if c["op"] == "logprob":
        return {"logprob": s["logprob"], "lse": s["lse"]}
    fo.preference_loss(s["spec"], s["logprob64"], s["offsets"], s["loss"], ref_logprob=s["ref"], weights=s["weights"],
                       margins=s["margins"], dlogprob=s["dlogprob"])
    fo.token_logprob_backward(s["logits"], s["tokens"], s["lse"], s["dlogprob"], s["dlogits"])
    return {"loss": s["loss"], "margins": s["margins"], "logprob": s["logprob"], "dlogits": s["dlogits"]}


def _log_probabilities(logits, tokens, temperature):
    """The scaled logits in FP32, and in FP64 the log of their sum of exponentials and the tokens' log-probabilities."""
    x = logits.float() if temperature == 1.0 else logits.float() / temperature
    most = x.max(1, keepdim=True).values
    lse = (x - most).exp_().sum(1, dtype=FP64).log() + most[:, 0]
    return x, lse, x.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - lse


def _logit_gradient(x, lse, tokens, d, dtype):
    """d ([j = token] - exp(x - lse)).  (x may be the logits themselves.)"""
    x = (x - lse[:, None].float()).exp_().mul_(-d[:, None].float())
    return x.scatter_add_(1, tokens.clamp(min=0)[:, None], d[:, None].float()).to(dtype)


def _plain_run(s):
    c = s["case"]
    if c["op"] in ("norm", "clip"):
        norm = s["grads"].float().square().sum(dtype=FP64).sqrt().reshape(1)
        scale = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
        out = {"norm": norm.float(), "scale": scale.float()}
        if c["op"] == "clip":
            out["grads"] = (s["grads"].float() * out["scale"]).to(BF16)
        return out
    x, lse, logp = _log_probabilities(s["logits"], s["tokens"], c.get("temperature", 1.0))
    counted = s["tokens"] >= 0
    zero = torch.zeros_like(lse)
    if c["op"] == "logprob":
        return {"logprob": torch.where(counted, logp, zero).float(), "lse": torch.where(counted, lse, zero).float()}
    w = s["weights"].double()
    if c["op"] == "policy":
        a, counted = s["advantages"].double(), w != 0
        ratio = torch.ones_like(logp) if s["old"] is None else (logp - s["old"]).exp()
        blocked = ((a > 0) & (ratio > 1 + CLIP_HIGH)) | ((a < 0) & (ratio < 1 - CLIP_LOW))
        surrogate = -torch.minimum(ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a)
        d = -a * ratio * ~blocked
        kl = zero
        if s["ref"] is not None:
            e = s["ref"] - logp
            kl = torch.expm1(e) - e
            d = d - c["kl"] * torch.expm1(e)
        sums = [(w * surrogate).sum(), (w * kl).sum(), (w * blocked).sum()]
        grad = _logit_gradient(x, lse, s["tokens"], w * d / c["temperature"], s["logits"].dtype)
        return {"stats": torch.stack([sums[0] + c["kl"] * sums[1]] + sums).float(),
                "logprob": torch.where(counted, logp, zero).float(), "dlogits": grad}
    logp = torch.where(counted, logp, zero)
    gain = (w * (logp - s["ref"])).cumsum(0)
    gain = torch.cat([gain.new_zeros(1), gain])[s["offsets"]].diff().view(-1, 2)
    margin = BETA * (gain[:, 0] - gain[:, 1])
    if c["kind"] == "sigmoid":
        e = c["smoothing"]
        soft = lambda v: v.clamp(min=0) + torch.log1p((-v.abs()).exp())      # noqa: E731
        loss = (1 - e) * soft(-margin) + e * soft(margin)
        d = e / (1 + (-margin).exp()) - (1 - e) / (1 + margin.exp())
    elif c["kind"] == "hinge":
        loss, d = (1 - margin).clamp(min=0), -(margin < 1).double()
    else:
        r = (margin - 0.5) / BETA
        loss, d = r.square(), 2 * r / BETA
    d = torch.stack([d, -d], 1).flatten() * (BETA / c["pairs"])
    of = torch.searchsorted(s["offsets"], torch.arange(c["rows"], device=w.device), right=True) - 1
    d = w * d[of]
    return {"loss": loss.mean().float().reshape(1), "margins": margin.float(), "logprob": logp.float(),
            "dlogits": _logit_gradient(x, lse, s["tokens"], d, s["logits"].dtype)}


# ---------------------------------------------------------------------------------------------------- exact --

def exact(case, seed):
    c = dict(case)
    if c["op"] in ("norm", "clip"):
        flat, _, _ = _gradients(c, seed)
        total = sum(float(p.double().pow(2).sum()) for p in flat.split(1 << 27))
        norm = math.sqrt(total)
        scale = min(1.0, MAX_NORM / norm) if norm else 1.0
        out = {"norm": torch.tensor([norm], dtype=FP64), "scale": torch.tensor([scale], dtype=FP64)}
        if c["op"] == "clip":
            out["grads"] = flat.double() * scale
        return out
    s = _inputs(c, seed)
    rows, t = c["rows"], c.get("temperature", 1.0)
    tokens = s["tokens"]
    logp, lse = torch.zeros(rows, dtype=FP64, device="cuda"), torch.zeros(rows, dtype=FP64, device="cuda")
    for a, b in _chunks(rows, c["vocab"]):
        x = s["logits"][a:b].double() / t
        lse[a:b] = torch.logsumexp(x, 1)
        logp[a:b] = x[torch.arange(b - a), tokens[a:b].clamp(min=0)] - lse[a:b]
    if c["op"] == "logprob":
        keep = (tokens >= 0).double()
        return {"logprob": logp * keep, "lse": lse * keep}
    w = s["weights"].double()
    keep = (w != 0).double()
    logp = logp * keep
    out = {"logprob": logp}
    if c["op"] == "policy":
        adv = s["advantages"].double()
        ratio = torch.exp(logp - s["old"].double()) if s["old"] is not None else torch.ones_like(logp)
        low, high = 1 - CLIP_LOW, 1 + CLIP_HIGH
        held = torch.minimum(torch.maximum(ratio, ratio.new_tensor(low)), ratio.new_tensor(high))
        inside = torch.where(adv >= 0, ratio <= high, ratio >= low)
        slope = torch.where(inside, -adv * ratio, 0.0)
        kl = torch.zeros_like(logp)
        if s["ref"] is not None:
            gap = s["ref"].double() - logp
            kl = torch.expm1(gap) - gap
            slope = slope + c["kl"] * (1 - torch.exp(gap))
        parts = [-(w * torch.minimum(ratio * adv, held * adv)).sum(), (w * kl).sum(),
                 (w * (~inside & (adv != 0)).double()).sum()]
        out["stats"] = torch.stack([parts[0] + c["kl"] * parts[1], *parts])
        slope = w * slope / t
    else:
        n, bounds = c["pairs"], _lengths(c)
        gain = [float((w[a:b] * (logp[a:b] - s["ref"][a:b].double())).sum()) for a, b in zip(bounds, bounds[1:])]
        loss, slope, margins = 0.0, torch.zeros(rows, dtype=FP64, device="cuda"), []
        for p in range(n):
            z = BETA * (gain[2 * p] - gain[2 * p + 1])
            if c["kind"] == "sigmoid":
                up, e = 1 / (1 + math.exp(-z)), c["smoothing"]
                loss += -(1 - e) * math.log(up) - e * math.log1p(-up)
                dz = e * up - (1 - e) * (1 - up)
            elif c["kind"] == "hinge":
                loss, dz = loss + max(0.0, 1 - z), -1.0 if z < 1 else 0.0
            else:
                loss, dz = loss + (z / BETA - 1 / (2 * BETA)) ** 2, 2 * (z / BETA - 1 / (2 * BETA)) / BETA
            margins.append(z)
            for q, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
                a, b = bounds[q], bounds[q + 1]
                slope[a:b] = sign * dz * BETA / n * w[a:b]
        out["loss"], out["margins"] = torch.tensor([loss / n], dtype=FP64), torch.tensor(margins, dtype=FP64)
    grad = torch.zeros(rows, c["vocab"], dtype=FP64, device="cuda")
    for a, b in _chunks(rows, c["vocab"]):
        p = torch.exp(s["logits"][a:b].double() / t - lse[a:b, None])
        p[torch.arange(b - a), tokens[a:b].clamp(min=0)] -= 1
        grad[a:b] = -p * slope[a:b, None]
    out["dlogits"] = grad
    return out
