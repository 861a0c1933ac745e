"""The operators of a low-precision transformer block around the optimizer step, as a training or serving program calls
them, each beside its plain form.

With `own` false, `run` computes an operator in elementary torch operations in 32 bits, rounded once at the end; with
`own` true it calls this package.  `exact` gives the same outputs from the definitions in 64 bits.

A case is a dict of plain values:
  op   quantize          a matrix to microscaled 4-bit floating point (blocks of 32 along a row share a power-of-two
                         scale) along its rows and, with `both`, along its columns, and the values back
       linear            y = Q(x) W^T on 4-bit weights; with `train`, Q(x^T) is kept for the backward pass
       linear_backward   dx = Q(dy) Q(W^T)^T and dW = Q(dy^T) Q(x^T)^T
       norm              h = a x + b act(gate) norm(f), y = norm(h), the statistics for the backward pass
       norm_backward     the gradients of all of that
  source   bf16, fp32 or split: a BF16 weight and its 8-bit correction
  random   the rounding is stochastic, with the given random bytes
  kind     rms or layer;  post: no branch ("none"), a branch as it is ("plain") or normalised ("norm")
  gate     none, or one row of gates for all rows ("channel"), for each `rows / groups` of them ("sample") or for each
           row ("token");  act: linear or sigmoid
  stream, branch   types of the residual stream (x, h) and of the branch (f, gate, y);  weights are BF16
"""
import math

import torch

own = False

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = {"bf16": BF16, "fp32": FP32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5


def listed():
    return [
        # a matrix of gradients of an odd size, stochastically rounded along its rows: a small call
        dict(name="quantize_odd_random", op="quantize", rows=257, cols=1000, source="bf16", both=False, random=True),
        # the 4-bit copies of the largest matrix of a Llama-3.1-8B layer, made from the split weight after a step
        dict(name="quantize_weight_split", op="quantize", rows=14336, cols=4096, source="split", both=True, random=False),
        # one token through an attention projection and eight through an up projection: serving
        dict(name="linear_1_token", op="linear", m=1, k=4096, n=4096, out="bf16", train=False),
        dict(name="linear_8_tokens", op="linear", m=8, k=4096, n=14336, out="bf16", train=False),
        # a GPT-2 sized projection of a ragged batch in training
        dict(name="linear_gpt2_train", op="linear", m=1001, k=768, n=2304, out="bf16", train=True),
        # the largest product: a prompt or batch of 8192 tokens through a layer's up projection
        dict(name="linear_8192_tokens", op="linear", m=8192, k=4096, n=14336, out="bf16", train=False),
        # gradients of a GPT-2 sized projection, dy rounded stochastically
        dict(name="linear_gpt2_backward", op="linear_backward", m=1024, k=768, n=2304, random=True),
        # gradients of a down projection over 4096 tokens
        dict(name="linear_down_backward", op="linear_backward", m=4096, k=14336, n=4096, random=False),
        # one token between two blocks: norm behind the branch, gate, residual, norm in front of the next
        dict(name="norm_1_token", op="norm", rows=1, cols=4096, kind="rms", post="norm", gate="channel", groups=1,
             act="linear", pre=True, stream="bf16", branch="bf16"),
        # a large batch: residual addition of the branch as it is, norm in front of the next block
        dict(name="norm_16384_tokens", op="norm", rows=16384, cols=4096, kind="rms", post="plain", gate="none", groups=1,
             act="linear", pre=True, stream="bf16", branch="bf16"),
        # a ragged batch with layer norms, FP32 residual stream and a sigmoid gate for each sample
        dict(name="norm_backward_layer", op="norm_backward", rows=1995, cols=768, kind="layer", post="norm", gate="sample",
             groups=3, act="sigmoid", pre=True, stream="fp32", branch="bf16"),
        # a training batch between two blocks, both norms, a gate for each channel
        dict(name="norm_backward_8192_tokens", op="norm_backward", rows=8192, cols=4096, kind="rms", post="norm",
             gate="channel", groups=1, act="linear", pre=True, stream="bf16", branch="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A matrix dimension: mostly a multiple of 64 or 16, as models have them, else any."""
    n, unit = _log_int(rng, lo, hi), rng.choice([64, 64, 16, 1])
    return max(unit, n // unit * unit)


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear_backward", "norm", "norm_backward"])
    if op == "quantize":
        rows, cols = _log_int(rng, 1, 14336), _width(rng, 32, 14336)
        rows = min(rows, 14336 * 4096 // cols)
        source = rng.choice(["bf16", "bf16", "fp32", "split"])
        return dict(op=op, rows=rows, cols=cols, source=source, both=rng.random() < 0.6, random=rng.random() < 0.4)
    if op == "linear":
        m, k, n = _log_int(rng, 1, 8192), _width(rng, 64, 14336), _width(rng, 64, 14336)
        m = min(m, 8192 * 4096 * 14336 // (k * n))
        return dict(op=op, m=m, k=k, n=n, out=rng.choice(["bf16", "bf16", "fp32"]), train=rng.random() < 0.4)
    if op == "linear_backward":
        m, k, n = _log_int(rng, 16, 8192), _width(rng, 64, 14336), _width(rng, 64, 14336)
        m = min(m, 4096 * 4096 * 14336 // (k * n))
        return dict(op=op, m=m, k=k, n=n, random=rng.random() < 0.5)
    c = dict(op=op, rows=_log_int(rng, 1, 16384), cols=_width(rng, 64, 8192), kind=rng.choice(["rms", "rms", "layer"]),
             post=rng.choice(["none", "plain", "norm", "norm"]), gate="none", groups=1, act="linear", pre=True,
             stream=rng.choice(["bf16", "bf16", "fp32"]), branch="bf16")
    most = 16384 * 4096 if op == "norm" else 8192 * 4096
    c["rows"] = max(1, min(c["rows"], most // c["cols"]))
    if c["post"] != "none":
        c["gate"], c["act"] = rng.choice(["none", "channel", "sample", "token"]), rng.choice(["linear", "sigmoid"])
        c["pre"] = rng.random() < 0.8
        if c["gate"] == "sample":
            c["groups"] = rng.choice([2, 3, 8])
            c["rows"] = max(1, c["rows"] // c["groups"]) * c["groups"]
    if c["stream"] == "fp32" and rng.random() < 0.3:
        c["branch"] = "fp32"
    return c


def _up(n, unit):
    return (n + unit - 1) // unit * unit


def _norm_sizes(c):
    """(rows, cols, rows of gates, bytes of a value of the stream, of the branch)."""
    gates = {"none": 0, "channel": 1, "sample": c["groups"], "token": c["rows"]}[c["gate"]]
    return c["rows"], c["cols"], gates, 2 if c["stream"] == "bf16" else 4, 2 if c["branch"] == "bf16" else 4


def work(case):
    c = case
    q = 0.5 + 1 / 32
    if c["op"] == "quantize":
        n = c["rows"] * c["cols"]
        layouts = 2 if c["both"] else 1
        read = {"bf16": 2, "fp32": 4, "split": 3}[c["source"]] + (1 if c["random"] else 0)
        return {"bytes": n * (read + layouts * (2 * q + 2)), "flops": 2 * n * layouts}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        kept = m * k * (2 * q + 2) if c["train"] else 0
        return {"bytes": 2 * m * k + q * n * k + (2 if c["out"] == "bf16" else 4) * m * n + kept, "flops": 2 * m * n * k}
    if c["op"] == "linear_backward":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": (3 if c["random"] else 2) * m * n + q * (n * k + m * k) + 2 * m * k + 2 * n * k,
                "flops": 4 * m * n * k}
    rows, cols, gates, s, b = _norm_sizes(c)
    per = 2 if c["kind"] == "layer" else 1
    norms = (1 if c["post"] == "norm" else 0) + (1 if c["pre"] else 0)
    branch = c["post"] != "none"
    n = rows * cols
    if c["op"] == "norm":
        data = n * s + (n * (b + s) if branch else 0) + (n * b if c["pre"] else 0)
        return {"bytes": data + gates * cols * b + 2 * norms * per * cols + 16 * rows, "flops": n * (4 * norms + 3)}
    data = n * s + (n * (b + s + b) if branch else 0) + (n * b if c["pre"] else 0) + n * s
    return {"bytes": data + 2 * gates * cols * b + (2 * norms + 2 * norms * per) * cols + 16 * rows,
            "flops": n * (10 * norms + 4)}


# --------------------------------------------------------------------------------------------------- inputs --

def _rng(seed, what=0):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 8 + what)


def _activations(g, rows, cols, dtype):
    """Normal values with a few channels far above the others, as hidden states have them."""
    loud = 1 + 15 * (torch.rand(cols, generator=g, device="cuda") < 0.01)
    return (torch.randn(rows, cols, generator=g, device="cuda") * loud).to(dtype)


def _gradients(g, rows, cols, dtype):
    """Small values, each row of its own size, and rows of masked tokens that are zero."""
    size = 1e-4 * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    size *= torch.rand(rows, 1, generator=g, device="cuda") >= 0.05
    return (torch.randn(rows, cols, generator=g, device="cuda") * size).to(dtype)


def _random_bytes(g, rows, cols):
    return torch.randint(0, 256, (rows, cols), generator=g, device="cuda", dtype=torch.uint8)


def _pack(values):
    """The codes (two to a byte, the even element in the low half, rows filled up to a multiple of 256) and scale bytes
    (rows filled up to a multiple of 16) of a matrix that a program has as 4-bit weights or kept activations."""
    rows, cols = values.shape
    wide = _up(cols, 256)
    t, byte, sign = _scaled(torch.nn.functional.pad(values.float(), (0, wide - cols)), False)
    code = _nearest_code(t) + 8 * sign
    code = code.to(torch.uint8).reshape(rows, wide // 2, 2)
    byte = torch.nn.functional.pad(byte.to(torch.uint8), (0, _up(wide // 32, 16) - wide // 32))
    return (code[..., 0] | code[..., 1] << 4).contiguous(), byte.contiguous()


def prepare(case, seed):
    c, g = dict(case), _rng(seed)
    s = {"case": c}
    if c["op"] == "quantize":
        rows, cols = c["rows"], c["cols"]
        if c["source"] == "split":
            s["x"] = (torch.randn(rows, cols, generator=g, device="cuda") * 0.02).to(BF16)
            s["rho"] = torch.randint(-127, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
        else:
            s["x"] = _gradients(g, rows, cols, TYPES[c["source"]])
        if c["random"]:
            s["rand"] = _random_bytes(g, rows, cols)
        s["out"] = torch.empty(rows, cols, dtype=BF16, device="cuda")
        s["out_t"] = torch.empty(cols, rows, dtype=BF16, device="cuda") if c["both"] else None
        if own:
            import paper_2602_23349_amd as fo
            s["q"], s["qt"] = fo.Mx4Tensor(rows, cols), fo.Mx4Tensor(cols, rows) if c["both"] else None
    elif c["op"] in ("linear", "linear_backward"):
        m, k, n = c["m"], c["k"], c["n"]
        w = torch.randn(n, k, generator=g, device="cuda") * 0.02
        if c["op"] == "linear":
            s["x"] = _activations(g, m, k, BF16)
            s["w"] = _pack(w)
            s["y"] = torch.empty(m, n, dtype=TYPES[c["out"]], device="cuda")
            s["xt_values"] = torch.empty(k, m, dtype=BF16, device="cuda") if c["train"] else None
        else:
            s["dy"] = _gradients(g, m, n, BF16)
            s["wt"] = _pack(w.t())
            s["xt"] = _pack(_activations(g, m, k, BF16).t())
            if c["random"]:
                s["rand"] = _random_bytes(g, m, n)
            s["dx"] = torch.empty(m, k, dtype=BF16, device="cuda")
            s["dw"] = torch.empty(n, k, dtype=BF16, device="cuda")
        if own:
            import paper_2602_23349_amd as fo
            if c["op"] == "linear":
                s["w_own"] = fo.Mx4Tensor(n, k, buffers=s["w"])
                s["xt_own"] = fo.Mx4Tensor(k, m) if c["train"] else None
                size = fo.mx4_linear_workspace(m, n, k)
            else:
                s["wt_own"], s["xt_own"] = fo.Mx4Tensor(k, n, buffers=s["wt"]), fo.Mx4Tensor(k, m, buffers=s["xt"])
                size = fo.mx4_linear_backward_workspace(m, n, k)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    else:
        _prepare_norm(s, c, g)
    return s


def _prepare_norm(s, c, g):
    rows, cols, gates, _, _ = _norm_sizes(c)
    stream, branch = TYPES[c["stream"]], TYPES[c["branch"]]
    near_one = lambda: (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(BF16)     # noqa: E731
    near_zero = lambda: (0.1 * torch.randn(cols, generator=g, device="cuda")).to(BF16)        # noqa: E731
    layer, post, pre = c["kind"] == "layer", c["post"] == "norm", c["pre"]
    s["post_weight"], s["post_bias"] = near_one() if post else None, near_zero() if post and layer else None
    s["pre_weight"], s["pre_bias"] = near_one() if pre else None, near_zero() if pre and layer else None
    s["residual_scale"], s["branch_scale"] = 1.0, 0.5
    s["x"] = _activations(g, rows, cols, stream)
    s["f"] = _activations(g, rows, cols, branch) * 0.5 if c["post"] != "none" else None
    s["gate"] = torch.randn(gates, cols, generator=g, device="cuda").to(branch) if gates else None
    empty = lambda like: None if like is None else torch.empty_like(like)                      # noqa: E731
    if c["op"] == "norm":
        s["h"] = empty(s["x"]) if s["f"] is not None else None
        s["y"] = torch.empty(rows, cols, dtype=branch, device="cuda") if pre else None
        s["stats"] = torch.zeros(4, rows, device="cuda")
    else:
        h, _, s["stats"] = _plain_norm(s, c)
        s["h"] = h.to(stream)
        del s["x"]
        s["dy"] = _gradients(g, rows, cols, branch) if pre else None
        s["dh"] = _gradients(g, rows, cols, stream)
        s["dx"], s["df"], s["dgate"] = empty(s["dh"]), empty(s["f"]), empty(s["gate"])
        for name in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
            s["d" + name] = empty(s[name])
    if own:
        import paper_2602_23349_amd as fo
        s["plan"] = fo.BlockNorm(cols, kind=c["kind"], eps=EPS, post_norm=post, gate_act=c["act"],
                                 residual_scale=s["residual_scale"], branch_scale=s["branch_scale"],
                                 post_weight=s["post_weight"], post_bias=s["post_bias"],
                                 pre_weight=s["pre_weight"], pre_bias=s["pre_bias"])
        if c["op"] == "norm_backward":
            size = fo.block_norm_backward_workspace(s["plan"], rows, max(gates, 1))
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------- plain forms --

def _scaled(v, random):
    """(|v| over its block's scale, scale bytes, sign) of an FP32 matrix whose rows are whole blocks of 32."""
    rows, wide = v.shape
    bits = v.reshape(rows, wide // 32, 32).view(torch.int32)
    largest = (bits & 0x7FFFFFFF).amax(-1, keepdim=True)
    byte = (largest >> 23) - 2
    if random:
        byte = byte + ((largest & 0x7FFFFF) > 0x400000).int()
    byte = torch.where(largest >= 0x7F800000, 255, byte.clamp(min=0))
    up = torch.where(byte < 254, (254 - byte) << 23, 0).view(FP32)            # 2^(127 - byte)
    t = (bits & 0x7FFFFFFF).view(FP32) * up
    t = torch.where(byte == 255, 0.0, t)
    return t.reshape(rows, wide), byte.reshape(rows, wide // 32), (bits < 0).int().reshape(rows, wide)


def _nearest_code(t):
    """Codes 0 to 7 of the grid values nearest to t, ties to the even code."""
    return torch.where(t < 2, torch.round(2 * t), torch.where(t < 4, 2 + torch.round(t), 4 + torch.round(t / 2))).clamp(max=7)


def _scale_of(byte):
    byte = byte.int()
    bits = torch.where(byte == 0, 0x00400000, torch.where(byte == 255, 0x7FC00000, byte << 23))
    return bits.view(FP32)                                                    # 2^(byte - 127), NaN for 255


def _plain_values(v, rand=None):
    """The values that the 4-bit form of an FP32 matrix stands for."""
    rows, cols = v.shape
    wide = _up(cols, 32)
    t, byte, sign = _scaled(torch.nn.functional.pad(v, (0, wide - cols)), rand is not None)
    if rand is None:
        q = torch.where(t < 2, torch.round(2 * t) / 2, torch.where(t < 4, torch.round(t), 2 * torch.round(t / 2))).clamp(max=6)
    else:
        step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
        low = torch.floor(t / step) * step
        q = low + step * ((t - low) / step * 256 > torch.nn.functional.pad(rand, (0, wide - cols)).float() + 0.5)
    q = torch.where(sign > 0, -q, q).reshape(rows, wide // 32, 32) * _scale_of(byte)[..., None]
    return q.reshape(rows, wide)[:, :cols]


def _plain_unpack(packed, cols):
    """The FP32 values of codes and scale bytes."""
    codes, byte = packed
    rows = codes.shape[0]
    table = torch.tensor(GRID + tuple(-v for v in GRID), device="cuda")
    q = table[torch.stack((codes & 15, codes >> 4), -1).long()]
    q = q.reshape(rows, -1, 32)
    return (q * _scale_of(byte)[:, :q.shape[1], None]).reshape(rows, -1)[:, :cols]


def _plain_master(param, rho):
    """The FP32 weight that a BF16 weight and its 8-bit correction stand for."""
    base = param.float()
    half_ulp = ((((base.view(torch.int32) >> 23) & 255).clamp(min=9) - 8) << 23).view(FP32)   # (smaller weights round to 0)
    fraction = (torch.arange(-128, 128, dtype=torch.float64, device="cuda") / 127).float()
    return base + fraction[rho.int() + 128] * half_ulp


def _moments(v, layer):
    mean = v.mean(-1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    return mean, torch.rsqrt((v - mean).square().mean(-1, keepdim=True) + EPS)


def _affine(v, weight, bias):
    v = v if weight is None else v * weight.float()
    return v if bias is None else v + bias.float()


def _gates(s, c, rows):
    """The gate of every row before its activation, and the activation, or None."""
    if s["gate"] is None:
        return None, None
    gate = s["gate"].float().repeat_interleave(rows // s["gate"].shape[0], 0)
    return gate, torch.sigmoid(gate) if c["act"] == "sigmoid" else gate


def _plain_norm(s, c):
    x, layer = s["x"].float(), c["kind"] == "layer"
    nothing = torch.zeros_like(x[:, :1])
    post = pre = (nothing, nothing)
    h = x
    if s["f"] is not None:
        u = s["f"].float()
        if c["post"] == "norm":
            post = _moments(u, layer)
            u = _affine((u - post[0]) * post[1], s["post_weight"], s["post_bias"])
        _, act = _gates(s, c, x.shape[0])
        h = s["residual_scale"] * x + s["branch_scale"] * (u if act is None else act * u)
    y = None
    if c["pre"]:
        pre = _moments(h, layer)
        y = _affine((h - pre[0]) * pre[1], s["pre_weight"], s["pre_bias"])
    return h, y, torch.cat([post[0], post[1], pre[0], pre[1]], 1).t().contiguous()


def _through_norm(grad, hat, rstd, layer):
    """The gradient in front of a norm from that of its normalised values."""
    back = grad - hat * (grad * hat).mean(-1, keepdim=True)
    return rstd * (back - grad.mean(-1, keepdim=True) if layer else back)


def _plain_norm_backward(s, c):
    layer, r = c["kind"] == "layer", {}
    post_mean, post_rstd, pre_mean, pre_rstd = (v[:, None] for v in s["stats"])
    total = s["dh"].float()
    if c["pre"]:
        dy = s["dy"].float()
        hat = (s["h"].float() - pre_mean) * pre_rstd
        total = total + _through_norm(dy * s["pre_weight"].float(), hat, pre_rstd, layer)
        r["dpre_weight"] = (dy * hat).sum(0).to(BF16)
        r["dpre_bias"] = dy.sum(0).to(BF16) if layer else None
    if s["f"] is None:
        return {**r, "dx": total.to(s["dx"].dtype)}
    r["dx"] = (s["residual_scale"] * total).to(s["dx"].dtype)
    f = s["f"].float()
    hat = (f - post_mean) * post_rstd if c["post"] == "norm" else f
    u = _affine(hat, s["post_weight"], s["post_bias"])
    gate, act = _gates(s, c, f.shape[0])
    du = s["branch_scale"] * total
    if gate is not None:
        dgate = du * u * (act * (1 - act) if c["act"] == "sigmoid" else 1.0)
        r["dgate"] = dgate.reshape(s["gate"].shape[0], -1, f.shape[1]).sum(1).to(s["gate"].dtype)
        du = du * act
    if c["post"] == "norm":
        r["dpost_weight"] = (du * hat).sum(0).to(BF16)
        r["dpost_bias"] = du.sum(0).to(BF16) if layer else None
        du = _through_norm(du * s["post_weight"].float(), hat, post_rstd, layer)
    r["df"] = du.to(s["df"].dtype)
    return r


def _plain(s):
    c = s["case"]
    if c["op"] == "quantize":
        v = _plain_master(s["x"], s["rho"]) if c["source"] == "split" else s["x"].float()
        rand = s.get("rand")
        r = {"rows": _plain_values(v, rand).to(BF16)}
        if c["both"]:
            r["columns"] = _plain_values(v.t().contiguous(), None if rand is None else rand.t()).to(BF16)
        return r
    if c["op"] == "linear":
        x = s["x"].float()
        r = {"y": (_plain_values(x) @ _plain_unpack(s["w"], c["k"]).t()).to(s["y"].dtype)}
        if c["train"]:
            r["xt"] = _plain_values(x.t().contiguous()).to(BF16)
        return r
    if c["op"] == "linear_backward":
        dy, rand = s["dy"].float(), s.get("rand")
        dx = _plain_values(dy, rand) @ _plain_unpack(s["wt"], c["n"]).t()
        dw = _plain_values(dy.t().contiguous(), None if rand is None else rand.t()) @ _plain_unpack(s["xt"], c["m"]).t()
        return {"dx": dx.to(BF16), "dw": dw.to(BF16)}
    if c["op"] == "norm":
        h, y, stats = _plain_norm(s, c)
        return {"h": None if s["f"] is None else h.to(s["h"].dtype), "y": None if y is None else y.to(s["y"].dtype),
                "stats": stats}
    return _plain_norm_backward(s, c)


# ------------------------------------------------------------------------------------------------ the calls --

def _calls(s):
    import paper_2602_23349_amd as fo
    c = s["case"]
    if c["op"] == "quantize":
        fo.mx4_quantize(s["x"], s["q"], s["qt"], rho=s.get("rho"), rand=s.get("rand"))
        fo.mx4_dequantize(s["q"], s["out"])
        if not c["both"]:
            return {"rows": s["out"]}
        fo.mx4_dequantize(s["qt"], s["out_t"])
        return {"rows": s["out"], "columns": s["out_t"]}
    if c["op"] == "linear":
        fo.mx4_linear(s["x"], s["w_own"], s["y"], xt=s["xt_own"], workspace=s["workspace"])
        if not c["train"]:
            return {"y": s["y"]}
        fo.mx4_dequantize(s["xt_own"], s["xt_values"])
        return {"y": s["y"], "xt": s["xt_values"]}
    if c["op"] == "linear_backward":
        fo.mx4_linear_backward(s["dy"], s["wt_own"], s["xt_own"], s["dx"], s["dw"], rand=s.get("rand"),
                               workspace=s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if c["op"] == "norm":
        fo.block_norm(s["plan"], s["x"], f=s["f"], gate=s["gate"], h=s["h"], y=s["y"], stats=s["stats"])
        return {"h": s["h"], "y": s["y"], "stats": s["stats"]}
    names = ("dx", "df", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
    fo.block_norm_backward(s["plan"], s["h"], s["stats"], f=s["f"], gate=s["gate"], dy=s["dy"], dh=s["dh"],
                           workspace=s["workspace"], **{name: s[name] for name in names})
    return {name: s[name] for name in names}


def run(state):
    return _calls(state) if own else _plain(state)


# ------------------------------------------------------------------------------------- definitions in 64 bits --

def _exact_values(v, rand=None):
    """Each block of 32 of a row over the power of two that its largest value asks for, on the grid."""
    rows, cols = v.shape
    v = torch.nn.functional.pad(v, (0, _up(cols, 32) - cols)).reshape(rows, -1, 32)
    mantissa, exponent = torch.frexp(v.abs().amax(-1, keepdim=True))          # largest = mantissa 2^exponent, in [1/2, 1)
    exponent = exponent - 3 + (mantissa > 0.75).int() * (rand is not None)
    scale = torch.exp2(exponent.clamp(min=-127).double())
    t = (v / scale).abs()
    grid = torch.tensor(GRID, dtype=v.dtype, device=v.device)
    if rand is None:
        middle = (grid[1:] + grid[:-1]) / 2
        above, reached = torch.bucketize(t, middle), torch.bucketize(t, middle, right=True)
        code = torch.where(above % 2 == 0, above, reached)                    # a tie lies between the two: the even one
    else:
        low = torch.bucketize(t, grid, right=True) - 1
        high = (low + 1).clamp(max=7)
        rand = torch.nn.functional.pad(rand.double(), (0, _up(cols, 32) - cols)).reshape(v.shape)
        code = torch.where(t - grid[low] > (rand + 0.5) / 256 * (grid[high] - grid[low]), high, low)
    return (grid[code] * torch.sign(v) * scale).reshape(rows, -1)[:, :cols]


def _exact_unpack(packed, cols):
    codes, byte = packed
    nibbles = torch.stack((codes % 16, codes // 16), -1).reshape(codes.shape[0], -1).long()
    size = nibbles % 8
    power = torch.where(size < 2, 0, size // 2 - 1).double()                  # exponent and mantissa bits of a code
    value = torch.where(size < 2, size / 2, torch.exp2(power) * (1 + (size % 2) / 2)) * (1 - 2 * (nibbles // 8))
    scale = torch.exp2(byte.double() - 127).repeat_interleave(32, 1)
    return value[:, :cols] * scale[:, :cols]


def _exact_norm(v, weight, bias, layer):
    mean = v.mean(1, keepdim=True) if layer else 0 * v[:, :1]
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + EPS)
    hat = (v - mean) * rstd
    out = hat if weight is None else hat * weight.double()
    return out if bias is None else out + bias.double(), hat, mean, rstd


def _exact_norm_gradient(grad, v, mean, rstd, layer):
    """From the derivative of (v - mean) / sqrt(var + eps), sums written out."""
    d, n = v - mean, v.shape[1]
    back = rstd * grad - rstd ** 3 * d * (grad * d).sum(1, keepdim=True) / n
    return back - back.sum(1, keepdim=True) / n if layer else back


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    double = lambda name: None if s.get(name) is None else s[name].double()  # noqa: E731
    rand = s.get("rand")
    across = None if rand is None else rand.t()
    if c["op"] == "quantize":
        v = double("x")
        if c["source"] == "split":
            _, exponent = torch.frexp(v)                                      # |v| in [2^(e-1), 2^e): spacing 2^(e-8)
            v = v + double("rho") / 127 * torch.exp2(exponent.clamp(min=-125).double() - 9)
        r = {"rows": _exact_values(v, rand)}
        if c["both"]:
            r["columns"] = _exact_values(v.t(), across)
        return r
    if c["op"] == "linear":
        x = double("x")
        r = {"y": _exact_values(x) @ _exact_unpack(s["w"], c["k"]).t()}
        if c["train"]:
            r["xt"] = _exact_values(x.t())
        return r
    if c["op"] == "linear_backward":
        dy = double("dy")
        return {"dx": _exact_values(dy, rand) @ _exact_unpack(s["wt"], c["n"]).t(),
                "dw": _exact_values(dy.t(), across) @ _exact_unpack(s["xt"], c["m"]).t()}
    layer, post = c["kind"] == "layer", c["post"] == "norm"
    gate, f = double("gate"), double("f")
    slope = 1.0
    if gate is not None:
        gate = gate.reshape(-1, 1, c["cols"]).expand(-1, c["rows"] // gate.shape[0], -1).reshape(c["rows"], -1)
        if c["act"] == "sigmoid":
            gate = 1 / (1 + torch.exp(-gate))
            slope = gate - gate ** 2
    if c["op"] == "norm":
        h, y = double("x"), None
        zero = torch.zeros(c["rows"], 1, dtype=torch.float64, device="cuda")
        stats = [zero, zero, zero, zero]
        if f is not None:
            if post:
                f, _, stats[0], stats[1] = _exact_norm(f, s["post_weight"], s["post_bias"], layer)
            h = s["residual_scale"] * h + s["branch_scale"] * (f if gate is None else gate * f)
        if c["pre"]:
            y, _, stats[2], stats[3] = _exact_norm(h, s["pre_weight"], s["pre_bias"], layer)
        return {"h": None if f is None else h, "y": y, "stats": torch.cat(stats, 1).t()}
    names = ("dx", "df", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
    r, total, stats = dict.fromkeys(names), double("dh"), s["stats"].double()[:, :, None]
    if c["pre"]:
        dy, h = double("dy"), double("h")
        r["dpre_weight"] = (dy * (h - stats[2]) * stats[3]).sum(0)
        r["dpre_bias"] = dy.sum(0) if layer else None
        total = total + _exact_norm_gradient(dy * double("pre_weight"), h, stats[2], stats[3], layer)
    if f is None:
        return {**r, "dx": total}
    r["dx"] = s["residual_scale"] * total
    hat = (f - stats[0]) * stats[1] if post else f
    u = hat * double("post_weight") if post else hat
    u = u + double("post_bias") if post and layer else u
    du = s["branch_scale"] * total
    if gate is not None:
        r["dgate"] = (du * u * slope).reshape(s["gate"].shape[0], -1, c["cols"]).sum(1)
        du = du * gate
    if post:
        r["dpost_weight"] = (du * hat).sum(0)
        r["dpost_bias"] = du.sum(0) if layer else None
        du = _exact_norm_gradient(du * double("post_weight"), f, stats[0], stats[1], layer)
    r["df"] = du
    return r
