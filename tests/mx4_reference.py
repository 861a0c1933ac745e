"""Microscaled 4-bit matrices and block norms from their definitions, in 64 bits on the CPU (test infrastructure)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(v, rand=None):
    """(codes 0..15 [rows, cols], scale bytes [rows, blocks]) of a float64 matrix that holds FP32 values."""
    rows, cols = v.shape
    blocks = -(-cols // 32)
    pad = np.zeros((rows, blocks * 32))
    pad[:, :cols] = v
    pad = pad.reshape(rows, blocks, 32)
    r = np.zeros((rows, blocks * 32))
    if rand is not None:
        r[:, :cols] = rand
    r = r.reshape(pad.shape)
    bad = ~np.isfinite(pad).all(-1)
    safe = np.where(bad[..., None], 0.0, pad)
    largest = np.abs(safe).max(-1)
    m, e = np.frexp(largest)                       # largest = m 2^e, 1/2 <= m < 1; the FP32 exponent field is e + 126
    field = np.where(largest == 0, 0, np.maximum(e + 126, 0))
    byte = field - 2
    if rand is not None:
        byte = byte + ((m > 0.75) & (field > 0))   # (a subnormal's mantissa field means something else, but its byte is 0)
    byte = np.maximum(byte, 0)
    t = np.abs(safe) / np.exp2(byte.astype(float) - 127)[..., None]
    if rand is None:
        far = np.abs(t[..., None] - GRID)          # the nearest; of two as near the even one
        best = far.min(-1, keepdims=True)
        near = far == best
        even = near & (np.arange(8) % 2 == 0)
        code = np.where(even.any(-1) & (near.sum(-1) > 1), even.argmax(-1), near.argmax(-1))
    else:
        low = np.searchsorted(GRID, t, side="right") - 1
        high = np.minimum(low + 1, 7)
        code = np.where(256 * (t - GRID[low]) > (r + 0.5) * (GRID[high] - GRID[low]), high, low)
    code = code + 8 * np.signbit(safe)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(rows, -1)[:, :cols].astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def pack(code, byte):
    """The arrays as the library lays them out, zeros behind the end of a row."""
    rows, cols = code.shape
    wide = np.zeros((rows, 256 * -(-cols // 256)), np.uint8)
    wide[:, :cols] = code
    scales = np.zeros((rows, 16 * -(-cols // 512)), np.uint8)
    scales[:, :byte.shape[1]] = byte
    return wide[:, 0::2] | wide[:, 1::2] << 4, scales


def unpack(codes, scales, cols):
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)[:, :cols]
    return values(code, scales)


def values(code, byte):
    rows, cols = code.shape
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(float) - 127)).repeat(32, 1)[:, :cols]
    return GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * scale


def master(param_bits, rho):
    """FP32 weights (as float64) of BF16 bit patterns and INT8 corrections, from Eq. 2, rounded once to FP32."""
    base = (param_bits.astype(np.uint32) << 16).view(np.float32).astype(float)
    e = np.maximum((param_bits >> 7) & 255, 1).astype(float)
    q = (rho.astype(np.float32) / np.float32(127)).astype(float)
    step = np.float32(q * np.exp2(e - 135)).astype(float)
    return (base.astype(np.float32) + step.astype(np.float32)).astype(float)


# ---------------------------------------------------------------------------------------------------- block norms --

def moments(v, layer, eps):
    mean = v.mean(1, keepdims=True) if layer else np.zeros((v.shape[0], 1))
    return mean, 1 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)


def act_of(gate, act):
    return 1 / (1 + np.exp(-gate)) if act == "sigmoid" else gate


def spread(gate, rows):
    return gate.repeat(rows // gate.shape[0], 0)


def norm_forward(x, f=None, gate=None, kind="rms", act="linear", post_norm=False, a=1.0, c=1.0, eps=1e-5, pw=None, pb=None, w=None, b=None,
                 pre=True):
    """(h, y, stats) with stats [4, rows]."""
    layer, rows = kind == "layer", x.shape[0]
    one = lambda t, other: other if t is None else t        # noqa: E731
    stats = np.zeros((4, rows))
    h = x
    if f is not None:
        u = f
        if post_norm:
            m, r = moments(f, layer, eps)
            stats[0], stats[1] = m[:, 0], r[:, 0]
            u = (f - m) * r * one(pw, 1.0) + one(pb, 0.0)
        h = a * x + c * u * (1.0 if gate is None else act_of(spread(gate, rows), act))
    y = None
    if pre:
        m, r = moments(h, layer, eps)
        stats[2], stats[3] = m[:, 0], r[:, 0]
        y = (h - m) * r * one(w, 1.0) + one(b, 0.0)
    return h, y, stats


def norm_backward(h, stats, f=None, gate=None, dy=None, dh=None, kind="rms", act="linear", post_norm=False, a=1.0, c=1.0, pw=None, pb=None,
                  w=None, size=False):
    """The gradients, and with `size` instead the same sums of magnitudes, which rounding errors are relative to."""
    layer, (rows, n) = kind == "layer", h.shape
    one = lambda t, other: other if t is None else mag(t)        # noqa: E731
    mag = np.abs if size else (lambda t: t)                      # noqa: E731
    sign = 1.0 if size else -1.0
    s = stats[:, :, None]
    centred = lambda v, m: np.abs(v) + np.abs(m) if size else v - m      # noqa: E731
    r = {}

    def through(g, hat, rstd):
        t = g + sign * hat * (g * hat).mean(1, keepdims=True)
        if layer:
            t = t + sign * g.mean(1, keepdims=True)
        return rstd * t

    total = np.zeros_like(h) if dh is None else mag(dh)
    if dy is not None:
        hat = centred(h, s[2]) * s[3]
        g = mag(dy)
        r["dpre_weight"], r["dpre_bias"] = (g * hat).sum(0), g.sum(0)
        total = total + through(g * one(w, 1.0), hat, s[3])
    r["dx"] = (abs(a) if size else a) * total if f is not None else total
    if f is None:
        return r
    hat = centred(f, s[0]) * s[1] if post_norm else mag(f)
    u = hat * one(pw, 1.0) + one(pb, 0.0) if post_norm else hat
    du = (abs(c) if size else c) * total
    if gate is not None:
        g = act_of(spread(gate, rows), act)
        slope = g * (1 - g) if act == "sigmoid" else 1.0
        r["dgate"] = (du * u * slope).reshape(gate.shape[0], -1, n).sum(1)
        du = du * mag(g)
    if post_norm:
        r["dpost_weight"], r["dpost_bias"] = (du * hat).sum(0), du.sum(0)
        du = through(du * one(pw, 1.0), hat, s[1])
    r["df"] = du
    return r
