"""The norms between two blocks and their gradients on the GPU, against their definition in 64 bits.

Tolerances.  With u = 2^-24: a sum over a row runs through fewer than 64 additions on any path (16 in a lane, 6 across the
wavefront, up to 16 wavefronts), so it is off by at most 64 u of the sum of magnitudes, and the few operations around it add a
few u each: C = 128 covers a norm with its scale, bias and gate.  Errors of h go on into y.  A sum over rows adds u for
every row.  BF16 results are off by 2^-8 of themselves in addition."""
import zlib

import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

U, C = 2.0 ** -24, 128
BF16, FP32 = torch.bfloat16, torch.float32
COLS = [1, 7, 8, 64, 500, 512, 513, 1000, 1024, 1025, 2048, 2100, 4096, 4100, 8192, 8200, 16384]


def rng(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def make(g, shape, dtype, scale=1.0, shift=0.0):
    return torch.from_numpy((g.standard_normal(shape) * scale + shift).astype(np.float32)).to(dtype).cuda()


def f64(t):
    return None if t is None else t.double().cpu().numpy()


class Case:
    def __init__(self, rows, cols, kind="rms", post_norm=True, branch=True, gates=1, act="linear", pre=True, stream=BF16, dtype=BF16,
                 params=BF16, seed=0, loud=0.3):
        g = rng(rows, cols, kind, post_norm, gates, act, seed)
        layer = kind == "layer"
        self.rows, self.cols, self.kind, self.act, self.post_norm, self.pre = rows, cols, kind, act, post_norm and branch, pre
        self.stream, self.dtype, self.params = stream, dtype, params
        self.x = make(g, (rows, cols), stream, 2.0, loud)
        self.f = make(g, (rows, cols), dtype, 1.5, -loud) if branch else None
        self.gate = make(g, (gates, cols), dtype) if gates and branch else None
        p = lambda there, shift: make(g, (cols,), params, 0.3, shift) if there else None        # noqa: E731
        self.w = dict(post_weight=p(self.post_norm, 1.0), post_bias=p(self.post_norm and layer, 0.0), pre_weight=p(pre, 1.0),
                      pre_bias=p(pre and layer, 0.0))
        self.dy = make(g, (rows, cols), dtype, 0.1) if pre else None
        self.dh = make(g, (rows, cols), stream, 0.1)
        self.a, self.c, self.eps = 0.75, 1.25, 1e-5
        self.spec = fo.BlockNorm(cols, kind=kind, eps=self.eps, post_norm=self.post_norm, gate_act=act, residual_scale=self.a,
                                 branch_scale=self.c, **self.w)

    def reference(self):
        w = {n: f64(t) for n, t in self.w.items()}
        return R.norm_forward(f64(self.x), f64(self.f), f64(self.gate), self.kind, self.act, self.post_norm, self.a, self.c,
                              float(np.float32(self.eps)), w["post_weight"], w["post_bias"], w["pre_weight"], w["pre_bias"], self.pre)

    def run(self, stream=None):
        self.h = torch.full_like(self.x, 7) if self.f is not None else None
        self.y = torch.full((self.rows, self.cols), 7, dtype=self.dtype, device="cuda") if self.pre else None
        self.stats = torch.full((4, self.rows), 7.0, device="cuda")
        fo.block_norm(self.spec, self.x, f=self.f, gate=self.gate, h=self.h, y=self.y, stats=self.stats, stream=stream)
        return self

    def norm_error(self, v, mean, rstd, w, b, err):
        """Bounds of the error of (v - mean) rstd w + b, of the mean and of rstd, for values v known to within err."""
        size = lambda t, other: other if t is None else np.abs(t)        # noqa: E731
        m_err = C * U * np.abs(v).mean(1, keepdims=True) + err.mean(1, keepdims=True)
        if self.kind == "rms":
            m_err = 0 * m_err
        r_err = rstd * (C * U + rstd * (np.sqrt((err ** 2).mean(1, keepdims=True)) + m_err))
        hat = np.abs(v - mean) * rstd
        e = size(w, 1.0) * (rstd * (err + m_err + 4 * U * (np.abs(v) + np.abs(mean))) + hat * (r_err / rstd) + C * U * hat) + C * U * size(b, 0.0)
        return e, m_err[:, 0], r_err[:, 0]

    def check_forward(self):
        h, y, stats = self.reference()
        w = {n: f64(t) for n, t in self.w.items()}
        err = np.zeros_like(h)
        got = f64(self.stats)
        if self.f is not None:
            f = f64(self.f)
            u_err, u = 0 * f, f
            if self.post_norm:
                mean, rstd = stats[0][:, None], stats[1][:, None]
                u_err, m_err, r_err = self.norm_error(f, mean, rstd, w["post_weight"], w["post_bias"], 0 * f)
                u = (f - mean) * rstd * (1 if w["post_weight"] is None else w["post_weight"])
                u = u + (0 if w["post_bias"] is None else w["post_bias"])
                assert (np.abs(got[0] - stats[0]) <= m_err).all() and (np.abs(got[1] - stats[1]) <= r_err).all()
            g = 1.0 if self.gate is None else np.abs(R.act_of(R.spread(f64(self.gate), self.rows), self.act))
            err = abs(self.c) * g * (u_err + C * U * np.abs(u)) + 4 * U * np.abs(self.a * f64(self.x))
            self.close(self.h, h, err)
        if not self.post_norm:
            assert (got[:2] == 0).all()
        if self.pre:
            y_err, m_err, r_err = self.norm_error(h, stats[2][:, None], stats[3][:, None], w["pre_weight"], w["pre_bias"], err)
            self.close(self.y, y, y_err)
            assert (np.abs(got[2] - stats[2]) <= m_err).all() and (np.abs(got[3] - stats[3]) <= r_err).all()
        else:
            assert (got[2:] == 0).all()

    @staticmethod
    def close(got, want, err):
        if got.dtype == BF16:
            err = err + 2.0 ** -8 * (np.abs(want) + err)
        off = np.abs(f64(got) - want)
        assert (off <= err).all(), (off - err).max()

    def backward(self, workspace=None, stream=None):
        like = lambda t: None if t is None else torch.full_like(t, 7)        # noqa: E731
        self.grads = dict(dx=like(self.x), df=like(self.f), dgate=like(self.gate), **{"d" + n: like(t) for n, t in self.w.items()})
        if workspace is None:
            size = fo.block_norm_backward_workspace(self.spec, self.rows, 1 if self.gate is None else self.gate.shape[0])
            workspace = torch.full((max(size, 4),), 0xFF, dtype=torch.uint8, device="cuda")
        fo.block_norm_backward(self.spec, self.x if self.h is None else self.h, self.stats, f=self.f, gate=self.gate, dy=self.dy, dh=self.dh,
                               workspace=workspace, stream=stream, **self.grads)
        return self

    def check_backward(self):
        w = {n: f64(t) for n, t in self.w.items()}
        args = (f64(self.x if self.h is None else self.h), f64(self.stats), f64(self.f), f64(self.gate), f64(self.dy), f64(self.dh), self.kind,
                self.act, self.post_norm, self.a, self.c, w["post_weight"], w["post_bias"], w["pre_weight"])
        want, size = R.norm_backward(*args), R.norm_backward(*args, size=True)
        for name, got in self.grads.items():
            if got is not None:
                depth = 4 * C + (0 if name in ("dx", "df") else self.rows)
                self.close(got, want[name], depth * U * size[name])


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("stream,dtype", [(BF16, BF16), (FP32, BF16), (FP32, FP32)])
def test_every_width(cols, kind, stream, dtype):
    for rows in (1, 5, 18):
        c = Case(rows, cols, kind, gates=1, act="sigmoid", stream=stream, dtype=dtype, params=dtype)
        c.run().check_forward()
        c.backward().check_backward()


@pytest.mark.parametrize("cols", [96, 700, 3000])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("branch,post_norm,pre", [(False, False, True), (True, False, True), (True, True, True), (True, True, False),
                                                  (True, False, False)])
@pytest.mark.parametrize("gates", [0, 1, 2, 12, 60])
@pytest.mark.parametrize("act", ["linear", "sigmoid"])
def test_every_form(cols, kind, branch, post_norm, pre, gates, act):
    if not branch and gates:
        pytest.skip("a gate is the branch's")
    c = Case(60, cols, kind, post_norm, branch, gates, act, pre, params=FP32)
    c.run().check_forward()
    c.backward().check_backward()


@pytest.mark.parametrize("rows,gates", [(3000, 1), (3000, 3), (3000, 300), (3000, 1500), (3000, 3000), (2049, 683)])
@pytest.mark.parametrize("cols", [40, 1100])
def test_many_rows_and_every_way_to_share_a_gate(rows, gates, cols):
    c = Case(rows, cols, "layer", gates=gates, act="sigmoid")
    c.run().check_forward()
    c.backward().check_backward()


@pytest.mark.parametrize("branch,pre", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("rows,gates", [(1, 1), (2, 1), (3, 3), (9, 3), (257, 1), (1030, 2), (1030, 103), (4095, 1), (4097, 1)])
def test_rows_that_do_not_fill_a_workgroup(rows, gates, branch, pre):
    for cols, kind in ((300, "layer"), (768, "layer"), (1024, "rms")):
        c = Case(rows, cols, kind, branch=branch, gates=gates, pre=pre)
        c.run().check_forward()
        c.backward().check_backward()


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_that_are_zero_or_constant(kind):
    c = Case(12, 777, kind)
    c.x[3] = 0
    c.f[3] = 0
    c.f[5] = 3.0
    c.x[6:8] = 0
    c.run().check_forward()
    c.backward().check_backward()
    assert all(torch.isfinite(t).all() for t in (c.h, c.y, c.stats))


def test_what_is_not_finite_stays_in_its_row():
    c = Case(9, 600, "layer", gates=9)
    c.x[2, 5], c.f[7, 100] = float("nan"), float("inf")
    c.run()
    bad = torch.tensor([2, 7], device="cuda")
    good = torch.tensor([0, 1, 3, 4, 5, 6, 8], device="cuda")
    assert torch.isfinite(c.y[good]).all() and torch.isfinite(c.h[good]).all() and not torch.isfinite(c.y[bad]).any()
    c.backward()
    assert torch.isfinite(c.grads["dx"][good]).all() and torch.isfinite(c.grads["df"][good]).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("cols", [100, 1500])
def test_rows_that_lie_apart_and_buffers_used_again(kind, cols):
    c = Case(21, cols, kind, gates=7)
    c.run().backward()
    want = [c.h, c.y, c.stats] + [c.grads[n] for n in ("dx", "df", "dgate")]

    def apart(t, offset=3):
        whole = torch.full((t.shape[0], t.shape[1] + 11), 5, dtype=t.dtype, device="cuda")
        whole[:, offset:offset + t.shape[1]] = t
        return whole, whole[:, offset:offset + t.shape[1]]

    (wx, x), (wf, f), (_, gate) = apart(c.x), apart(c.f), apart(c.gate, 1)
    stats = torch.empty_like(c.stats)
    fo.block_norm(c.spec, x, f=f, gate=gate, h=x, y=f, stats=stats)             # h over x, y over f
    assert torch.equal(x, want[0]) and torch.equal(f, want[1]) and torch.equal(stats, want[2])
    for whole in (wx, wf):
        assert (whole[:, :3] == 5).all() and (whole[:, 3 + cols:] == 5).all()
    (_, f), (_, dy), (_, dh), (wg, dgate) = apart(c.f), apart(c.dy), apart(c.dh), apart(torch.zeros_like(c.gate), 1)
    ws = torch.empty(fo.block_norm_backward_workspace(c.spec, c.rows, 7), dtype=torch.uint8, device="cuda")
    fo.block_norm_backward(c.spec, x, stats, f=f, gate=gate, dy=dy, dh=dh, dx=dh, df=dy, dgate=dgate, workspace=ws)      # dx over dh, df over dy
    assert torch.equal(dh, want[3]) and torch.equal(dy, want[4]) and torch.equal(dgate, want[5])
    assert (wg[:, :1] == 5).all() and (wg[:, 1 + cols:] == 5).all()


@pytest.mark.parametrize("stream", [BF16, torch.float32])
@pytest.mark.parametrize("cols", [768, 8000, 8192, 12008, 16000])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_over_what_they_were_made_from(kind, cols, stream):
    c = Case(300, cols, kind, gates=3, stream=stream)          # (several rows to a workgroup)
    c.run().backward()
    want = [c.grads[n] for n in ("dx", "df", "dgate", "dpre_weight")]
    ws = torch.empty(fo.block_norm_backward_workspace(c.spec, c.rows, 3), dtype=torch.uint8, device="cuda")
    for over in ("f", "dy"):
        dh, f, dy, dgate, dpre = c.dh.clone(), c.f.clone(), c.dy.clone(), torch.empty_like(c.gate), torch.empty_like(want[3])
        df = f if over == "f" else dy
        fo.block_norm_backward(c.spec, c.h, c.stats, f=f, gate=c.gate, dy=dy, dh=dh, dx=dh, df=df, dgate=dgate, dpre_weight=dpre, workspace=ws)
        assert all(torch.equal(x, y) for x, y in zip((dh, df, dgate, dpre), want)), over


def test_gradients_that_are_not_wanted_change_nothing():
    c = Case(50, 900, "layer", gates=5)
    c.run().backward()
    ws = torch.empty(fo.block_norm_backward_workspace(c.spec, 50, 5), dtype=torch.uint8, device="cuda")
    for name, want in c.grads.items():
        got = torch.full_like(want, 7)
        fo.block_norm_backward(c.spec, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dh=c.dh, workspace=ws, **{name: got})
        assert torch.equal(got, want), name
    # no gradient from elsewhere is a gradient of zero
    zero, none = torch.empty_like(c.x), torch.empty_like(c.x)
    fo.block_norm_backward(c.spec, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dh=torch.zeros_like(c.dh), dx=zero, workspace=ws)
    fo.block_norm_backward(c.spec, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dx=none, workspace=ws)
    assert torch.equal(zero, none)


def test_no_rows():
    c = Case(6, 64, "layer", gates=2)
    c.run()
    empty = lambda dtype: torch.empty(0, 64, dtype=dtype, device="cuda")        # noqa: E731
    fo.block_norm(c.spec, empty(BF16), f=empty(BF16), gate=c.gate, h=empty(BF16), y=empty(BF16))
    sums = {"d" + n: torch.full_like(t, 7) for n, t in c.w.items()}
    dgate = torch.full_like(c.gate, 7)
    fo.block_norm_backward(c.spec, empty(BF16), torch.empty(4, 0, device="cuda"), f=empty(BF16), gate=c.gate, dy=empty(BF16), dx=empty(BF16),
                           dgate=dgate, **sums)
    assert all((t == 0).all() for t in sums.values()) and (dgate == 0).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("act", ["linear", "sigmoid"])
def test_gradients_against_differences(kind, act):
    # Differences of the GPU's own forward call, all in FP32, along a random direction.  They are off by the difference's own
    # truncation, which the 64-bit definition has alike, and by the forward call's rounding (at most 8 C u of the sum of magnitudes in
    # either of two calls) over the step.
    def case():
        return Case(6, 90, kind, gates=3, act=act, stream=FP32, dtype=FP32, params=FP32)

    step = 2.0 ** -6
    base = case().run().backward()
    dy, dh = f64(base.dy), f64(base.dh)

    def loss(c):
        c.run()
        gpu = (f64(c.y) * dy).sum() + (f64(c.h) * dh).sum()
        h, y, _ = c.reference()
        return gpu, (y * dy).sum() + (h * dh).sum(), (np.abs(y * dy)).sum() + (np.abs(h * dh)).sum()

    named = dict(x="dx", f="df", gate="dgate", post_weight="dpost_weight", post_bias="dpost_bias", pre_weight="dpre_weight", pre_bias="dpre_bias")
    for name, grad in named.items():
        if base.grads[grad] is None:
            continue
        c = case()
        t = getattr(c, name) if hasattr(c, name) else c.w[name]
        start = t.clone()
        d = torch.from_numpy(rng(name, kind).choice([-1.0, 1.0], tuple(t.shape))).float().cuda()
        t.copy_(start + step * d)
        up, up_exact, size = loss(c)
        moved = f64(t)
        t.copy_(start - step * d)
        down, down_exact, _ = loss(c)
        moved = moved - f64(t)
        slope = (f64(base.grads[grad]) * moved).sum()
        w = {n: f64(v) for n, v in base.w.items()}
        h, _, stats = base.reference()
        exact = R.norm_backward(h, stats, f64(base.f), f64(base.gate), dy, dh, kind, act, True, base.a, base.c, w["post_weight"],
                                w["post_bias"], w["pre_weight"])[grad]
        truncation = abs(up_exact - down_exact - (exact * moved).sum())
        rounding = 2 * 8 * C * U * size
        assert abs((up - down) - slope) <= 2 * truncation + rounding + 8 * C * U * (np.abs(exact) * np.abs(moved)).sum(), name


def test_another_stream_and_replays_of_a_captured_graph():
    c = Case(300, 2000, "layer", gates=3, act="sigmoid")
    ws = torch.empty(fo.block_norm_backward_workspace(c.spec, 300, 3), dtype=torch.uint8, device="cuda")
    c.run().backward(workspace=ws)
    want = [t.clone() for t in (c.h, c.y, c.stats, *c.grads.values())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.run().backward(workspace=ws)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (c.h, c.y, c.stats, *c.grads.values())))

    def calls():
        fo.block_norm(c.spec, c.x, f=c.f, gate=c.gate, h=c.h, y=c.y, stats=c.stats)
        fo.block_norm_backward(c.spec, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dh=c.dh, workspace=ws, **c.grads)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        c.f.copy_(make(rng("replay", i), (300, 2000), BF16))
        graph.replay()
        got = [t.clone() for t in (c.h, c.y, c.stats, *c.grads.values())]
        torch.cuda.synchronize()
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, (c.h, c.y, c.stats, *c.grads.values())))


def test_gradients_of_saturated_gates():
    # Beside the same call with linear gates, which leaves c dH u, the sigmoid's slope is a factor s(g) s(-g) for each value: relative to
    # it, the exponent g log2(e) (two roundings) makes an error of 2 |g| u, and exponential, reciprocals, sums and products, each within an
    # ulp (2 u), less than 16 u.
    rows, cols = 61, 300
    c = Case(rows, cols, "rms", gates=rows, act="sigmoid", stream=FP32, dtype=FP32, params=FP32)
    g = np.linspace(-60, 60, rows * cols).reshape(rows, cols).astype(np.float32)
    c.gate.copy_(torch.from_numpy(g))
    c.run().backward()
    linear = fo.BlockNorm(cols, kind="rms", eps=c.eps, post_norm=True, gate_act="linear", residual_scale=c.a, branch_scale=c.c, **c.w)
    without = torch.empty_like(c.gate)
    ws = torch.empty(fo.block_norm_backward_workspace(linear, rows, rows), dtype=torch.uint8, device="cuda")
    fo.block_norm_backward(linear, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dh=c.dh, dgate=without, workspace=ws)
    g = g.astype(np.float64)
    want = f64(without) / (1 + np.exp(-g)) / (1 + np.exp(g))
    off = np.abs(f64(c.grads["dgate"]) - want)
    assert (off <= (2 * np.abs(g) + 16) * U * np.abs(want)).all(), np.nanmax(off / np.abs(want)) / U


def test_only_the_given_stream_is_launched_on():
    # Captured on one stream and called on another, which is not captured: what goes to the given stream is in the graph and nothing of it has
    # run when the capture ends; the current stream, on which it would have run at once, has seen nothing.
    c = Case(300, 2000, "layer", gates=3, act="sigmoid")
    ws = torch.empty(fo.block_norm_backward_workspace(c.spec, 300, 3), dtype=torch.uint8, device="cuda")
    c.run().backward(workspace=ws)
    outs = (c.h, c.y, c.stats, *c.grads.values())
    want = [t.clone() for t in outs]
    for t in outs:
        t.fill_(7)
    torch.cuda.synchronize()
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin(capture_error_mode="relaxed")
    with torch.cuda.stream(other):
        fo.block_norm(c.spec, c.x, f=c.f, gate=c.gate, h=c.h, y=c.y, stats=c.stats, stream=side)
        fo.block_norm_backward(c.spec, c.h, c.stats, f=c.f, gate=c.gate, dy=c.dy, dh=c.dh, workspace=ws, stream=side, **c.grads)
    with torch.cuda.stream(side):
        graph.capture_end()
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in outs)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
