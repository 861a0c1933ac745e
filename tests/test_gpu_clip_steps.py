"""The steps that take a clipping factor, on the GPU.

Their gradients are BF16 values times the factor's scale, rounded to FP32.  So with a scale that is a power of two, where the product is a BF16 value again, they
are the steps without it on gradients scaled beforehand; and with any scale they are the algorithm in FP32 operations (made here by torch on the CPU, whose
sums, products and quotients are the IEEE ones; its FP32 root is not, and is made from the FP64 one, whose 53 bits are more than the 2 * 24 + 2 that make the second
rounding harmless) between the library's own codecs.  All comparisons are bit for bit."""
import gc
import zlib

import pytest
import torch

import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
KINDS = ["adamw", "adamw_exact", "sgd", "lion"]
# one tensor of each shape of launch, and lists; the last ones are as large as stores that go through to memory need
SIZES = {"one": [1], "odd": [4097], "middle": [5_000_003], "list": [1, 31, 32, 33, 4097, 0, 70_001], "large": [70_000_001],
         "large_list": [66_000_000, 7, 2_000_003]}
NAMES = ("param", "rho", "m_q", "m_scale", "v_q", "v_scale")


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()
    yield
    torch.cuda.empty_cache()


def gen(*key):
    return torch.Generator("cuda").manual_seed(zlib.crc32(repr(key).encode()))


def buffers(sizes, kind, seed=0):
    out = []
    for i, n in enumerate(sizes):
        g = gen(n, i, seed)
        b = fo.ParamBuffers(n, "adamw" if kind.startswith("adamw") else kind)
        if n:
            fo.split_weights(torch.randn(n, generator=g, device="cuda"), b.param, b.rho)
            b.grad.copy_(torch.randn(n, generator=g, device="cuda"))
        b.lr, b.weight_decay = 1e-2 * (1 + i % 3), 0.1
        out.append(b)
    return out


def step(kind, tensors, t=1, clip=None, stream=None):
    if kind == "adamw":
        fo.adamw_step(tensors, 0.9, 0.95, 1e-8, t, stream=stream, clip=clip)
    elif kind == "adamw_exact":
        fo.adamw_step_exact(tensors, 0.9, 0.95, 1e-8, t, stream=stream, clip=clip)
    elif kind == "sgd":
        fo.sgd_step(tensors, 0.9, stream=stream, clip=clip)
    else:
        fo.lion_step(tensors, 0.9, 0.99, stream=stream, clip=clip)


def same(a, b):
    for x, y in zip(a, b):
        for name in NAMES:
            p, q = getattr(x, name), getattr(y, name)
            assert p is None or torch.equal(p.view(torch.int16) if p.dtype == torch.float16 else p, q.view(torch.int16) if q.dtype == torch.float16 else q), name


def factor_of(scale):
    f = fo.ClipFactor()
    f.sum_squares.fill_(float("nan"))
    f.norm.fill_(float("nan"))
    f.scale.fill_(scale)
    return f


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes", SIZES)
def test_a_power_of_two_is_the_step_on_scaled_gradients(sizes, kind):
    a, b = buffers(SIZES[sizes], kind), buffers(SIZES[sizes], kind)
    ta, tb = fo.TensorList(a), fo.TensorList(b)
    for t, scale in ((1, 0.125), (2, 1.0), (200, 2.0 ** -20)):          # (from step 165 on the momentum's correction is 1)
        grads = [x.grad.clone() for x in a]
        for x, g in zip(b, grads):
            x.grad.copy_(g.float() * scale)
        step(kind, ta, t, clip=factor_of(scale))
        step(kind, tb, t)
        same(a, b)
        assert all(torch.equal(x.grad, g) for x, g in zip(a, grads))


def f32(x):
    return torch.tensor(x, dtype=FP32)


def state(b):
    """theta, m, v of a tensor in FP32 on the CPU."""
    n = b.numel
    theta, m, v = (torch.empty(n, device="cuda") for _ in range(3))
    fo.reconstruct_weights(b.param, b.rho, theta)
    fo.dequantize_momentum(b.m_q, b.m_scale, m)
    if b.v_q is not None:
        fo.dequantize_variance(b.v_q, b.v_scale, v)
    return theta.cpu(), m.cpu(), v.cpu()


def expected(kind, b, scale, t):
    theta, m, v = state(b)
    g = b.grad.float().cpu() * scale
    lr, wd = f32(b.lr), f32(b.weight_decay)
    out = fo.ParamBuffers(b.numel, b.kind)
    if kind == "adamw_exact":
        b1, b2, eps, one = f32(0.9), f32(0.95), f32(1e-8), f32(1.0)
        m = (b1 * m) + ((one - b1) * g)
        v = (b2 * v) + ((one - b2) * (g * g))
        r1, r2 = (one / f32(1.0 - float(x) ** t) for x in (b1, b2))
        theta = theta - (lr * (((m * r1) / (torch.sqrt((v * r2).double()).float() + eps)) + (wd * theta)))
    elif kind == "sgd":
        m = (f32(0.9) * m) + g
        theta = theta - (lr * (m + (wd * theta)))
    else:
        b1, b2, one = f32(0.9), f32(0.99), f32(1.0)
        u = torch.sign((b1 * m) + ((one - b1) * g))
        m = (b2 * m) + ((one - b2) * g)
        theta = theta - (lr * (u + (wd * theta)))
    fo.split_weights(theta.cuda(), out.param, out.rho)
    fo.quantize_momentum(m.cuda(), out.m_q, out.m_scale)
    if out.v_q is not None:
        fo.quantize_variance(v.cuda(), out.v_q, out.v_scale)
    return out


@pytest.mark.parametrize("kind", ["adamw_exact", "sgd", "lion"])
@pytest.mark.parametrize("sizes", [[4097], [33, 70_001, 32]])
def test_any_scale_is_the_algorithm_in_fp32(sizes, kind):
    bufs = buffers(sizes, kind)
    tensors = fo.TensorList(bufs)
    for t, scale in ((1, 0.3137), (2, 1e-3), (3, 0.99999)):
        f = factor_of(scale)
        want = [expected(kind, b, f.scale.cpu(), t) for b in bufs]
        step(kind, tensors, t, clip=f)
        same(bufs, want)
        for b in bufs:
            b.grad.mul_(1.5)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes", ["odd", "list", "large"])
def test_gradients_that_are_not_finite_leave_everything_as_it_is(sizes, kind):
    a = buffers(SIZES[sizes], kind)
    tensors = fo.TensorList(a)
    step(kind, tensors, 1)
    kept = [[getattr(x, n).clone() for n in NAMES if getattr(x, n) is not None] for x in a]
    good = a[0].grad.clone()
    a[0].grad[0] = float("inf")
    grads, f = fo.GradList.of(tensors), fo.ClipFactor()
    ws = torch.empty(fo.grad_norm_workspace(grads), dtype=torch.uint8, device="cuda")
    fo.grad_norm(grads, 1.0, f, workspace=ws)
    step(kind, tensors, 2, clip=f)
    for x, old in zip(a, kept):
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip([getattr(x, n) for n in NAMES if getattr(x, n) is not None], old))
    # and the next step is as if it had not been
    a[0].grad.copy_(good)
    b = buffers(SIZES[sizes], kind)
    tb = fo.TensorList(b)
    step(kind, tb, 1)
    fo.grad_norm(grads, 1.0, f, workspace=ws)
    step(kind, tensors, 2, clip=f)
    step(kind, tb, 2, clip=f)
    same(a, b)


@pytest.mark.parametrize("kind", KINDS)
def test_norm_and_step_replay_like_eager_calls(kind):
    a, b = buffers(SIZES["list"], kind), buffers(SIZES["list"], kind)
    ta, tb = fo.TensorList(a), fo.TensorList(b)
    fa, fb = fo.ClipFactor(), fo.ClipFactor()
    grads = [fo.GradList.of(t) for t in (ta, tb)]
    ws = [torch.empty(fo.grad_norm_workspace(g), dtype=torch.uint8, device="cuda") for g in grads]

    def both(tensors, g, f, w):
        fo.grad_norm(g, 0.5, f, workspace=w)
        step(kind, tensors, 3, clip=f)
    both(ta, grads[0], fa, ws[0])
    both(tb, grads[1], fb, ws[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(ta, grads[0], fa, ws[0])
    for replay in range(4):
        for x, y in zip(a, b):
            g = torch.randn(x.numel, generator=gen(x.numel, replay), device="cuda") * (1e-3 if replay == 2 else 1.0)
            x.grad.copy_(g)
            y.grad.copy_(g)
        if replay == 1:
            a[4].grad[5] = b[4].grad[5] = float("nan")
        fa.data.fill_(float("nan"))
        ws[0].fill_(0xFF)
        graph.replay()
        both(tb, grads[1], fb, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(fa.data.view(torch.int64), fb.data.view(torch.int64))
        same(a, b)


def test_on_another_stream_and_with_a_changed_rate():
    a, b = buffers(SIZES["list"], "sgd"), buffers(SIZES["list"], "sgd")
    ta, tb = fo.TensorList(a), fo.TensorList(b)
    side, f = torch.cuda.Stream(), factor_of(0.25)
    torch.cuda.synchronize()
    for lr in (0.5, 0.25):
        for i in range(len(a)):
            ta.set_hyper(i, lr=lr)
            tb.set_hyper(i, lr=lr)
        for x in b:
            x.grad.mul_(0.25)
        torch.cuda.synchronize()
        step("sgd", ta, clip=f, stream=side)
        step("sgd", tb)
        torch.cuda.synchronize()
        same(a, b)
        for x in b:
            x.grad.mul_(4.0)


def test_it_saves_the_clipping_its_rounding_only():
    # clipped in place the gradients are rounded to BF16 once more: half a step of 2^-8 apart at most, and with them SGD's first momentum
    a, b = buffers([4096], "sgd"), buffers([4096], "sgd")
    f = factor_of(0.3)
    fo.clip_gradients(fo.GradList.of(fo.TensorList(b)), f)
    exact = a[0].grad.float() * f.scale
    assert float(((b[0].grad.float() - exact).abs() / exact.abs().clamp(min=1e-30)).max()) <= 2.0 ** -8
