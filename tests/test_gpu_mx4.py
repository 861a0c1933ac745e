"""Microscaled 4-bit matrices on the GPU: quantisation bit for bit against its definition in 64 bits, products within the bound of
their FP32 sums, refusals, streams and graphs."""
import zlib

import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 31), (3, 32), (33, 33), (1, 256), (5, 255), (2, 257), (129, 127), (128, 128), (127, 513), (64, 1000), (300, 96),
         (257, 768), (513, 1025)]


def rng(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def hard_values(g, rows, cols):
    """FP32 values over the whole range: blocks of every size, zeros, ties on the grid, subnormals, the largest."""
    v = g.standard_normal((rows, cols)) * np.exp2(g.integers(-140, 120, (rows, 1)).astype(float))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.5])
    some = g.random((rows, cols)) < 0.3
    v = np.where(some, g.choice(ties, (rows, cols)) * g.choice([-1, 1], (rows, cols)) * np.exp2(g.integers(-130, 120, (rows, 1)).astype(float)), v)
    v[g.random((rows, cols)) < 0.1] = 0.0
    v[g.random(rows) < 0.1] = 0.0
    v = np.clip(v, -3e38, 3e38).astype(np.float32)
    return v


def make_source(source, rows, cols, seed=0):
    """(GPU tensor, rho, float64 values)"""
    g = rng(source, rows, cols, seed)
    v = hard_values(g, rows, cols)
    if source == "fp32":
        return torch.from_numpy(v).cuda(), None, v.astype(float)
    t = torch.from_numpy(v).bfloat16()
    if source == "bf16":
        return t.cuda(), None, t.double().numpy()
    rho = g.integers(-127, 128, (rows, cols)).astype(np.int8)
    bits = t.view(torch.int16).numpy().view(np.uint16)
    return t.cuda(), torch.from_numpy(rho).cuda(), R.master(bits, rho)


def same(q, v, rand=None):
    codes, scales = R.pack(*R.quantize(v, rand))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)


def dirty(rows, cols):
    """A matrix whose arrays hold something else before the call."""
    q = fo.Mx4Tensor(rows, cols)
    q.codes.fill_(0xA5)
    q.scales.fill_(0x5A)
    return q


@pytest.mark.parametrize("source", ["bf16", "fp32", "split"])
@pytest.mark.parametrize("random", [False, True])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize_is_the_definition_bit_for_bit(source, random, rows, cols):
    x, rho, v = make_source(source, rows, cols)
    rand = rng("rand", rows, cols).integers(0, 256, (rows, cols)).astype(np.uint8) if random else None
    rand_gpu = torch.from_numpy(rand).cuda() if random else None
    rand_t = rand.T if random else None
    only, both, both_t, only_t = dirty(rows, cols), dirty(rows, cols), dirty(cols, rows), dirty(cols, rows)
    fo.mx4_quantize(x, only, rho=rho, rand=rand_gpu)
    fo.mx4_quantize(x, both, both_t, rho=rho, rand=rand_gpu)
    fo.mx4_quantize(x, None, only_t, rho=rho, rand=rand_gpu)
    same(only, v, rand)
    same(both, v, rand)
    same(both_t, v.T, rand_t)
    same(only_t, v.T, rand_t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("random", [False, True])
def test_quantize_marks_blocks_that_are_not_finite(dtype, random):
    g = rng("nan", random)
    x = torch.from_numpy(g.standard_normal((70, 200)).astype(np.float32)).to(dtype)
    for row, col, bad in ((0, 0, np.inf), (3, 199, np.nan), (33, 40, -np.inf), (69, 64, np.nan)):
        x[row, col] = bad
    rand = g.integers(0, 256, (70, 200)).astype(np.uint8) if random else None
    q, qt = dirty(70, 200), dirty(200, 70)
    fo.mx4_quantize(x.cuda(), q, qt, rand=None if rand is None else torch.from_numpy(rand).cuda())
    same(q, x.double().numpy(), rand)
    same(qt, x.double().numpy().T, None if rand is None else rand.T)
    out = torch.empty(70, 200, device="cuda")
    fo.mx4_dequantize(q, out)
    assert np.array_equal(np.isnan(out.cpu().numpy()), np.isnan(R.unpack(q.codes.cpu().numpy(), q.scales.cpu().numpy(), 200)))


@pytest.mark.parametrize("offset", [1, 3, 8])
def test_quantize_takes_rows_that_lie_apart_and_begin_anywhere(offset):
    rows, cols = 45, 300
    whole = torch.from_numpy(hard_values(rng("stride"), rows, 2 * cols)).cuda().bfloat16()
    x = whole[:, offset:offset + cols]
    q, qt = dirty(rows, cols), dirty(cols, rows)
    fo.mx4_quantize(x, q, qt)
    same(q, x.double().cpu().numpy())
    same(qt, x.double().cpu().numpy().T)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dequantize_is_exact_for_every_code_and_scale(rows, cols, dtype):
    g = rng("codes", rows, cols)
    code, byte = g.integers(0, 16, (rows, cols)).astype(np.uint8), g.integers(0, 253, (rows, -(-cols // 32))).astype(np.uint8)
    byte[g.random(byte.shape) < 0.2] = 0
    byte[g.random(byte.shape) < 0.1] = 1
    codes, scales = R.pack(code, byte)
    q = fo.Mx4Tensor(rows, cols, buffers=(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()))
    whole = torch.full((rows, cols + 5), 7.0, dtype=dtype, device="cuda")
    fo.mx4_dequantize(q, whole[:, 2:2 + cols])
    got = whole.cpu().double().numpy()
    assert np.array_equal(got[:, 2:2 + cols], R.values(code, byte))
    assert (got[:, :2] == 7).all() and (got[:, 2 + cols:] == 7).all()


# A sum of k products in FP32 is off by at most k 2^-24 of the sum of their magnitudes (each of at most k additions rounds once);
# BF16 results by 2^-8 of themselves, or half the spacing of its smallest numbers, in addition.
def check_product(out, a, b):
    k = a.shape[1]
    exact, size = a @ b.T, np.abs(a) @ np.abs(b).T
    bound = k * 2.0 ** -24 * size
    if out.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(exact) + bound) + 2.0 ** -134
    assert (np.abs(out.cpu().double().numpy() - exact) <= bound).all()


def random_matrix(rows, cols, key, spread=8):
    g = rng("matrix", rows, cols, key)
    code = g.integers(0, 16, (rows, cols)).astype(np.uint8)
    byte = g.integers(127 - spread, 127 + spread, (rows, -(-cols // 32))).astype(np.uint8)
    codes, scales = R.pack(code, byte)
    return fo.Mx4Tensor(rows, cols, buffers=(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())), R.values(code, byte)


def scratch(n):
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")


PRODUCTS = [(1, 1, 1), (1, 17, 33), (2, 64, 256), (16, 16, 255), (17, 130, 257), (5, 300, 1024), (64, 64, 64), (100, 77, 513), (128, 256, 768),
            (33, 1000, 2304), (200, 129, 4097), (257, 385, 1281), (512, 640, 96), (1, 2049, 4096), (300, 2200, 640), (700, 1100, 512)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul(m, n, k, dtype):
    a, av = random_matrix(m, k, "a")
    b, bv = random_matrix(n, k, "b")
    ws = scratch(fo.mx4_matmul_workspace(m, n, k))
    out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    fo.mx4_matmul(a, b, out, workspace=ws)
    check_product(out, av, bv)
    again = torch.full((m, n + 3), 7.0, dtype=dtype, device="cuda")
    fo.mx4_matmul(a, b, again[:, 1:1 + n], workspace=ws)
    assert torch.equal(again[:, 1:1 + n], out)
    assert (again[:, 0] == 7).all() and (again[:, 1 + n:] == 7).all()


@pytest.mark.parametrize("m", [1, 40, 300])
def test_matmul_carries_blocks_that_are_not_finite(m):
    a, av = random_matrix(m, 300, "a")
    b, bv = random_matrix(70, 300, "b")
    b.scales[5, 3] = 255
    out = torch.zeros(m, 70, device="cuda")
    fo.mx4_matmul(a, b, out, workspace=scratch(fo.mx4_matmul_workspace(m, 70, 300)))
    got = out.cpu().numpy()
    assert np.isnan(got[:, 5]).all() and np.isfinite(np.delete(got, 5, 1)).all()


def test_products_over_nothing_are_zero_and_of_nothing_do_nothing():
    out = torch.full((5, 7), float("nan"), device="cuda")
    fo.mx4_matmul(fo.Mx4Tensor(5, 0), fo.Mx4Tensor(7, 0), out)
    assert (out == 0).all()
    fo.mx4_matmul(fo.Mx4Tensor(0, 64), fo.Mx4Tensor(7, 64), torch.empty(0, 7, device="cuda"))
    fo.mx4_quantize(torch.empty(0, 64, device="cuda"), fo.Mx4Tensor(0, 64))
    w, _ = random_matrix(7, 64, "w")
    fo.mx4_linear(torch.empty(0, 64, device="cuda"), w, torch.empty(0, 7, device="cuda"), workspace=scratch(fo.mx4_linear_workspace(0, 7, 64)))
    dw = torch.full((7, 64), float("nan"), device="cuda")
    wt, _ = random_matrix(64, 7, "wt")
    fo.mx4_linear_backward(torch.empty(0, 7, device="cuda"), wt, fo.Mx4Tensor(64, 0), torch.empty(0, 64, device="cuda"), dw,
                           workspace=scratch(fo.mx4_linear_backward_workspace(0, 7, 64)))
    assert (dw == 0).all()


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("keep", [False, True])
def test_linear_is_quantise_and_product(m, n, k, dtype, keep):
    x = torch.from_numpy(hard_values(rng("x", m, k), m, k).clip(-1e4, 1e4)).cuda().to(dtype)
    w, wv = random_matrix(n, k, "w")
    xt = dirty(k, m) if keep else None
    out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    fo.mx4_linear(x, w, out, xt=xt, workspace=scratch(fo.mx4_linear_workspace(m, n, k)))
    v = x.double().cpu().numpy()
    check_product(out, R.values(*R.quantize(v)), wv)
    if keep:
        same(xt, v.T)


@pytest.mark.parametrize("m", [1, 3, 16])
def test_linear_of_few_rows_that_lie_apart(m):
    k, n = 1000, 333
    whole = torch.randn(m, 2 * k, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    w, wv = random_matrix(n, k, "w")
    x = whole[:, 3:3 + k]
    x[0, 64:96] = float("nan")
    out = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    fo.mx4_linear(x, w, out, workspace=scratch(fo.mx4_linear_workspace(m, n, k)))
    assert out[0].isnan().all()
    if m > 1:
        check_product(out[1:], R.values(*R.quantize(x[1:].double().cpu().numpy())), wv)


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("random", [False, True])
def test_linear_backward(m, n, k, random):
    dy = (torch.from_numpy(rng("dy", m, n).standard_normal((m, n)).astype(np.float32)) * 1e-4).bfloat16()
    dy[torch.from_numpy(rng("rows", m).random(m) < 0.2)] = 0
    rand = rng("r", m, n).integers(0, 256, (m, n)).astype(np.uint8) if random else None
    wt, wtv = random_matrix(k, n, "wt")
    xt, xtv = random_matrix(k, m, "xt")
    dx, dw = torch.empty(m, k, dtype=torch.bfloat16, device="cuda"), torch.empty(n, k, device="cuda")
    ws = scratch(fo.mx4_linear_backward_workspace(m, n, k))
    gpu_rand = torch.from_numpy(rand).cuda() if random else None
    fo.mx4_linear_backward(dy.cuda(), wt, xt, dx, dw, rand=gpu_rand, workspace=ws)
    v = dy.double().numpy()
    check_product(dx, R.values(*R.quantize(v, rand)), wtv)
    check_product(dw, R.values(*R.quantize(v.T, rand.T if random else None)), xtv)
    for one in (dict(wt=wt, xt=None, dx=torch.empty_like(dx), dw=None), dict(wt=None, xt=xt, dx=None, dw=torch.empty_like(dw))):
        fo.mx4_linear_backward(dy.cuda(), rand=gpu_rand, workspace=ws, **one)
        assert torch.equal(one["dx"], dx) if one["dw"] is None else torch.equal(one["dw"], dw)


def representable(rows, cols, key):
    """Values that are their own 4-bit form along rows and along columns: small multiples of 1/2 with a 4 in every block of either."""
    g = rng("rep", rows, cols, key)
    v = g.choice([-3.0, -1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0], (rows, cols))
    v[::16, :] = 4.0
    v[:, ::16] = 4.0
    return v


def test_linear_gradients_against_differences():
    # the forward call is linear in what its operands stand for, so between two points that are exactly representable the difference of
    # sum(dy y) is the gradient times the step: exactly, but for the rounding of the sums, all of whose terms are multiples of 1/8 below 2^24 / 8
    m, n, k = 96, 64, 128
    dy, x0, x1, w0, w1 = representable(m, n, "dy"), representable(m, k, 0), representable(m, k, 1), representable(n, k, 2), representable(n, k, 3)
    gpu = lambda v: torch.from_numpy(v).cuda().float()           # noqa: E731
    ws = scratch(max(fo.mx4_linear_workspace(m, n, k), fo.mx4_linear_backward_workspace(m, n, k)))

    def quantised(v):
        q, qt = fo.Mx4Tensor(*v.shape), fo.Mx4Tensor(v.shape[1], v.shape[0])
        fo.mx4_quantize(gpu(v), q, qt)
        return q, qt

    def loss(x, w):
        y = torch.empty(m, n, device="cuda")
        xt = fo.Mx4Tensor(k, m)
        fo.mx4_linear(gpu(x), quantised(w)[0], y, xt=xt, workspace=ws)
        return (y.double().cpu().numpy() * dy).sum(), xt

    dx, dw = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    base, xt = loss(x0, w0)
    fo.mx4_linear_backward(gpu(dy), quantised(w0)[1], xt, dx, dw, workspace=ws)
    assert loss(x1, w0)[0] - base == (dx.double().cpu().numpy() * (x1 - x0)).sum()
    assert loss(x0, w1)[0] - base == (dw.double().cpu().numpy() * (w1 - w0)).sum()


def test_calls_on_another_stream_wait_for_nothing_else_and_agree():
    m, n, k = 65, 200, 700
    x = torch.randn(m, k, device="cuda").bfloat16()
    w, _ = random_matrix(n, k, "w")
    ws = scratch(fo.mx4_linear_workspace(m, n, k))
    want, got = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    fo.mx4_linear(x, w, want, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fo.mx4_linear(x, w, got, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("m", [1, 50, 600])
def test_replays_of_a_captured_graph_follow_their_inputs(m):
    n, k = 300, 640
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    w, _ = random_matrix(n, k, "w")
    wt, _ = random_matrix(k, n, "wt")
    xt, y, dx, dw = fo.Mx4Tensor(k, m), torch.empty(m, n, device="cuda"), torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    ws = scratch(max(fo.mx4_linear_workspace(m, n, k), fo.mx4_linear_backward_workspace(m, n, k)))

    def calls():
        fo.mx4_linear(x, w, y, xt=xt, workspace=ws)
        fo.mx4_linear_backward(y, wt, xt, dx, dw, workspace=ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        x.copy_(torch.randn(m, k, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        got = [t.clone() for t in (y, dx, dw, xt.codes, xt.scales)]
        torch.cuda.synchronize()
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw, xt.codes, xt.scales)))


def test_refusals():
    x = torch.zeros(40, 64, device="cuda", dtype=torch.bfloat16)
    q, w, y = fo.Mx4Tensor(40, 64), fo.Mx4Tensor(48, 64), torch.empty(40, 48, device="cuda")
    ws = scratch(fo.mx4_linear_workspace(40, 48, 64))
    status = lambda call, *a, **k: pytest.raises(fo.FlashOptimError, call, *a, **k).value.status        # noqa: E731
    assert status(fo.mx4_quantize, x) == -1
    assert status(fo.mx4_quantize, x, fo.Mx4Tensor(40, 65)) == -1
    assert status(fo.mx4_quantize, x, None, fo.Mx4Tensor(40, 64)) == -1
    assert status(fo.mx4_quantize, x.float(), q, rho=torch.zeros(40, 64, device="cuda", dtype=torch.int8)) == -1
    assert status(fo.mx4_dequantize, q, torch.empty(40, 63, device="cuda")) == -1
    assert status(fo.mx4_matmul, q, fo.Mx4Tensor(48, 65), y) == -1
    assert status(fo.mx4_matmul, q, w, torch.empty(48, 40, device="cuda")) == -1
    assert status(fo.mx4_linear, x[:, :63], w, y, workspace=ws) == -1
    assert status(fo.mx4_linear, x, w, y) == -1
    assert status(fo.mx4_linear, x, w, y, workspace=ws[:16]) == -8
    assert status(fo.mx4_linear, x, w, y, xt=fo.Mx4Tensor(40, 64), workspace=ws) == -1
    assert status(fo.mx4_linear_backward, x, None, None, None, None, workspace=ws) == -1
    assert status(fo.mx4_linear_workspace, 1 << 31, 1, 1) == -3
    assert status(fo.mx4_matmul_workspace, -1, 1, 1) == -1
    odd = fo.Mx4Tensor(40, 64, buffers=(scratch(40 * 128 + 1)[1:40 * 128 + 1].view(40, 128), q.scales))
    assert status(fo.mx4_quantize, x, odd) == -2
    for call in (lambda: fo.mx4_quantize(x.half(), q), lambda: fo.mx4_quantize(x.t(), q), lambda: fo.mx4_quantize(x[0], q),
                 lambda: fo.mx4_quantize(x.cpu(), q), lambda: fo.mx4_quantize(x, fo.Mx4Tensor(40, 64, device="cpu")),
                 lambda: fo.mx4_quantize(x, q, rand=torch.zeros(40, 63, device="cuda", dtype=torch.uint8)),
                 lambda: fo.Mx4Tensor(40, 64, buffers=(q.codes, q.scales[:, :8]))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("m,n,k", [(1, 48, 64), (1, 4096, 4096), (16, 300, 1000)])
def test_a_few_rows_take_no_workspace(m, n, k):
    x = torch.randn(m, k, device="cuda", generator=torch.Generator("cuda").manual_seed(m)).bfloat16()
    w, wv = random_matrix(n, k, "w")
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    fo.mx4_linear(x, w, out)
    check_product(out, R.values(*R.quantize(x.double().cpu().numpy())), wv)
    status = lambda **kw: pytest.raises(fo.FlashOptimError, fo.mx4_linear, x, w, out, **kw).value.status        # noqa: E731
    assert status(xt=fo.Mx4Tensor(k, m)) == -1              # Q(x) of the training form goes through memory
    assert status(xt=fo.Mx4Tensor(k, m), workspace=scratch(16)) == -8
