"""The 4-bit calls on the GPU at sizes that reach every way in which they are dispatched (mx4_sizes), against their definition in 64 bits: products of
the operands' values, in float64, and quantisation bit for bit.

Tolerances, as of the small sizes: a sum of k products in FP32 is off by at most k 2^-24 of the sum of their magnitudes (at most k additions, each
rounded once); BF16 results by 2^-8 of themselves, or half the spacing of its smallest numbers, in addition."""
import zlib

import numpy as np
import pytest
import torch

import mx4_reference as R
import mx4_sizes as S
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, FP32])


def generator(*key):
    return torch.Generator("cuda").manual_seed(zlib.crc32(repr(key).encode()))


def random_matrix(rows, cols, key, spread=8):
    """Every code, with scales around 1."""
    g = generator(rows, cols, key)
    q = fo.Mx4Tensor(rows, cols)
    blocks = -(-cols // 32)
    q.scales[:, :blocks] = torch.randint(127 - spread, 127 + spread, (rows, blocks), generator=g, device="cuda", dtype=torch.uint8)
    code = torch.zeros(rows, 2 * q.codes.shape[1], dtype=torch.uint8, device="cuda")
    code[:, :cols] = torch.randint(0, 16, (rows, cols), generator=g, device="cuda", dtype=torch.uint8)
    q.codes.copy_(code[:, 0::2] | code[:, 1::2] << 4)
    return q


def values(q):
    """What the codes and scales stand for, in float64."""
    code = torch.stack([q.codes & 15, q.codes >> 4], -1).view(q.rows, -1)[:, :q.cols]
    signed = torch.from_numpy(np.concatenate([R.GRID, -R.GRID])).cuda()
    scale = torch.from_numpy(np.append(np.exp2(np.arange(255.0) - 127), np.nan)).cuda()
    return signed[code.int()] * scale[q.scales[:, :-(-q.cols // 32)].int()].repeat_interleave(32, 1)[:, :q.cols]


def quantised(v, rand=None):
    """Q(v) in float64 of a float64 matrix, on the GPU, by the definition."""
    parts = [R.values(*R.quantize(v[i:i + 500], None if rand is None else rand[i:i + 500])) for i in range(0, v.shape[0], 500)]
    return torch.from_numpy(np.concatenate(parts)).cuda()


def check_product(out, a, b):
    k = a.shape[1]
    exact, size = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    bound = k * 2.0 ** -24 * size
    if out.dtype == BF16:
        bound = bound + 2.0 ** -8 * (exact.abs() + bound) + 2.0 ** -134
    off = (out.double() - exact).abs()
    assert bool((off <= bound).all()), float((off - bound).max())


def framed(m, n, dtype):
    """A matrix within a larger one, and the larger one."""
    whole = torch.full((m + 2, n + 5), 7.0, dtype=dtype, device="cuda")
    return whole, whole[1:-1, 2:2 + n]


def untouched(whole):
    return bool((whole[0] == 7).all() and (whole[-1] == 7).all() and (whole[:, :2] == 7).all() and (whole[:, -3:] == 7).all())


def scratch(n):
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")


def inputs(m, k, dtype, key):
    """Values of many sizes, with ties and zeros."""
    g = generator(m, k, key)
    x = torch.randn(m, k, generator=g, device="cuda") * torch.randint(-12, 13, (m, 1), generator=g, device="cuda").double().exp2().float()
    tie = torch.randint(0, 8, (m, k), generator=g, device="cuda") == 0
    x = torch.where(tie, torch.randint(-10, 11, (m, k), generator=g, device="cuda") / 4.0, x)
    return x.to(dtype)


@TYPES
@pytest.mark.parametrize("way,m,n,k", S.PRODUCTS)
def test_products(way, m, n, k, dtype):
    a, b = random_matrix(m, k, "a"), random_matrix(n, k, "b")
    whole, out = framed(m, n, dtype)
    fo.mx4_matmul(a, b, out, workspace=scratch(fo.mx4_matmul_workspace(m, n, k)))
    check_product(out, values(a), values(b))
    assert untouched(whole)
    again = torch.empty(m, n, dtype=dtype, device="cuda")
    fo.mx4_matmul(a, b, again)
    assert torch.equal(again, out)


@pytest.mark.parametrize("way,m,n,k", [p for p in S.PRODUCTS if not p[0].startswith("16")])
def test_a_block_that_is_not_finite_stays_in_its_row_and_column(way, m, n, k):
    a, b = random_matrix(m, k, "a"), random_matrix(n, k, "b")
    clean, out = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    fo.mx4_matmul(a, b, clean)
    rows, cols = sorted({0, m // 2, m - 1}), sorted({1, n // 3, n - 1})
    for i, row in enumerate(rows):
        a.scales[row, (i * 7) % -(-k // 32)] = 255
    for i, col in enumerate(cols):
        b.scales[col, -(-k // 32) - 1 - i % -(-k // 32)] = 255
    fo.mx4_matmul(a, b, out)
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[rows, :] = True
    bad[:, cols] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])


@TYPES
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("way,m,n,k", [("64", 300, 1200, 1301), ("128", 1001, 2304, 768), ("256", 3000, 4097, 1300)])
def test_linear_layers_in_training_and_for_prompts(way, m, n, k, keep, dtype):
    x, w = inputs(m, k, dtype, "x"), random_matrix(n, k, "w")
    xt = fo.Mx4Tensor(k, m) if keep else None
    whole, y = framed(m, n, dtype)
    fo.mx4_linear(x, w, y, xt=xt, workspace=scratch(fo.mx4_linear_workspace(m, n, k)))
    v = x.double().cpu().numpy()
    check_product(y, quantised(v), values(w))
    assert untouched(whole)
    if keep:
        codes, scales = R.pack(*R.quantize(v[:, :40].T))
        assert np.array_equal(xt.codes[:40].cpu().numpy(), codes) and np.array_equal(xt.scales[:40].cpu().numpy(), scales)


@TYPES
@pytest.mark.parametrize("random", [False, True])
@pytest.mark.parametrize("way,m,n,k", S.GRADIENTS)
def test_both_gradients_of_one_type(way, m, n, k, random, dtype):
    dy, wt, xt = inputs(m, n, BF16, "dy"), random_matrix(k, n, "wt"), random_matrix(k, m, "xt")
    rand = torch.randint(0, 256, (m, n), generator=generator("r"), device="cuda", dtype=torch.uint8) if random else None
    (whole_dx, dx), (whole_dw, dw) = framed(m, k, dtype), framed(n, k, dtype)
    ws = scratch(fo.mx4_linear_backward_workspace(m, n, k))
    fo.mx4_linear_backward(dy, wt, xt, dx, dw, rand=rand, workspace=ws)
    v, r = dy.double().cpu().numpy(), None if rand is None else rand.cpu().numpy()
    check_product(dx, quantised(v, r), values(wt))
    check_product(dw, quantised(np.ascontiguousarray(v.T), None if r is None else np.ascontiguousarray(r.T)), values(xt))
    assert untouched(whole_dx) and untouched(whole_dw)
    # each by itself is the same sums
    one = torch.empty(m, k, dtype=dtype, device="cuda")
    fo.mx4_linear_backward(dy, wt, None, one, None, rand=rand, workspace=ws)
    other = torch.empty(n, k, dtype=dtype, device="cuda")
    fo.mx4_linear_backward(dy, None, xt, None, other, rand=rand, workspace=ws)
    assert torch.equal(one, dx) and torch.equal(other, dw)


@TYPES
@pytest.mark.parametrize("out_dtype", [BF16, FP32])
@pytest.mark.parametrize("way,m,n,k", S.FEW)
def test_a_few_rows(way, m, n, k, dtype, out_dtype):
    x, w = inputs(m, k, dtype, "x"), random_matrix(n, k, "w")
    whole, y = framed(m, n, out_dtype)
    fo.mx4_linear(x, w, y)                         # (without a workspace: in one launch)
    check_product(y, quantised(x.double().cpu().numpy()), values(w))
    assert untouched(whole)
    # a row by itself is the same function of it: both are within the bound of the same exact sums, and here held to it
    if m > 1:
        token = torch.empty(1, n, dtype=out_dtype, device="cuda")
        fo.mx4_linear(x[m - 1:], w, token)
        check_product(token, quantised(x[m - 1:].double().cpu().numpy()), values(w))


def sources(source, rows, cols):
    """(matrix, corrections, float64 values of some rows or columns of it)"""
    if source == "fp32":
        x = inputs(rows, cols, FP32, source)
        return x, None, lambda i: x[i].double().cpu().numpy()
    x = inputs(rows, cols, BF16, source)
    if source == "bf16":
        return x, None, lambda i: x[i].double().cpu().numpy()
    rho = torch.randint(-127, 128, (rows, cols), generator=generator("rho"), device="cuda", dtype=torch.int8)
    bits = x.view(torch.int16)
    return x, rho, lambda i: R.master(bits[i].cpu().numpy().view(np.uint16), rho[i].cpu().numpy())


@pytest.mark.parametrize("random", [False, True])
@pytest.mark.parametrize("source", ["bf16", "fp32", "split"])
@pytest.mark.parametrize("way,rows,cols", S.QUANTISED)
def test_quantisation_both_ways(way, rows, cols, source, random):
    x, rho, exact = sources(source, rows, cols)
    rand = torch.randint(0, 256, (rows, cols), generator=generator("rand"), device="cuda", dtype=torch.uint8) if random else None
    q, qt, only_t = (fo.Mx4Tensor(*s) for s in ((rows, cols), (cols, rows), (cols, rows)))
    for t in (q, qt, only_t):
        t.codes.fill_(0xA5)
        t.scales.fill_(0x5A)
    fo.mx4_quantize(x, q, qt, rho=rho, rand=rand)
    fo.mx4_quantize(x, None, only_t, rho=rho, rand=rand)
    assert torch.equal(qt.codes, only_t.codes) and torch.equal(qt.scales, only_t.scales)
    # rows and columns at the ends of blocks, tiles and bands and in between, by the definition
    g = np.random.default_rng(zlib.crc32(repr((rows, cols)).encode()))

    def sample(n):
        ends = [i + d for unit in (32, 64, 128, 256, 1024) for i in (unit, n // unit * unit) for d in (-1, 0)]
        return sorted({i for i in [0, n - 1] + ends + g.integers(0, n, 24).tolist() if 0 <= i < n})

    for index, got, columns in ((sample(rows), q, False), (sample(cols), qt, True)):
        where = (slice(None), index) if columns else index
        v, r = exact(where), None if rand is None else rand[where].cpu().numpy()
        codes, scales = R.pack(*R.quantize(v.T if columns else v, r.T if columns and random else r))
        assert np.array_equal(got.codes[index].cpu().numpy(), codes) and np.array_equal(got.scales[index].cpu().numpy(), scales)
    # and all of it as the pieces of 512 rows, which the tests of small sizes hold to the definition
    for begin in range(0, rows, 512):
        end = min(begin + 512, rows)
        part = slice(begin, end)
        p, pt = fo.Mx4Tensor(end - begin, cols), fo.Mx4Tensor(cols, end - begin)
        cut = lambda t: None if t is None else t[part]        # noqa: E731
        fo.mx4_quantize(x[part], p, pt, rho=cut(rho), rand=cut(rand))
        assert torch.equal(q.codes[part], p.codes) and torch.equal(q.scales[part], p.scales)
        width, blocks = pt.codes.shape[1], -(-(end - begin) // 32)
        assert torch.equal(qt.codes[:, begin // 2:begin // 2 + width], pt.codes)
        assert torch.equal(qt.scales[:, begin // 32:begin // 32 + blocks], pt.scales[:, :blocks])


def test_only_the_given_stream_is_launched_on():
    # Captured on one stream and called on another, which is not captured: what goes to the given stream is in the graph and nothing of it has
    # run when the capture ends; the current stream, on which it would have run at once, has seen nothing.
    cases = [(1, 300, 1000), (65, 200, 700), (300, 500, 640)]
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for m, n, k in cases:
        x, w, wt = inputs(m, k, BF16, "x"), random_matrix(n, k, "w"), random_matrix(k, n, "wt")
        ws = scratch(max(fo.mx4_linear_workspace(m, n, k), fo.mx4_linear_backward_workspace(m, n, k)))
        q, xt = fo.Mx4Tensor(m, k), fo.Mx4Tensor(k, m)
        back, few, y, c = (torch.empty(m, s, device="cuda") for s in (k, n, n, n))
        dx, dw = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
        outs = (q.codes, q.scales, xt.codes, xt.scales, back, few, y, c, dx, dw)

        def calls(stream=None):
            fo.mx4_quantize(x, q, stream=stream)
            fo.mx4_dequantize(q, back, stream=stream)
            fo.mx4_linear(x, w, few, workspace=ws, stream=stream)
            fo.mx4_linear(x, w, y, xt=xt, workspace=ws, stream=stream)
            fo.mx4_matmul(q, w, c, stream=stream)
            fo.mx4_linear_backward(y, wt, xt, dx, dw, workspace=ws, stream=stream)

        calls()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(0x55 if t.dtype == torch.uint8 else 7)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            graph.capture_begin(capture_error_mode="relaxed")
        with torch.cuda.stream(other):
            calls(side)
        with torch.cuda.stream(side):
            graph.capture_end()
        torch.cuda.synchronize()
        assert all(bool((t == (0x55 if t.dtype == torch.uint8 else 7)).all()) for t in outs)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
