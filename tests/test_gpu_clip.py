"""The global norm of a list of gradients and their clipping on the GPU, against their definitions in 64 bits.

The sum of squares is FP64 (2^-53 for each of at most 2^24 additions here, of positive values: 2^-29 of itself at the very most), so norm and scale are
off by their rounding to FP32, 2^-24 of themselves, and what that 2^-29 makes of it.  A clipped gradient is the product with the FP32 scale,
rounded to FP32 and, for BF16, once more: held to the same two roundings bit for bit."""
import gc
import math
import zlib

import pytest
import torch

import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TILE = 8192
SIZES = {
    "one": [1], "eight": [8], "odd": [1, 7, 0, 9, 255, 1000, 4097], "tile": [TILE - 1, TILE, TILE + 1, 2 * TILE], "empty": [0, 0, 5, 0],
    "none": [], "many": [(i * 37) % 5000 for i in range(300)], "lots": [3] * 700, "large": [5_000_003, 17, 40 * TILE],
}


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()


def gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def make(sizes, dtype, scale=1.0, seed=0):
    """Tensors that lie 16-byte aligned in one array, with 77 between them."""
    g = gen(str(sizes)[:50], seed)
    first, end = [], 0
    for n in sizes:
        first.append(end)
        end += n + 8 + -n % 8
    flat = torch.full((end + 8,), 77.0, dtype=dtype, device="cuda")
    views = [flat[f:f + n] for f, n in zip(first, sizes)]
    for v in views:
        v.copy_(torch.randn(v.numel(), generator=g, device="cuda") * scale)
    return flat, views


def norm_of(grads, max_norm, factor=None):
    factor = factor or fo.ClipFactor()
    factor.data.fill_(float("nan"))
    size = fo.grad_norm_workspace(grads)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None
    fo.grad_norm(grads, max_norm, factor, workspace=ws)
    return factor


def expected(views, max_norm):
    total = math.fsum(float(v.double().square().sum()) for v in views)
    norm = math.sqrt(total)
    limit = float(torch.tensor(max_norm, dtype=FP32))
    return total, norm, limit / norm if norm > limit else 1.0


def check_norm(factor, views, max_norm):
    total, norm, scale = expected(views, max_norm)
    assert abs(float(factor.sum_squares) - total) <= 2.0 ** -28 * total
    for got, want in ((factor.norm, norm), (factor.scale, scale)):
        assert abs(float(got) - want) <= (2.0 ** -24 + 2.0 ** -28) * abs(want)


def times(v, scale, dtype):
    return (v.float() * scale).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("sizes", SIZES)
def test_norm_and_clipping(sizes, dtype):
    for max_norm in (0.0, 0.5, 1e9, float("inf")):
        flat, views = make(SIZES[sizes], dtype)
        before = flat.clone()
        factor = norm_of(fo.GradList(views), max_norm)
        check_norm(factor, views, max_norm)
        assert torch.equal(flat, before)
        scale = factor.scale.clone()
        # into other tensors, of the same type and (FP32) as BF16
        for to in {dtype, BF16}:
            other, out = make(SIZES[sizes], to, seed=1)
            rest = other.clone()
            fo.clip_gradients(fo.GradList(views, out), factor)
            for v, o in zip(views, out):
                assert torch.equal(o, times(v, scale, to))
                o.fill_(0)
            at = 0
            for n in SIZES[sizes]:
                rest[at:at + n] = 0
                at += n + 8 + -n % 8
            assert torch.equal(other, rest)                   # nothing between the tensors
        # in place
        want = [times(v, scale, dtype) for v in views]
        fo.clip_gradients(fo.GradList(views), factor)
        assert all(torch.equal(a, b) for a, b in zip(views, want))


@pytest.mark.parametrize("count", [2, 15, 16, 17, 62, 63, 64, 65, 176, 177, 280, 281])
def test_numbers_of_tensors(count):
    # tensors of one tile and of several, whole and not, where a launch's table has one more or less
    sizes = [(TILE, 1, 2 * TILE + 9, 0, 4095, 3 * TILE)[i % 6] for i in range(count)]
    for dtype in (BF16, FP32):
        _, views = make(sizes, dtype)
        _, out = make(sizes, BF16, seed=1)
        factor = norm_of(fo.GradList(views, out), 0.5)
        check_norm(factor, views, 0.5)
        fo.clip_gradients(fo.GradList(views, out), factor)
        assert all(torch.equal(o, times(v, factor.scale, BF16)) for v, o in zip(views, out))


@pytest.mark.parametrize("tiles", [1, 3, 4, 5, 11, 12, 13, 16, 17])
def test_numbers_of_tiles(tiles):
    for dtype in (BF16, FP32):
        for sizes in ([tiles * TILE], [(tiles - 1) * TILE + 1], [TILE - 5] * tiles):
            _, views = make(sizes, dtype)
            check_norm(norm_of(fo.GradList(views), 1.0), views, 1.0)


def test_some_in_place_and_some_not():
    for max_norm in (0.5, 1e9):
        _, views = make([100, 9000, 31], BF16)
        _, out = make([100, 9000, 31], BF16, seed=1)
        factor = norm_of(fo.GradList(views), max_norm)
        want = [times(v, factor.scale, BF16) for v in views]
        fo.clip_gradients(fo.GradList(views, [views[0], out[1], views[2]]), factor)
        assert torch.equal(views[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(views[2], want[2])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_the_largest_and_smallest_values(dtype):
    top = torch.finfo(dtype).max
    big = torch.full((70_000,), top, dtype=dtype, device="cuda")
    factor = norm_of(fo.GradList([big]), 2.0)
    want = top * math.sqrt(70_000)
    assert abs(float(factor.sum_squares) - want ** 2) <= 1e-9 * want ** 2
    assert float(factor.norm) == float("inf")                 # (beyond FP32)
    assert abs(float(factor.scale) - 2.0 / want) <= 2.0 ** -149 + 1e-6 * 2.0 / want
    small = torch.full((100,), 2.0 ** -133 if dtype == BF16 else 2.0 ** -149, dtype=dtype, device="cuda")
    factor = norm_of(fo.GradList([small]), 2.0)
    assert abs(float(factor.sum_squares) - 100 * float(small[0]) ** 2) <= 1e-12 * 100 * float(small[0]) ** 2 and float(factor.scale) == 1.0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_gradient_that_is_not_finite(dtype, bad):
    for at in (0, 8191, 20_000):
        _, views = make([5, 20_001, 9], dtype)
        views[1][at] = bad
        factor = norm_of(fo.GradList(views), 1.0)
        assert not math.isfinite(float(factor.norm)) and math.isnan(float(factor.scale))
        fo.clip_gradients(fo.GradList(views), factor)
        assert all(bool(torch.isnan(v).all()) for v in views)


def test_sums_of_several_lists():
    _, a = make([5000, 3], BF16)
    _, b = make([70_000], FP32, seed=1)
    fa, fb = norm_of(fo.GradList(a), 1.0), norm_of(fo.GradList(b), 1.0)
    fa.sum_squares.add_(fb.sum_squares)
    fo.clip_factor_from_sum(fa, 1.5)
    check_norm(fa, a + b, 1.5)


def test_the_gradients_of_a_list_of_parameters():
    bufs = [fo.ParamBuffers(n, "sgd") for n in (1000, 0, 5, 30_000)]
    for i, b in enumerate(bufs):
        b.grad.copy_(torch.randn(b.numel, generator=gen(i), device="cuda"))
    grads = fo.GradList.of(fo.TensorList(bufs))
    factor = norm_of(grads, 1.0)
    check_norm(factor, [b.grad for b in bufs], 1.0)
    want = [times(b.grad, factor.scale, BF16) for b in bufs]
    fo.clip_gradients(grads, factor)
    assert all(torch.equal(b.grad, w) for b, w in zip(bufs, want))


def test_same_bits_every_time_and_on_any_stream():
    _, views = make(SIZES["large"] + SIZES["many"], BF16)
    grads = fo.GradList(views)
    first = norm_of(grads, 1.0).data.clone()
    ws = torch.empty(fo.grad_norm_workspace(grads), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    factor = fo.ClipFactor()
    torch.cuda.synchronize()
    for stream in (side, None, side):
        fo.grad_norm(grads, 1.0, factor, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(factor.data.view(torch.int64), first.view(torch.int64))


def test_captured_calls_replay_like_eager_calls():
    sizes = [4097, 1, 30_000] + [50] * 300
    flat, views = make(sizes, FP32)
    out = [torch.empty(n, dtype=BF16, device="cuda") for n in sizes]
    want = [torch.empty(n, dtype=BF16, device="cuda") for n in sizes]
    grads, other = fo.GradList(views, out), fo.GradList(views, want)
    factor, eager = fo.ClipFactor(), fo.ClipFactor()
    ws = [torch.empty(fo.grad_norm_workspace(grads), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(g, f, w):
        fo.grad_norm(g, 1.0, f, workspace=w)
        fo.clip_gradients(g, f)
    step(grads, factor, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(grads, factor, ws[0])
    for replay in range(4):
        flat.mul_(0.7 if replay % 2 else 1e-4 if replay else 1.0)
        factor.data.fill_(float("nan"))
        ws[0].fill_(0xFF)
        for o in out:
            o.fill_(7.0)
        graph.replay()
        step(other, eager, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(factor.data.view(torch.int64), eager.data.view(torch.int64))
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_tensor_of_more_than_2_to_32_bytes():
    n = (1 << 31) + 12_345
    x = torch.zeros(n, dtype=BF16, device="cuda")
    at = torch.tensor([0, 1 << 30, (1 << 31) - 1, n - 1], device="cuda")
    x[at] = torch.tensor([3.0, 4.0, 12.0, 84.0], dtype=BF16, device="cuda")
    grads = fo.GradList([x])
    factor = norm_of(grads, 8.5)
    assert float(factor.sum_squares) == 85.0 ** 2 and float(factor.norm) == 85.0
    fo.clip_gradients(grads, factor)
    assert torch.equal(x[at].float(), (torch.tensor([3.0, 4.0, 12.0, 84.0]).cuda() * factor.scale).to(BF16).float())
    assert int(torch.count_nonzero(x)) == 4
