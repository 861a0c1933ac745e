"""The 64-bit definitions that the GPU tests of the 4-bit matrices and block norms compare with: pinned to hand-computed values and,
for gradients, to differences.  Host checks of the library's sizes and refusals that need no GPU."""
import ctypes as C

import numpy as np
import pytest

import mx4_reference as R
import paper_2602_23349_amd as fo
from paper_2602_23349_amd import binding as B


def test_quantisation_of_a_block_by_hand():
    v = np.zeros((1, 64))
    v[0, :8] = [7.9, -5.0, 2.5, 0.25, 0.75, -0.2, 1.75, 3.5]       # largest 7.9: scale 1
    v[0, 32:36] = [12.0, 10.0, 1.0, -0.5]                         # largest 12: scale 2
    code, byte = R.quantize(v)
    assert byte.tolist() == [[127, 128]]
    assert R.GRID[code[0, :8] & 7].tolist() == [6.0, 4.0, 2.0, 0.0, 1.0, 0.0, 2.0, 4.0]
    assert (code[0, :8] >> 3).tolist() == [0, 1, 0, 0, 0, 1, 0, 0]
    assert R.values(code, byte)[0, 32:36].tolist() == [12.0, 8.0, 1.0, -0.0]
    rand = np.zeros((1, 64), np.uint8)
    code, byte = R.quantize(v, rand)                              # 7.9 > 6: scale 2 for the first block; 12 = 6 * 2 stays
    assert byte.tolist() == [[128, 128]]
    assert R.values(code, byte)[0, :3].tolist() == [8.0, -6.0, 3.0]
    code, byte = R.quantize(v, rand + 255)
    assert R.values(code, byte)[0, :3].tolist() == [6.0, -4.0, 2.0]


def test_stochastic_rounding_is_unbiased_over_the_random_bytes():
    # over all 256 bytes a value between a and b goes to b k times of 256, k the nearest integer to its share: half a byte's weight off
    t = np.linspace(0, 6, 97)
    v = np.zeros((256, 128))
    v[:, :97] = t
    v[:, 97:] = 6.0
    v[:, ::32] = 6.0
    rand = np.arange(256, dtype=np.uint8)[:, None].repeat(128, 1)
    mean = R.values(*R.quantize(v, rand)).mean(0)
    assert (np.abs(mean - v[0]) <= 2.0 / 512).all()


def test_packing_is_undone():
    g = np.random.default_rng(0)
    for rows, cols in ((1, 1), (3, 33), (2, 257), (4, 512), (5, 700)):
        code, byte = g.integers(0, 16, (rows, cols)).astype(np.uint8), g.integers(0, 255, (rows, -(-cols // 32))).astype(np.uint8)
        codes, scales = R.pack(code, byte)
        assert codes.shape == (rows, 128 * -(-cols // 256)) and scales.shape == (rows, 16 * -(-cols // 512))
        assert np.array_equal(R.unpack(codes, scales, cols), R.values(code, byte))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("act", ["linear", "sigmoid"])
@pytest.mark.parametrize("post_norm,gates,pre,branch", [(False, 0, True, False), (False, 0, True, True), (True, 0, True, True), (True, 1, True, True),
                                                        (True, 3, True, True), (True, 6, False, True), (False, 2, True, True)])
def test_gradient_formulas_against_differences(kind, act, post_norm, gates, pre, branch):
    g = np.random.default_rng(1)
    rows, n = 6, 10
    p = dict(x=g.standard_normal((rows, n)))
    if branch:
        p["f"] = g.standard_normal((rows, n))
    if gates:
        p["gate"] = g.standard_normal((gates, n))
    for name, there in (("pw", post_norm), ("pb", post_norm and kind == "layer"), ("w", pre), ("b", pre and kind == "layer")):
        if there:
            p[name] = g.standard_normal(n)
    fixed = dict(kind=kind, act=act, post_norm=post_norm, a=0.7, c=1.3)
    dy, dh = g.standard_normal((rows, n)) if pre else None, g.standard_normal((rows, n))

    def loss(**q):
        h, y, _ = R.norm_forward(**q, **fixed, pre=pre)
        return (h * dh).sum() + ((y * dy).sum() if pre else 0.0)

    h, _, stats = R.norm_forward(**p, **fixed, pre=pre)
    r = R.norm_backward(h, stats, f=p.get("f"), gate=p.get("gate"), dy=dy, dh=dh, pw=p.get("pw"), pb=p.get("pb"), w=p.get("w"), **fixed)
    names = dict(x="dx", f="df", gate="dgate", pw="dpost_weight", pb="dpost_bias", w="dpre_weight", b="dpre_bias")
    eps = 1e-5
    for name, v in p.items():
        for i in np.ndindex(*v.shape):
            up, down = v.copy(), v.copy()
            up[i] += eps
            down[i] -= eps
            slope = (loss(**{**p, name: up}) - loss(**{**p, name: down})) / (2 * eps)
            assert abs(slope - r[names[name]][i]) < 1e-7 * (1 + abs(slope)), (name, i)


def test_workspace_sizes():
    assert fo.mx4_linear_workspace(0, 10, 10) >= 0
    # what is quantised on the way fits: codes and scales of x, of dy and of its transpose
    assert fo.mx4_linear_workspace(100, 50, 300) >= 100 * (256 + 16)
    assert fo.mx4_linear_backward_workspace(100, 50, 300) >= 100 * (128 + 16) + 50 * (128 + 16)
    for bad in ((-1, 1, 1), (1, 1 << 31, 1)):
        for call in (fo.mx4_matmul_workspace, fo.mx4_linear_workspace, fo.mx4_linear_backward_workspace):
            with pytest.raises(fo.FlashOptimError):
                call(*bad)
    # enormous sizes are refused or sized without overflow
    most = (1 << 31) - 1
    for sizes in ((most, most, most), (most, 1, 1), (1, most, 1), (1, 1, most)):
        try:
            assert fo.mx4_linear_backward_workspace(*sizes) >= 0
        except fo.FlashOptimError as e:
            assert e.status == -3


def test_block_norm_refusals_before_anything_runs():
    L = fo.load_library()
    status = lambda **k: L.flashoptim_block_norm_backward_workspace(spec(**k), 8, 2)        # noqa: E731

    def spec(**k):
        s = B._BlockNormSpec(cols=64, eps=1e-5, residual_scale=1, branch_scale=1)
        for name, v in k.items():
            setattr(s, name, v)
        return s

    assert status() > 0
    assert status(cols=0) == -1 and status(cols=16385) == -3
    assert status(kind=2) == -1 and status(gate_act=-1) == -1 and status(param_dtype=2) == -1 and status(eps=float("nan")) == -1
    assert status(pre_bias=64) == -1                                                       # RMS norms have no bias
    assert status(kind=1, pre_bias=64) > 0
    assert status(pre_weight=65) == -2
    assert L.flashoptim_block_norm_backward_workspace(spec(), 9, 2) == -1
    assert L.flashoptim_block_norm_backward_workspace(spec(), 1 << 31, 1) == -3
    m = lambda rows, cols, dtype=0, data=4096, stride=None: B._Matrix(data, rows, cols, cols if stride is None else stride, dtype)       # noqa: E731
    x, f32 = m(8, 64), m(8, 64, 1)
    call = L.flashoptim_block_norm
    assert call(spec(), x, None, None, None, None, None, None) == -1                        # nothing to do
    assert call(spec(), x, x, None, None, x, None, None) == -1                              # a branch without h
    assert call(spec(), x, None, x, None, x, None, None) == -1                              # a gate without a branch
    assert call(spec(), x, f32, None, x, None, None, None) == -1                            # a branch wider than the stream
    assert call(spec(), x, x, m(3, 64), x, x, None, None) == -1                             # 3 does not divide 8
    assert call(spec(), m(8, 63), None, None, None, x, None, None) == -1
    assert call(spec(), m(8, 64, data=4097), None, None, None, x, None, None) == -2
    assert call(spec(), m(8, 64, stride=63), None, None, None, x, None, None) == -1
    assert call(spec(), m(8, 64, data=None), None, None, None, x, None, None) == -1
    for cols, rows in ((64, 1 << 26), (1024, 1 << 25), (2048, 1 << 24), (16384, 1 << 23)):  # more lanes than a launch has
        assert call(spec(cols=cols), m(rows, cols), None, None, None, m(rows, cols), None, None) == -3
    back = L.flashoptim_block_norm_backward
    grads = lambda **k: B._BlockNormGrads(**{n: C.pointer(v) if isinstance(v, B._Matrix) else v for n, v in k.items()})     # noqa: E731
    assert back(spec(), x, None, None, 4096, grads(dx=x), 4096, 1 << 30, None) == -1        # no gradient comes in
    assert back(spec(), x, None, None, None, grads(dy=x, dx=x), 4096, 1 << 30, None) == -1  # no statistics
    assert back(spec(), x, None, None, 4096, grads(dy=x, dx=x), 4096, 8, None) == -8
    assert back(spec(), x, None, None, 4096, grads(dy=x, dx=x), None, 0, None) == -1
    assert back(spec(), x, None, None, 4096, grads(dy=x, df=x), 4096, 1 << 30, None) == -1  # df without a branch
    assert back(spec(), x, x, None, 4096, grads(dy=x, dpost_weight=4096), 4096, 1 << 30, None) == -1    # no norm behind
    assert back(spec(), x, None, None, 4096, grads(dy=x, dpre_bias=4096), 4096, 1 << 30, None) == -1    # RMS
