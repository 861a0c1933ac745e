"""What the calls on logits and on lists of gradients refuse, and how a list is cut into launches, without a GPU: every refusal comes before
any device work, so that the pointers below are never dereferenced."""
import ctypes as C
import math
import os
import shutil
import subprocess

import pytest
import torch

import paper_2602_23349_amd as fo
from paper_2602_23349_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000


def matrix(rows=4, cols=100, stride=None, dtype=0, data=P):
    return B._Matrix(data, rows, cols, cols if stride is None else stride, dtype)


def logprob(x=None, tokens=P, temperature=1.0, out=P, wide=P, lse=P, ws=P, size=1 << 30):
    return fo.load_library().flashoptim_token_logprob(matrix() if x is None else x, tokens, temperature, out, wide, lse, ws, size, None)


def backward(x=None, tokens=P, temperature=1.0, lse=P, d=P, dx=None):
    return fo.load_library().flashoptim_token_logprob_backward(matrix() if x is None else x, tokens, temperature, lse, d,
                                                               matrix(data=2 * P) if dx is None else dx, None)


def policy(x=None, spec=(1.0, 0.2, 0.2, 0.0, 1.0), inputs=(P, P, P, P), tokens=P, stats=P, lp=P, dx=None, ws=P, size=1 << 30):
    return fo.load_library().flashoptim_policy_loss(B._PolicySpec(*spec), matrix() if x is None else x, tokens, B._PolicyInputs(*inputs),
                                                    stats, lp, matrix(data=2 * P) if dx is None else dx, ws, size, None)


def preference(spec=(0, 0, 0.1, 0.0, 1.0), lp=P, wide=None, ref=P, w=P, rows=10, offsets=P, pairs=2, loss=P, m=P, d=P):
    return fo.load_library().flashoptim_preference_loss(B._PreferenceSpec(*spec), lp, wide, ref, w, rows, offsets, pairs, loss, m, d, None)


BAD_LOGITS = [(dict(x=matrix(rows=-1)), -1), (dict(x=matrix(cols=0)), -1), (dict(x=matrix(dtype=2)), -1), (dict(x=matrix(stride=99)), -1),
              (dict(x=matrix(data=None)), -1), (dict(x=matrix(data=P + 1)), -2), (dict(x=matrix(dtype=1, data=P + 2)), -2),
              (dict(x=matrix(rows=1 << 31)), -3), (dict(x=matrix(rows=1, cols=(1 << 31) - 4096)), -3),
              (dict(x=matrix(rows=(1 << 31) - 1, cols=8), dx=matrix(rows=(1 << 31) - 1, cols=8)), -3),
              (dict(tokens=None), -1), (dict(tokens=P + 4), -2)]
NUMBERS = [0.0, -1.0, math.nan, math.inf, 1e-45]


def without(kw, name):
    return {k: v for k, v in kw.items() if k != name}


def test_log_probabilities_refuse():
    for kw, status in BAD_LOGITS:
        assert logprob(**without(kw, "dx")) == status, kw
        assert backward(**kw) == status, kw
    for t in NUMBERS:
        assert logprob(temperature=t) == -1 and backward(temperature=t) == -1
    assert logprob(out=None, wide=None, lse=None) == -1 and logprob(wide=P + 4) == -2 and logprob(out=P + 2) == -2 and logprob(lse=P + 1) == -2
    assert backward(lse=None) == -1 and backward(d=None) == -1 and backward(lse=P + 2) == -2
    for dx in (matrix(rows=3), matrix(cols=99), matrix(dtype=1), matrix(stride=101)):       # (the last: over the logits, rows elsewhere)
        assert backward(dx=dx) == -1
    assert logprob(x=matrix(rows=0)) == 0 and backward(x=matrix(rows=0), dx=matrix(rows=0)) == 0
    L = fo.load_library()
    assert L.flashoptim_token_logprob_workspace(-1, 5, 0) == -1 and L.flashoptim_token_logprob_workspace(4, 5, 3) == -1
    assert L.flashoptim_token_logprob_workspace(1 << 31, 5, 0) == -3 and L.flashoptim_policy_loss_workspace(5, 1 << 31, 0) == -3


def test_policy_loss_refuses():
    for kw, status in BAD_LOGITS:
        assert policy(**kw) == status, kw
    for i, values in ((0, NUMBERS), (1, [-0.1, math.nan, math.inf]), (2, [-0.1, math.nan]), (3, [-0.1, math.nan, math.inf])):
        for v in values:
            spec = [1.0, 0.2, 0.2, 0.0, 1.0]
            spec[i] = v
            assert policy(spec=spec) == -1, spec
    assert policy(inputs=(None, P, P, P)) == -1 and policy(stats=None) == -1
    for i in range(4):
        assert policy(inputs=[P + 2 if k == i else P for k in range(4)]) == -2
    assert policy(stats=P + 1) == -2 and policy(lp=P + 2) == -2
    for dx in (matrix(rows=3), matrix(cols=99), matrix(dtype=1), matrix(stride=101)):
        assert policy(dx=dx) == -1
    need = fo.load_library().flashoptim_policy_loss_workspace(4, 100, 0)
    assert need > 0 and policy(size=need - 1) == -8 and policy(ws=None, size=0) == -1 and policy(ws=P + 8) == -2


def test_preference_loss_refuses():
    for i, values in ((0, [-1, 3]), (1, [-1, 2]), (2, [0.0, -1.0, math.nan, math.inf]), (3, [-0.1, 0.6, math.nan])):
        for v in values:
            spec = [0, 0, 0.1, 0.0, 1.0]
            spec[i] = v
            assert preference(spec=spec) == -1, spec
    assert preference(spec=(1, 0, 0.1, 0.1, 1.0)) == -1
    assert preference(rows=-1) == -1 and preference(pairs=-1) == -1 and preference(rows=1 << 31) == -3 and preference(pairs=1 << 30) == -3
    assert preference(wide=P) == -1 and preference(lp=None, wide=P + 4) == -2
    assert preference(lp=None) == -1 and preference(offsets=None) == -1 and preference(loss=None) == -1
    assert preference(offsets=P + 4) == -2 and preference(m=P + 2) == -2 and preference(d=P + 1) == -2 and preference(w=P + 3) == -2


def grads(*entries):
    return (B._Gradient * max(len(entries), 1))(*[B._Gradient(*e) for e in entries])


def test_calls_on_gradients_refuse():
    L = fo.load_library()
    good = grads((P, P, 1000), (None, None, 0))
    norm = lambda g=good, n=2, dtype=0, limit=1.0, factor=P, ws=P, size=1 << 20: L.flashoptim_grad_norm(g, n, dtype, limit, factor, ws, size, None)   # noqa: E731
    clip = lambda g=good, n=2, src=0, dst=0, factor=P: L.flashoptim_clip_gradients(g, n, src, dst, factor, None)                                     # noqa: E731
    for call in (norm, clip):
        assert call(n=-1) == -1 and call(g=None) == -1 and call(factor=None) == -1 and call(factor=P + 8) == -2
        for g, status in ((grads((P, P, -1), (P, P, 1)), -3), (grads((P, P, 1 << 40), (P, P, 1)), -3), (grads((None, P, 5), (P, P, 1)), -1),
                          (grads((P + 8, P, 5), (P, P, 1)), -2)):
            assert call(g=g) == status
        assert call(g=grads(*[(P, P, (1 << 40) - 1)] * 9), n=9) == -3
    for dtype in (-1, 2):
        assert norm(dtype=dtype) == -1 and clip(src=dtype) == -1 and clip(dst=dtype) == -1
        assert L.flashoptim_grad_norm_workspace(good, 2, dtype) == -1
    for limit in (-1.0, math.nan):
        assert norm(limit=limit) == -1 and L.flashoptim_clip_factor_from_sum(P, limit, None) == -1
    assert L.flashoptim_clip_factor_from_sum(None, 1.0, None) == -1 and L.flashoptim_clip_factor_from_sum(P + 4, 1.0, None) == -2
    need = L.flashoptim_grad_norm_workspace(good, 2, 0)
    assert need > 0 and norm(size=need - 1) == -8 and norm(ws=None) == -1 and norm(ws=P + 8) == -2
    assert clip(dst=1) == -1                                        # BF16 into FP32
    assert clip(src=1, dst=0) == -1                                 # in place, of two types
    assert clip(g=grads((P, None, 5), (P, P, 1))) == -1 and clip(g=grads((P, P + 8, 5), (P, P, 1))) == -2
    assert clip(n=0) == 0 and L.flashoptim_grad_norm_workspace(None, 0, 0) == 0


def test_the_binding_refuses():
    x = torch.zeros(2, 3)
    with pytest.raises(ValueError):
        fo.GradList([x])                                            # not on the GPU
    with pytest.raises(ValueError):
        fo.GradList([], [x])
    assert fo.GradList([]).n == 0
    for spec, name in ((fo.PreferenceLoss(kind="other"), "kind"), (fo.PreferenceLoss(order="other"), "order")):
        assert getattr(spec.desc, name) == -1


def test_log_probabilities_over_the_inputs_of_the_policy_loss_are_refused():
    # one lane writes a row's logprob while others still read its inputs
    for i in range(4):
        assert policy(inputs=[P if k == i else 3 * P for k in range(4)], stats=4 * P) == -1


class Tensor:
    """What a list of gradients looks at, on a GPU that exists in name only."""
    dtype, is_cuda = torch.bfloat16, True

    def __init__(self, device):
        self.get_device, self.is_contiguous, self.numel, self.data_ptr = lambda: device, lambda: True, lambda: 8, lambda: P


class Factor:
    address = P

    def __init__(self, device):
        self.device = device


def test_lists_over_several_devices_are_refused(monkeypatch):
    from paper_2602_23349_amd import _marshal as M
    names = [n for n in B.EXPORTED_SYMBOLS if n.startswith(("flashoptim_mx4_", "flashoptim_block_norm", "flashoptim_grad_norm", "flashoptim_clip_"))]
    M.bind({n: C.cast(getattr(fo.load_library(), n), C.c_void_p).value for n in names}, lambda device: 0, lambda: 0)
    monkeypatch.setattr(B, "_fast", M)
    here, there = Tensor(0), Tensor(1)
    for args in (([here, there],), ([here], [there])):
        with pytest.raises(ValueError):
            fo.GradList(*args)
    for tensor, factor in ((here, 1), (there, 0), (there, 1)):
        grads = fo.GradList([tensor])
        with pytest.raises(ValueError):
            fo.grad_norm(grads, 1.0, Factor(factor))
        with pytest.raises(ValueError):
            fo.clip_gradients(grads, Factor(factor))


def test_struct_layouts():
    assert C.sizeof(B._Gradient) == 24 and C.sizeof(B._PolicySpec) == 20 and C.sizeof(B._PolicyInputs) == 32 and C.sizeof(B._PreferenceSpec) == 20


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_element_of_a_list_lies_in_one_tile(tmp_path):
    # by the table of a launch, workgroup for workgroup, over tensors of awkward sizes
    src, exe = tmp_path / "clip.cpp", tmp_path / "clip"
    src.write_text("""#include <cstdio>
#include <vector>
#include "flashoptim_clip.h"
int main() {
    const long long sizes[] = {1, 8191, 8192, 8193, 16384, 5, 100000, 7};
    fo::GradTable<16, true> t;
    uint32_t n = 0, tiles = 0;
    for (long long numel : sizes) {
        const int64_t k = fo::grad_tiles(numel);
        t.first[n] = tiles;
        t.lack[n] = (uint16_t)(k * fo::kGradTile - numel);
        tiles += (uint32_t)k;
        t.first[++n] = tiles;
    }
    std::vector<std::vector<int>> seen;
    for (long long numel : sizes) seen.push_back(std::vector<int>(numel, 0));
    long long outside = 0, wrong = 0;
    for (uint32_t b = 0; b < tiles; ++b) {
        const uint32_t i = fo::entry_of(b, 0u, n - 1, [&](uint32_t k) { return t.first[k]; });
        const long long begin = (long long)(b - t.first[i]) * fo::kGradTile;
        const int left = b == t.first[i + 1] - 1 ? fo::kGradTile - (int)t.lack[i] : fo::kGradTile;
        for (int e = 0; e < left; ++e) {
            if (begin + e >= sizes[i]) ++outside; else ++seen[i][begin + e];
        }
    }
    for (auto& v : seen) for (int k : v) wrong += k != 1;
    std::printf("%lld %lld %zu %zu\\n", outside, wrong, sizeof(fo::GradTable<fo::kGradMany, false>), sizeof(fo::GradTable<fo::kClipMany, true>));
}
""")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-I", os.path.join(ROOT, "paper_2602_23349_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    outside, wrong, norm, clip = (int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert outside == 0 and wrong == 0 and norm <= 4032 and clip <= 4032
