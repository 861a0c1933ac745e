"""The module that marshals tensors for the calls of the layers (csrc/marshal.cpp), without a GPU: tensors that have no memory are refused
by a Python error, as they are by the calls that go through ctypes."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Each call of the module, `t` being a matrix on a GPU that exists in name only and `r` a row of it inside torch.vmap or torch.func.grad: the
# shape and type of such a tensor are there, its memory is not.  In a process of its own, which an exception that nobody catches ends.
PROGRAM = """
import ctypes, sys, warnings
import torch
from torch._subclasses import FakeTensorMode
import paper_2602_23349_amd as fo
from paper_2602_23349_amd import binding as B
from paper_2602_23349_amd import _marshal as M
warnings.simplefilter("ignore")
lib = fo.load_library()
names = [n for n in B.EXPORTED_SYMBOLS if n.startswith(("flashoptim_mx4_", "flashoptim_block_norm"))]
M.bind({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names}, lambda device: 0, lambda: 0)
spec = B._BlockNormSpec(cols=64, eps=1e-5, residual_scale=1, branch_scale=1)
mx4, norm = ctypes.addressof(B._Mx4(4096, 4096, 1, 64)), ctypes.addressof(spec)
calls = {
    "quantize": lambda r, b, s: M.quantize(r, mx4, None, None, None, 0),
    "rand": lambda r, b, s: M.quantize(None, mx4, None, None, b, 0),
    "dequantize": lambda r, b, s: M.dequantize(mx4, r, 0),
    "matmul": lambda r, b, s: M.matmul(mx4, mx4, r, None, 0),
    "workspace": lambda r, b, s: M.matmul(mx4, mx4, None, b, 0),
    "linear": lambda r, b, s: M.linear(r, mx4, None, r, None, 0),
    "linear_backward": lambda r, b, s: M.linear_backward(r, None, mx4, mx4, r, r, None, 0),
    "norm": lambda r, b, s: M.norm(norm, r, None, None, None, r, None, 0),
    "stats": lambda r, b, s: M.norm(norm, None, None, None, None, None, s, 0),
    "norm_backward": lambda r, b, s: M.norm_backward(norm, r, None, *[None] * 12, 0),
}

def one(row):
    r = row[None]
    for name, call in calls.items():
        print(name, flush=True)
        try:
            call(r, row[:0, None].expand(0, 0).to(torch.uint8), row[:0].float())
        except RuntimeError as e:
            assert "storage" in str(e) or "data pointer" in str(e), e
            print("refused")
    raise Done                    # (torch's own pass over the result needs a GPU)

class Done(Exception):
    pass

with FakeTensorMode():
    t = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")
    try:
        torch.vmap(one)(t) if sys.argv[1] == "vmap" else torch.func.grad(one)(t[0])
    except Done:
        print("end")
"""


@pytest.mark.parametrize("how", ["vmap", "grad"])
def test_a_tensor_without_memory_is_an_error_and_not_the_end(how):
    r = subprocess.run([sys.executable, "-c", PROGRAM, how], cwd=ROOT, capture_output=True, text=True, timeout=300)
    calls = ["quantize", "rand", "dequantize", "matmul", "workspace", "linear", "linear_backward", "norm", "stats", "norm_backward"]
    assert r.returncode == 0 and r.stdout.split() == [w for call in calls for w in (call, "refused")] + ["end"], (r.stdout, r.stderr[-600:])
