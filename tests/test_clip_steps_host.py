"""What the steps that take a clipping factor refuse, before any device work."""
import pytest

import paper_2602_23349_amd as fo
from paper_2602_23349_amd import binding as B

HP = {"adamw_step": B._AdamWHp(0.9, 0.99, 1e-8, 1), "adamw_step_exact": B._AdamWHp(0.9, 0.99, 1e-8, 1), "sgd_step": B._SgdHp(0.9),
      "lion_step": B._LionHp(0.9, 0.99)}


@pytest.mark.parametrize("name", HP)
def test_clipped_steps_refuse(name):
    lib = fo.load_library()
    call = getattr(lib, f"flashoptim_{name}_clipped")
    codes = {}
    t = (B._Tensor * 1)()
    for field in ("param", "rho", "grad", "m_q", "m_scale", "v_q", "v_scale"):
        setattr(t[0], field, 0x1000)
    t[0].numel = 0
    assert call(t, 1, HP[name], 0x1000, None) == 0            # nothing to do
    assert call(t, 0, HP[name], 0x1000, None) == 0
    codes["invalid"], codes["misaligned"] = call(t, 1, HP[name], None, None), call(t, 1, HP[name], 0x1008, None)
    plain = getattr(lib, f"flashoptim_{name}")
    t[0].numel = 5
    t[0].grad = None
    assert codes["invalid"] == call(t, 1, HP[name], 0x1000, None) == plain(t, 1, HP[name], None) != 0
    t[0].grad = 0x1008
    assert codes["misaligned"] == call(t, 1, HP[name], 0x1000, None) == plain(t, 1, HP[name], None) != 0
    assert codes["invalid"] != codes["misaligned"]
    t[0].grad = 0x1000
    assert call(t, 1, None, 0x1000, None) == codes["invalid"]
    t[0].numel = -1
    assert call(t, 1, HP[name], 0x1000, None) == plain(t, 1, HP[name], None) != 0
