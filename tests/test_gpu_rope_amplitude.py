"""The amplitude that goes with a ramp: 0.1 log(factor) + 1 where positions are stretched, 1 where they are not."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("factor,want", [(0.25, 1.0), (0.999, 1.0), (1.0, 1.0), (2.0, 0.1 * math.log(2.0) + 1.0), (32.0, 0.1 * math.log(32.0) + 1.0)])
def test_ramp(factor, want):
    import paper_2603_05210_b200 as vt
    rope = vt.vt_rope_table(64, scaling="ramp", factor=factor)
    assert rope.amplitude == want
    q = torch.randn(5, 3, 64, device="cuda").bfloat16()
    y = vt.vt_rope(q, None, torch.arange(5, dtype=torch.int32, device="cuda") * 1000, rope)[0]
    norms = [t.double().norm(dim=-1) for t in (y, q)]
    assert bool(((norms[0] - want * norms[1]).abs() <= (2.0 ** -8 + 1e-5) * want * norms[1]).all())       # elements are rounded once
    assert vt.vt_rope_table(64, scaling="ramp", factor=factor, amplitude=1.3).amplitude == 1.3


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "wavelength"])
def test_others_have_none(scaling):
    import paper_2603_05210_b200 as vt
    assert vt.vt_rope_table(64, scaling=scaling, factor=4.0).amplitude == 1.0
