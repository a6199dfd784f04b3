"""The gated activation in fp32 is as exact as fp32 arithmetic: s = 1 / (1 + e^-x) from an exponential within 2 ulp (2^-22), one
rounded addition and one rounded reciprocal, then products of one rounding each: h within 2^-21 of its value wherever s is a normal
number; the gradients within 2^-20 of their largest terms."""
import pytest
import torch

import ops_reference as R
from paper_2502_11034_b200 import act8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [4096, 4099])
def test_fp32_activation_far_from_zero(cols):
    gen = torch.Generator("cuda").manual_seed(cols)
    g = torch.rand(20, cols, device="cuda", generator=gen) * 160 - 80
    u, dh = (torch.randn(20, cols, device="cuda", generator=gen) for _ in range(2))
    h, g8, u8 = act8.swiglu(g, u)
    want = R.swiglu(g.double(), u.double())
    rel = ((h.double() - want).abs() / want.abs()).max()
    assert float(rel) <= 2 ** -21, float(rel)
    dg, du, _ = act8.swiglu_backward(dh, g8, u8)
    gh, uh = act8.decode(g8, torch.float32).double(), act8.decode(u8, torch.float32).double()
    wg, wu = R.swiglu_grad(dh.double(), gh, uh)
    s = 1 / (1 + torch.exp(-gh))
    tol_g = (dh.double() * uh).abs() * s * (1 + gh.abs()) * 2 ** -20 + 1e-37
    assert float(((dg.double() - wg).abs() / tol_g).max()) <= 1
    assert ((du.double() - wu).abs() <= wu.abs() * 2 ** -21 + 1e-37).all()
