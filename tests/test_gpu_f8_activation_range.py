"""The activations on 8-bit blocks where exponentials leave fp32's normal range while the result, or its slope, is still a number of
the type; every 16-bit value.

Tolerances as in test_gpu_f8_blocks.py, but nothing counts as zero: relative to the result (the slope: to the size of its terms)
2^-17 for the short forms of 16-bit results and what the exponents' roundings add, half a step of the type, half its smallest step.
An exponential below 2^-126 has lost up to 2^-150, which the factor |x| <= 128 multiplies: 2^-143.
"""
import math

import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import TYPES, UNIT
from test_gpu_f8_blocks import U, act64, room, slack

pytestmark = pytest.mark.gpu

STEP = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}       # half the smallest
CURVED = [co3.ACT_GELU, co3.ACT_SILU]


LOST = 2.0 ** -143


@pytest.mark.parametrize("type_", ["f16", "bf16"])
@pytest.mark.parametrize("act", CURVED)
def test_every_16_bit_value(act, type_):
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.uint16).view(TYPES[type_]).view(512, 128)
    y = torch.empty(512, 128, dtype=TYPES[type_], device="cuda")
    assert co3.co3_f8_activation(x.cuda(), act, y) == co3.OK
    torch.cuda.synchronize()
    x64, got = x.double(), y.double().cpu()
    fine = torch.isfinite(x64)
    want = act64(act, x64)[0]
    err = (slack(act, type_, x64) + UNIT[type_]) * want.abs() + LOST + STEP[type_]
    assert ((got - want).abs() <= err)[fine].all()
    assert torch.isnan(got[torch.isnan(x64)]).all()
    assert (got[x64 == math.inf] == math.inf).all() and (got[x64 == -math.inf] == 0).all()


@pytest.mark.parametrize("act", CURVED)
def test_far_below_zero_fp32(act):
    """GELU to where erfc leaves the normal range, SILU beyond the last subnormal."""
    x = torch.linspace(-13.0 if act == co3.ACT_GELU else -112.0, 20, 1 << 16).view(512, 128)
    y = torch.empty(512, 128, device="cuda")
    assert co3.co3_f8_activation(x.cuda(), act, y) == co3.OK
    torch.cuda.synchronize()
    want = act64(act, x.double())[0]
    err = (slack(act, "f32", x.double()) + U) * want.abs() + LOST + STEP["f32"]
    assert ((y.double().cpu() - want).abs() <= err).all()


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("act", CURVED)
def test_slopes(act, type_):
    """Rows of one value each, of four significant bits, so that the blocks hold it exactly."""
    m = torch.arange(8, 16).float()
    v = torch.cat([m * 2.0 ** k for k in range(-12, 5)])
    v = v[v <= (13.0 if act == co3.ACT_GELU and type_ == "f32" else 120.0)]
    v = torch.cat([v, -v])
    x8, dx = room(v.numel(), 128), torch.empty(v.numel(), 128, dtype=TYPES[type_], device="cuda")
    assert co3.co3_f8_pack(v[:, None].expand(-1, 128).contiguous().cuda(), x8) == co3.OK
    assert co3.co3_f8_activation_backward(torch.ones_like(dx), x8, act, dx) == co3.OK
    torch.cuda.synchronize()
    _, want, size = act64(act, v.double())
    err = 2 * slack(act, type_, v.double()) * size + UNIT[type_] * want.abs() + 2 * LOST + STEP[type_]
    got = dx.double().cpu()
    assert ((got - want[:, None]).abs() <= err[:, None]).all()
