"""y8, the activation's result in 8-bit blocks, to the code."""
import math

import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import BLOCK, TYPES, e4m3, padded
from test_gpu_f8_blocks import ACTS, act64, inputs, room, slack

pytestmark = pytest.mark.gpu

LOST = 2.0 ** -143                   # of act(x), where an exponential is below 2^-126


def exponent(most):
    """The smallest k >= -126 with most <= 448 * 2^k."""
    k = max(-126, int(math.frexp(most)[1]) - 10) if most else -126
    while 448.0 * 2.0 ** k < most:
        k += 1
    return k


def codes_within(got, y, err):
    """Whether each block of `got` is the packed form of some values within err of y: with one of the scales that their largest magnitude
    can have, every entry lies between the codes of y - err and y + err (rounding is monotonous)."""
    for r in range(y.shape[0]):
        for c in range(0, y.shape[1], BLOCK):
            g, v, e = (t[r, c:c + BLOCK].numpy() for t in (got, y, err))
            most = [max(0.0, float((abs(v) - e).max())), float((abs(v) + e).max())]
            fits = False
            for k in range(exponent(most[0]), exponent(most[1]) + 1):
                lo, hi = e4m3((v - e) / 2.0 ** k) * 2.0 ** k, e4m3((v + e) / 2.0 ** k) * 2.0 ** k
                fits |= bool(((lo <= g) & (g <= hi)).all())
            if not fits:
                return False
    return True


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cols,pad", [(3, 127, 1), (33, 512, 0), (20, 1000, 0)])
def test_y8_to_the_code(rows, cols, pad, act, type_):
    _, x = padded(inputs(rows, cols, rows + act, 1.5), type_, pad, pad)
    y8, got = room(rows, cols), torch.empty(rows, cols, device="cuda")
    assert co3.co3_f8_activation(x, act, None, y8) == co3.OK and co3.co3_f8_unpack(y8, got) == co3.OK
    torch.cuda.synchronize()
    x64 = x.double().cpu()
    y64 = act64(act, x64)[0]
    assert codes_within(got.double().cpu(), y64, slack(act, type_, x64) * y64.abs() + (LOST if act >= co3.ACT_GELU else 0.0))


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("act", [co3.ACT_GELU, co3.ACT_SILU])
def test_y8_within_the_stated_bound(act, type_):
    """The header's bound, 2^-15 of act(x) where |x| <= 10."""
    x = torch.linspace(-10, 10, 40 * 256).view(40, 256).to(TYPES[type_])
    y8, got = room(40, 256), torch.empty(40, 256, device="cuda")
    assert co3.co3_f8_activation(x.cuda(), act, None, y8) == co3.OK and co3.co3_f8_unpack(y8, got) == co3.OK
    torch.cuda.synchronize()
    y64 = act64(act, x.double())[0]
    assert codes_within(got.double().cpu(), y64, 2.0 ** -15 * y64.abs())


def test_the_check_of_codes_notices_a_neighbour():
    """Planted in the values compared, on the host: one entry moved to the next code."""
    x = inputs(2, 256, 7).double()
    k = torch.tensor([[exponent(float(x[r, c:c + BLOCK].abs().max())) for c in range(0, 256, BLOCK)] for r in range(2)]).repeat_interleave(BLOCK, 1)
    u = torch.from_numpy(e4m3((x / 2.0 ** k).numpy()))
    err = 2.0 ** -17 * x.abs()
    assert codes_within(u * 2.0 ** k, x, err)
    r, c = 1, 200
    step = 2.0 ** (max(-6, math.floor(math.log2(abs(u[r, c])))) - 3)
    u[r, c] += step if u[r, c].abs() < 400 else -step
    assert not codes_within(u * 2.0 ** k, x, err)
