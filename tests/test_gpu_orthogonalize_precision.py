"""fp32 and fp16 results of co3_orthogonalize against a few times the plain fp32 form's own error: tight enough to tell
operands of 22 bits from such of 11 in any of the steps.

Tolerance as in test_gpu_orthogonalize_bf16.py: four times the plain form's error on the same input (values are held to
2^-22, four times fp32's unit) plus 16 units of 2^-22; twice that beside the rounding itself where the result is fp16."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from test_gpu_orthogonalize import COEF, SHAPES, TYPES, definition, orthogonalize, spectrum
from test_gpu_orthogonalize_bf16 import allowed

pytestmark = pytest.mark.gpu


def single_halves(g, steps):
    """The definition with the operands of the first `steps` steps rounded to 11 bits, as fp16 values near 1 are."""
    def cut(x):
        m, e = torch.frexp(x)
        return torch.ldexp(torch.round(m * 2048) / 2048, e)
    x = g.double().cpu()
    if x.shape[0] > x.shape[1]:
        return single_halves(x.T, steps).T
    x = x / (torch.linalg.norm(x) + 1e-7)
    a, b, c = COEF
    for k in range(5):
        h = cut if k < steps else lambda t: t
        s = h(x) @ h(x).T
        x = a * x + h(b * s + c * (h(s) @ h(s))) @ h(x)
    return x


@pytest.mark.parametrize("kind", ["normal", "lowrank", "heavy"])
@pytest.mark.parametrize("rows,cols", SHAPES + [(8, 4096), (2100, 12), (512, 512), (1024, 1100)])
def test_fp32(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 1009 + cols + 1)
    g = spectrum(kind, rows, cols, gen).float().cuda()
    out = torch.empty_like(g)
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out)
    want = definition(g)
    assert r["status"] == co3.OK
    assert torch.linalg.norm(out.double().cpu() - want).item() <= allowed(g, want)


@pytest.mark.parametrize("tin", ["f32", "f16"])
@pytest.mark.parametrize("rows,cols", [(5, 3), (64, 147), (128, 640), (200, 513), (1000, 513), (8, 4096)])
def test_fp16(rows, cols, tin):
    gen = torch.Generator().manual_seed(rows + cols)
    g = spectrum("normal", rows, cols, gen).to(TYPES[tin]).cuda()
    out = torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out)
    want = definition(g)
    assert r["status"] == co3.OK
    rounding = torch.linalg.norm(want.half().double() - want).item()
    assert torch.linalg.norm(out.double().cpu() - want).item() <= rounding + 2 * allowed(g, want)


@pytest.mark.parametrize("rows,cols", [(16, 16), (64, 147), (200, 513), (513, 200), (8, 4096)])
@pytest.mark.parametrize("kind", ["normal", "lowrank", "heavy"])
def test_the_tolerance_tells_22_bits_from_11(rows, cols, kind):
    """Two steps of 11 bits would not pass."""
    gen = torch.Generator().manual_seed(rows * 1009 + cols + 1)
    g = spectrum(kind, rows, cols, gen).float()
    want = definition(g)
    assert torch.linalg.norm(single_halves(g, 2) - want).item() > allowed(g, want)
