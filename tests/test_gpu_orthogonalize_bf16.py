"""bf16 results of co3_orthogonalize carry the rounding to bf16 and no more, whatever the sides and the spectrum.

Tolerance.  Let X be the definition's result in 64 bits and E the error before the rounding.  Rounding to nearest gives
|round(X + E) - (X + E)| <= |round(X) - X| + |E| element by element, so that in Frobenius norms
    ||result - X|| <= ||round(X) - X|| + 2 ||E||.
Values are held to 2^-22, four times the unit of fp32: ||E|| is allowed four times the error of the plain fp32 form on the
same input, plus 16 units of 2^-22 of ||X|| for inputs on which the plain form is exact by chance.
"""
import pytest
import torch

import paper_2204_08211_b200 as co3
from test_gpu_orthogonalize import TYPES, definition, orthogonalize, spectrum

pytestmark = pytest.mark.gpu


def plain32(g):
    """The formula in fp32 on the CPU."""
    x = g.detach().float().cpu()
    if x.shape[0] > x.shape[1]:
        return plain32(x.T.contiguous()).T
    x = x / (x.square().sum().sqrt() + 1e-7)
    for _ in range(5):
        s = x @ x.T
        x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
    return x


def allowed(g, want):
    """What the values before the last rounding may be off (see above)."""
    return 4 * torch.linalg.norm(plain32(g).double() - want).item() + 16 * 2.0 ** -22 * torch.linalg.norm(want).item()


@pytest.mark.parametrize("tin", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "lowrank", "heavy"])
@pytest.mark.parametrize("rows,cols", [(8, 4096), (2100, 12), (32, 3000), (64, 8192), (300, 300), (512, 512), (1024, 1100), (1500, 1030)])
def test_no_error_but_the_rounding(rows, cols, kind, tin):
    gen = torch.Generator().manual_seed(rows * 31 + cols)
    g = spectrum(kind, rows, cols, gen).to(TYPES[tin]).cuda()
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out)
    want = definition(g)
    assert r["status"] == co3.OK
    rounding = torch.linalg.norm(want.to(torch.bfloat16).double() - want).item()
    assert torch.linalg.norm(out.double().cpu() - want).item() <= rounding + 2 * allowed(g, want)


@pytest.mark.parametrize("other", [(0, 0), (5, 7)])
def test_precision_does_not_depend_on_the_other_matrices(other):
    """A small or an empty matrix in the list leaves the large one's accuracy as it is."""
    rows, cols = 1024, 1100
    gen = torch.Generator().manual_seed(77)
    g = torch.cat([spectrum("heavy", rows, cols, gen).reshape(-1), torch.randn(35, generator=gen, dtype=torch.float64)]).float().cuda()
    out = torch.empty(g.numel(), dtype=torch.bfloat16, device="cuda")
    r = orthogonalize(g, co3.make_mats([(0, rows, cols), (rows * cols, *other)]), out)
    m = g[:rows * cols].view(rows, cols)
    want = definition(m)
    assert r["status"] == co3.OK
    rounding = torch.linalg.norm(want.to(torch.bfloat16).double() - want).item()
    assert torch.linalg.norm(out[:rows * cols].view(rows, cols).double().cpu() - want).item() <= rounding + 2 * allowed(m, want)
