"""Which iterations co3_orthogonalize takes: those that keep every singular value in [0, 1] inside [-2, 2], not only the
values on some grid, with what the arithmetic rounds on the way."""
import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu

DEFAULT = (3.4445, -4.7750, 2.0315)


def call(coef):
    g = torch.randn(48, 64, generator=torch.Generator().manual_seed(1)).cuda()
    mats = co3.make_mats([(0, 48, 64)])
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res = torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
    out = torch.full_like(g, 7.0)
    st = co3.co3_orthogonalize(g, mats, out, None, ws, res, co3.make_ns(coef))
    torch.cuda.synchronize()
    return st, out


def largest(coef, n=2000001):
    """Of |x| on the way, from n points of [0, 1]."""
    x, most = np.linspace(0, 1, n), 0.0
    for a, b, c in np.asarray(coef, dtype=np.float32).astype(np.float64):
        q = x * x
        x = x * (a + q * (b + c * q))
        most = max(most, np.abs(x).max())
    return most


@pytest.mark.parametrize("steps", [10, 12, 14])
def test_refuses_values_that_escape_between_the_points_of_a_grid(steps):
    """x -> x^3 - 3 x keeps [-2, 2]; a millionth more and a few values leave it, and then grow without bound."""
    coef = [(0.9845923, 0.0, 0.0)] + [(-3.000003, 1.000001, 0.0)] * (steps - 1)
    assert largest(coef) > 10
    st, out = call(coef)
    assert st == co3.ERR_INVALID_ARG and (out == 7.0).all()


@pytest.mark.parametrize("coef", [[(-3.0, 1.0, 0.0)] * 16, [(2.01, 0.0, 0.0)], [(1.5, 0.0, 0.0)] * 2, [(4.1, -4.0, 0.0)],
                                  [(1.0, 0.0, 0.0)] * 3 + [(9.0, -4.0, 2.0)]])
def test_refuses(coef):
    """The first keeps [-2, 2] in exact arithmetic, where every rounding beyond it grows nine times a step."""
    st, out = call(coef)
    assert st == co3.ERR_INVALID_ARG and (out == 7.0).all()


@pytest.mark.parametrize("coef", [[DEFAULT] * 5, [DEFAULT] * 16, [(1.5, -0.5, 0.0)] * 16, [(1.875, -1.25, 0.375)] * 16, [(1.0, 0.0, 0.0)] * 16,
                                  [(2.0, 0.0, 0.0)], [(4.0, -4.0, 0.0)], [(-1.5, 0.5, 0.0)] * 5, [(0.0, 0.0, 0.0)], [(-0.5, 4.1, -4.0)],
                                  [DEFAULT] * 3 + [(1.875, -1.25, 0.375)] * 5])
def test_accepts(coef):
    st, out = call(coef)
    assert st == co3.OK and torch.isfinite(out).all() and (out != 7.0).all()
