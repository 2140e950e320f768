"""What co3_muon_update says of layers that hold a NaN or an infinity, plain layers among them: each counted once, the first
one's place in the list, and nothing of what an earlier call left in the result."""
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu

# matrices beside the plain layers: none, such as go to clusters, and one that does not
MATRICES = {"none": [], "small": [(20, 30), (64, 100)], "large": [(300, 300), (20, 30)]}


def setup(matrices, plain):
    """Layers, plain ones first and last; the list's places of the plain ones."""
    half = len(plain) // 2
    shapes = [(n, 0) for n in plain[:half]] + matrices + [(n, 0) for n in plain[half:]]
    rows, off = [], 0
    for r, c in shapes:
        rows.append((off, r, c, c, 1.0, 0) if c else (off, 1, r, r, 1.0, co3.MAT_PLAIN))
        off += r * max(c, 1)
    return co3.make_mats(rows), off, [k for k, (_, c) in enumerate(shapes) if c == 0]


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("kind", list(MATRICES))
def test_plain_layers(kind, value):
    mats, n, plain = setup(MATRICES[kind], [10, 100000, 1, 7, 20000, 3])      # the long ones take many blocks
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res = torch.full((co3.RESULT_DTYPE.itemsize,), 0x55, dtype=torch.uint8, device="cuda")

    def call(bad):
        g = torch.randn(n, generator=torch.Generator().manual_seed(4)).cuda()
        for at in bad:
            g[at] = value
        p, m = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        assert co3.co3_muon_update(g, m, p, mats, 0.9, True, 0.1, 0.0, ws, res) == co3.OK
        torch.cuda.synchronize()
        finite = torch.isfinite(p)
        want = torch.ones(n, dtype=torch.bool)
        want[bad] = False
        assert torch.equal(finite.cpu(), want)                                 # a plain layer's other entries are stepped
        return co3.read_results(res, 1)[0]

    offsets = [int(mats["offset"][k]) for k in plain]
    sizes = [int(mats["cols"][k]) for k in plain]
    for first in range(len(plain)):
        for at in {offsets[first], offsets[first] + sizes[first] - 1}:         # its first and its last entry
            r = call([at])
            assert r["status"] == co3.ERR_NONFINITE and r["n_nonfinite"] == 1 and r["first_bad_chunk"] == plain[first]
    r = call([])                                                               # the result held an error before
    assert r["status"] == co3.OK and r["n_nonfinite"] == 0
    r = call([offsets[1] + k for k in (5, 9000, 70000)] + [offsets[4]])        # several entries of a layer count once
    assert r["status"] == co3.ERR_NONFINITE and r["n_nonfinite"] == 2 and r["first_bad_chunk"] == plain[1]


@pytest.mark.parametrize("kind", ["small", "large"])
def test_plain_layers_and_matrices_together(kind):
    mats, n, plain = setup(MATRICES[kind], [10, 20])
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res = torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
    g = torch.randn(n, generator=torch.Generator().manual_seed(4)).cuda()
    for k in (1, 2, 3):                                                        # both matrices and the last plain layer
        g[int(mats["offset"][k])] = float("nan")
    p, m = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    assert co3.co3_muon_update(g, m, p, mats, 0.9, True, 0.1, 0.0, ws, res) == co3.OK
    torch.cuda.synchronize()
    r = co3.read_results(res, 1)[0]
    assert r["status"] == co3.ERR_NONFINITE and r["n_nonfinite"] == 3 and r["first_bad_chunk"] == 1


def test_a_plain_layer_of_a_later_batch():
    """More layers than one batch of launches holds; many calls in a row, each with the report of its own."""
    mats, n, _ = setup([], [5] * 250)
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    size = co3.RESULT_DTYPE.itemsize
    places = [0, 95, 96, 191, 192, 249] * 20
    res = torch.full((len(places) * size,), 0xFF, dtype=torch.uint8, device="cuda")
    for i, k in enumerate(places):
        g = torch.ones(n, device="cuda")
        g[5 * k + 2] = float("nan")
        p, m = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        assert co3.co3_muon_update(g, m, p, mats, 0.9, False, 0.1, 0.0, ws, res[i * size:(i + 1) * size]) == co3.OK
    torch.cuda.synchronize()
    got = co3.read_results(res, len(places))
    assert (got["status"] == co3.ERR_NONFINITE).all() and (got["n_nonfinite"] == 1).all()
    assert got["first_bad_chunk"].tolist() == places
