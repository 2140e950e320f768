"""Matrices that a cluster of blocks works on together, call after call: every result against the definition, and the same
bits each time.  Short sides of 113 to 128 fill the blocks' shared memory, where what one block still reads must not be
what another one writes."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from test_gpu_orthogonalize import bound, definition, result

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(113, 129), (120, 300), (127, 2048), (128, 256), (128, 1152), (128, 2048), (2048, 128), (600, 125)])
@pytest.mark.parametrize("count", [1, 6])
def test_full_blocks(rows, cols, count):
    """One matrix, and as many as keep the GPU's clusters busy at the same time."""
    gen = torch.Generator().manual_seed(rows + cols + count)
    g = torch.randn(count, rows, cols, generator=gen).cuda()
    mats = co3.make_mats([(k * rows * cols, rows, cols) for k in range(count)])
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res, first, out = result(), torch.empty_like(g), torch.empty_like(g)
    same = torch.ones((), dtype=torch.bool, device="cuda")
    assert co3.co3_orthogonalize(g, mats, first, None, ws, res) == co3.OK
    for _ in range(200):
        assert co3.co3_orthogonalize(g, mats, out, None, ws, res) == co3.OK
        same &= (out == first).all()
    torch.cuda.synchronize()
    assert co3.read_results(res, 1)[0]["status"] == co3.OK
    for k in range(count):
        want = definition(g[k])
        assert torch.linalg.norm(first[k].double().cpu() - want).item() <= bound(g[k], want, "f32")
    assert same.item()
