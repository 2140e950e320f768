"""How a product of few tiles divides its sum among blocks follows from the sizes alone, as the header promises of its bits.

The division is read off the result.  A row of x has 2^24 in the first block of 128 columns and two ones in neighbouring blocks, the
weights are ones: where one block of threads adds up both ones, its part is 2 and the sum 2^24 + 2; where they lie in two
parts, each of them is added to 2^24 alone and rounds to nothing (ties to even).
"""
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu

BLOCKS = 16                                                # of columns of the sum
PARTS = {15: 8, 16: 4, 33: 4, 34: 2, 74: 2}                # of it, for so many tiles of 128 features


@pytest.mark.parametrize("rows", [4, 64])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tiles", list(PARTS))
def test_parts(tiles, transposed, rows):
    features, cols, parts = 128 * tiles, 128 * BLOCKS, PARTS[tiles]
    outs, ins = (cols, features) if transposed else (features, cols)
    w8 = torch.empty(co3.co3_f8_bytes(outs, ins, co3.F8_SQUARE), dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_pack(torch.ones(outs, ins, device="cuda"), w8, co3.F8_SQUARE) == co3.OK
    x8 = torch.empty(co3.co3_f8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    at = list(range(BLOCKS // parts, BLOCKS - 1))          # neighbours from the second part on
    for i in range(0, len(at), rows):
        some = at[i:i + rows]
        x, y = torch.zeros(rows, cols, device="cuda"), torch.empty(rows, features, device="cuda")
        x[:, 0] = 2.0 ** 24
        for r, q in enumerate(some):
            x[r, 128 * q], x[r, 128 * (q + 1)] = 1.0, 1.0
        assert co3.co3_f8_linear(x, x8, w8, None, y, transposed) == co3.OK
        torch.cuda.synchronize()
        for r, q in enumerate(some):
            together = q * parts // BLOCKS == (q + 1) * parts // BLOCKS
            assert (y[r] == 2.0 ** 24 + (2.0 if together else 0.0)).all(), q
