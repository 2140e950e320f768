"""Calls on 8-bit blocks whose outputs lie over their inputs, or over one another, in a way that has no defined result: refused
before any CUDA call (no address that is passed here is looked at)."""
import pytest

import paper_2204_08211_b200 as co3

AT, ROOM = 1 << 20, 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2204_08211_b200 import binding
    return binding._load()


@pytest.mark.parametrize("x_stride,y_stride", [(8, 16), (16, 8)])
def test_rows_over_themselves_need_one_stride(lib, x_stride, y_stride):
    act = lambda a: lib.co3_f8_activation(AT, 0, 8, 8, x_stride, a, AT, y_stride, None, None, ROOM, None)
    back = lambda a: lib.co3_f8_activation_backward(AT, 0, 8, 8, x_stride, 4 * AT, ROOM, a, AT, y_stride, None)
    for a in (co3.ACT_NONE, co3.ACT_RELU, co3.ACT_GELU, co3.ACT_SILU):
        assert act(a) == co3.ERR_INVALID_ARG and back(a) == co3.ERR_INVALID_ARG


def test_the_two_buffers_of_blocks_lie_apart(lib):
    """8 x 8 entries take 16384 + 512 bytes."""
    act = lambda y8, x8: lib.co3_f8_activation(8 * AT, 0, 8, 8, 8, co3.ACT_RELU, None, 0, y8, x8, ROOM, None)
    assert co3.co3_f8_bytes(8, 8) == 16896
    for d in (0, 256, 16640):
        assert act(AT, AT + d) == co3.ERR_INVALID_ARG and act(AT + d, AT) == co3.ERR_INVALID_ARG
