"""8-bit blocks without a GPU: sizes, and the arguments that the calls refuse before any CUDA call (no address that is passed
here is looked at)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import blocks, e4m3

AT, U31 = 1 << 20, 1 << 31


@pytest.fixture(scope="module")
def lib():
    from paper_2204_08211_b200 import binding
    return binding._load()


def test_reference_is_the_format():
    """The reference the GPU tests use: all 256 codes are their own nearest values, midpoints go to the even code."""
    codes = np.sort(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64))
    codes = np.unique(codes[np.isfinite(codes)])
    assert np.array_equal(e4m3(codes), codes) and codes.max() == 448.0
    mid = (codes[1:] + codes[:-1]) / 2
    want = torch.from_numpy(mid.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(e4m3(mid), want.astype(np.float64))
    exps, vals = blocks(np.array([[448.0, 1.0], [449.0, 1.0], [0.0, 0.0], [np.inf, 2.0]]), False)
    assert exps[:, 0].tolist() == [0, 1, -126, -7] and vals[0, 0] == 448.0 and vals[3, 1] == 2.0 and np.isnan(vals[3, 0])


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (1, 128), (128, 129), (129, 513), (3001, 1023)])
def test_bytes(rows, cols):
    """Whole tiles of 128 x 128, 512 bytes of exponents for 128 rows and four blocks (square blocks: in both directions)."""
    tiles, kb = -(-rows // 128), -(-cols // 128)
    by_rows = tiles * kb * 16384 + tiles * -(-kb // 4) * 512
    assert co3.co3_f8_bytes(rows, cols) == max(256, by_rows)
    assert co3.co3_f8_bytes(rows, cols, co3.F8_SQUARE) == max(256, by_rows + -(-tiles // 4) * kb * 512)


def test_bytes_refusals(lib):
    out = ctypes.c_size_t(0)
    for rows, cols, kind in ((U31, 1, 0), (1, U31, 0), (U31 - 1, 128 * 512, 0), (1, 1, 2), (1, 1, -1)):
        assert lib.co3_f8_bytes(rows, cols, kind, ctypes.byref(out)) == co3.ERR_INVALID_ARG
    assert lib.co3_f8_bytes(1, 1, 0, None) == co3.ERR_INVALID_ARG
    assert lib.co3_f8_bytes(U31 - 1, 128, 0, ctypes.byref(out)) == co3.OK
    for rows, outs, ins, clients in ((U31, 8, 8, 1), (1 << 20, 8, 8, 1 << 11), (8, U31, 8, 1), (8, 8, U31, 1), (8, 1 << 20, 1 << 20, 1), (8, 8, 8, 0)):
        assert lib.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, clients, ctypes.byref(out)) == co3.ERR_INVALID_ARG


def test_sizes_that_would_be_cut_to_32_bits():
    for rows, cols in ((1, 2 ** 32 + 5), (2 ** 32 + 5, 1), (-1, 4), (4, -1), (2 ** 31, 1)):
        with pytest.raises(ValueError):
            co3.co3_f8_bytes(rows, cols)
        with pytest.raises(ValueError):
            co3.co3_f8_weight_gradient_workspace_bytes(rows, cols, 8)
    with pytest.raises(ValueError):
        co3.co3_f8_weight_gradient_workspace_bytes(8, 8, 2 ** 32 + 8)


def test_pack_and_activation_refusals(lib):
    big = 1 << 40
    pack = lambda x=AT, t=0, rows=8, cols=8, stride=8, kind=0, out=AT, n=big: lib.co3_f8_pack(x, t, rows, cols, stride, kind, out, n, None)
    unpack = lambda x=AT, n=big, kind=0, y=AT, t=0, rows=8, cols=8, stride=8: lib.co3_f8_unpack(x, n, kind, y, t, rows, cols, stride, None)
    for kind in (0, 1):
        for bad in (dict(x=None), dict(x=AT + 2), dict(t=3), dict(t=-1), dict(stride=7), dict(stride=big), dict(out=None), dict(out=AT + 128), dict(rows=U31)):
            assert pack(kind=kind, **bad) == co3.ERR_INVALID_ARG, bad
        assert pack(kind=kind, n=co3.co3_f8_bytes(8, 8, kind) - 1) == co3.ERR_CAPACITY
        for bad in (dict(x=None), dict(x=AT + 16), dict(t=3), dict(stride=7), dict(y=None), dict(y=AT + 1)):
            assert unpack(kind=kind, **bad) == co3.ERR_INVALID_ARG, bad
        assert unpack(kind=kind, n=co3.co3_f8_bytes(8, 8, kind) - 1) == co3.ERR_CAPACITY
        assert pack(kind=kind, rows=0, x=None) == co3.OK and unpack(kind=kind, cols=0, y=None) == co3.OK
    assert pack(kind=2) == co3.ERR_INVALID_ARG and unpack(kind=-1) == co3.ERR_INVALID_ARG
    act = lambda x=AT, t=0, rows=8, cols=8, xs=8, act=1, y=AT, ys=8, y8=AT, x8=2 * AT, n=big: lib.co3_f8_activation(x, t, rows, cols, xs, act, y, ys, y8, x8, n, None)
    for bad in (dict(x=None), dict(act=4), dict(act=-1), dict(y=AT + 1), dict(ys=7), dict(y8=AT + 16), dict(x8=AT + 8), dict(x8=AT), dict(y=None, y8=None, x8=None)):
        assert act(**bad) == co3.ERR_INVALID_ARG, bad
    assert act(n=co3.co3_f8_bytes(8, 8) - 1) == co3.ERR_CAPACITY
    back = lambda dy=AT, t=0, rows=8, cols=8, ds=8, x8=AT, n=big, act=1, dx=AT, xs=8: lib.co3_f8_activation_backward(dy, t, rows, cols, ds, x8, n, act, dx, xs, None)
    for bad in (dict(dy=None), dict(dy=AT + 2), dict(ds=7), dict(act=4), dict(act=-1), dict(x8=None), dict(x8=AT + 64), dict(dx=None), dict(xs=7)):
        assert back(**bad) == co3.ERR_INVALID_ARG, bad
    assert back(n=100) == co3.ERR_CAPACITY


def test_linear_refusals(lib):
    big = 1 << 40

    def linear(x=AT, xt=0, xs=8, x8=AT, n8=big, w8=AT, nw=big, outs=8, ins=8, tr=0, bias=AT, y=AT, yt=0, ys=8, rows=8, res=AT):
        return lib.co3_f8_linear(x, xt, xs, x8, n8, w8, nw, outs, ins, tr, bias, y, yt, ys, rows, res, None)
    for tr in (0, 1):
        for bad in (dict(xt=3), dict(yt=-1), dict(x8=None), dict(x8=AT + 16), dict(w8=None), dict(w8=AT + 16), dict(y=None), dict(y=AT + 2), dict(ys=7),
                    dict(bias=AT + 2), dict(res=AT + 4), dict(rows=U31), dict(outs=U31), dict(xs=7), dict(x=AT + 1)):
            assert linear(tr=tr, **bad) == co3.ERR_INVALID_ARG, bad
        assert linear(tr=tr, n8=co3.co3_f8_bytes(8, 8) - 1) == co3.ERR_CAPACITY
        assert linear(tr=tr, nw=co3.co3_f8_bytes(8, 8, co3.F8_SQUARE) - 1) == co3.ERR_CAPACITY
        assert linear(tr=tr, rows=0) == co3.OK
    assert linear(ins=0) == co3.ERR_INVALID_ARG and linear(outs=0) == co3.OK
    assert linear(outs=0, tr=1) == co3.ERR_INVALID_ARG and linear(ins=0, tr=1) == co3.OK


def test_weight_gradient_refusals(lib):
    big = 1 << 40

    def grad(dy=AT, t=0, ds=8, x8=AT, n8=big, rows=8, outs=8, ins=8, dw=AT, db=AT, clients=2, stride=72, acc=0, ws=AT, nws=big, res=AT):
        return lib.co3_f8_weight_gradient(dy, t, ds, x8, n8, rows, outs, ins, dw, db, clients, stride, acc, ws, nws, res, None)
    for bad in (dict(dy=None), dict(dy=AT + 2), dict(t=3), dict(ds=7), dict(x8=None), dict(x8=AT + 16), dict(dw=AT + 2), dict(db=AT + 1), dict(clients=0),
                dict(stride=63), dict(stride=big), dict(ws=None), dict(ws=AT + 128), dict(res=AT + 4), dict(rows=U31 // 2), dict(outs=U31), dict(outs=1 << 20, ins=1 << 20)):
        assert grad(**bad) == co3.ERR_INVALID_ARG, bad
    assert grad(n8=100) == co3.ERR_CAPACITY and grad(nws=100) == co3.ERR_CAPACITY
    assert grad(outs=0) == co3.OK and grad(dw=None, db=None) == co3.OK and grad(rows=0, acc=1) == co3.OK


def test_binding_refuses_tensors_of_the_host():
    x, f8 = torch.zeros(4, 8), torch.zeros(1 << 15, dtype=torch.uint8)
    for call in (lambda: co3.co3_f8_pack(x, f8), lambda: co3.co3_f8_unpack(f8, x), lambda: co3.co3_f8_activation(x, co3.ACT_RELU, x),
                 lambda: co3.co3_f8_activation_backward(x, f8, co3.ACT_RELU, x), lambda: co3.co3_f8_linear(x, f8, f8, None, x),
                 lambda: co3.co3_f8_weight_gradient(x, f8, 8, x, None, 1, 64, f8)):
        with pytest.raises(ValueError):
            call()
