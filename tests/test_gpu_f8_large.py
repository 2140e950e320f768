"""8-bit blocks beyond 32-bit offsets: more than 2^32 bytes and 2^31 elements in one buffer, looked at in pieces."""
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu


def pieces(rows, cols, gen):
    return torch.randn(rows, cols, generator=gen, device="cuda", dtype=torch.float32).bfloat16()


def test_blocks_and_products():
    """The last rows of a long matrix are packed, unpacked, multiplied and activated like the same rows alone."""
    rows, cols, outs, tail = 70000, 65536, 200, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-tail:] = pieces(tail, cols, gen)
    x[:tail] = pieces(tail, cols, gen)
    w = torch.randn(outs, cols, generator=gen, device="cuda") / 256
    w8 = torch.empty(co3.co3_f8_bytes(outs, cols, co3.F8_SQUARE), dtype=torch.uint8, device="cuda")
    x8 = torch.empty(co3.co3_f8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    assert x8.numel() > 1 << 32 and x.numel() > 1 << 32
    y = torch.empty(rows, outs, device="cuda")
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, None, y) == co3.OK
    back = torch.empty_like(x)
    assert co3.co3_f8_unpack(x8, back) == co3.OK
    torch.cuda.synchronize()
    t8 = torch.empty(co3.co3_f8_bytes(tail, cols), dtype=torch.uint8, device="cuda")
    wv = torch.empty(outs, cols, device="cuda")
    assert co3.co3_f8_unpack(w8, wv, co3.F8_SQUARE) == co3.OK
    for where in (slice(0, tail), slice(rows - tail, rows)):
        t, v = x[where].clone(), torch.empty(tail, cols, dtype=torch.bfloat16, device="cuda")
        assert co3.co3_f8_pack(t, t8) == co3.OK and co3.co3_f8_unpack(t8, v) == co3.OK
        torch.cuda.synchronize()
        assert torch.equal(back[where], v)
        want, size = v.double() @ wv.double().T, v.double().abs() @ wv.double().abs().T
        assert ((y[where].double() - want).abs() <= (cols / 32 + 2) * 2.0 ** -19.9 * size).all()     # as for the smaller products
    assert (y[tail:-tail] == 0).all() and (back[tail:-tail] == 0).all()
    assert co3.co3_f8_activation(x, co3.ACT_RELU, back, None, x8) == co3.OK
    dx = x  # in place: the gradient of ones times x
    assert co3.co3_f8_activation_backward(dx, x8, co3.ACT_RELU, dx) == co3.OK
    torch.cuda.synchronize()
    assert (back[-tail:] >= 0).all() and torch.equal(dx[-tail:] != 0, (back[-tail:] != 0) & (dx[-tail:] != 0))


def test_weight_gradient():
    """A gradient of 1.2e9 entries for the second of two clients lies beyond 2^32 bytes."""
    clients, rows, outs, ins = 2, 40, 40000, 30000
    gen = torch.Generator(device="cuda").manual_seed(2)
    dy = pieces(clients * rows, outs, gen)
    x = torch.randn(clients * rows, ins, generator=gen, device="cuda")
    x8, v = torch.empty(co3.co3_f8_bytes(clients * rows, ins), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    assert co3.co3_f8_pack(x, x8) == co3.OK and co3.co3_f8_unpack(x8, v) == co3.OK
    stride = outs * ins + outs
    grads = torch.full((clients * stride,), 7.0, device="cuda")
    ws = torch.empty(co3.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, clients), dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, grads, grads[outs * ins:], clients, stride, ws) == co3.OK
    torch.cuda.synchronize()
    for u in range(clients):
        d, xv = dy[u * rows:(u + 1) * rows].double(), v[u * rows:(u + 1) * rows].double()
        for o in (slice(0, 130), slice(outs - 130, outs)):
            got = grads[u * stride:u * stride + outs * ins].view(outs, ins)[o].double()
            want, size = d[:, o].T @ xv, d[:, o].abs().T @ xv.abs()
            assert ((got - want).abs() <= (rows / 16 + 3) * 2.0 ** -20.8 * size + 2.0 ** -140).all()
        got = grads[u * stride + outs * ins:(u + 1) * stride].double()
        assert ((got - d.sum(0)).abs() <= (rows + 3) * 2.0 ** -24 * d.abs().sum(0)).all()
