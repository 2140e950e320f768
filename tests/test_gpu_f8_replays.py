"""Replays of a captured product one by one, forks and joins of streams, and values of the activation beyond 32-bit offsets."""
import math

import pytest
import torch

import paper_2204_08211_b200 as co3
from test_gpu_f8_blocks import room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 200, 3000])
@pytest.mark.parametrize("transposed", [False, True])
def test_each_replay_has_the_bits_of_a_call(rows, transposed):
    """A captured product, replayed on inputs that change from replay to replay."""
    ins, outs = 500, 1700
    cols, to = (outs, ins) if transposed else (ins, outs)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    new = lambda: torch.randn(rows, cols, generator=gen, device="cuda")
    x, b = new(), torch.randn(to, generator=gen, device="cuda")
    w8 = torch.empty(co3.co3_f8_bytes(outs, ins, co3.F8_SQUARE), dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_pack(torch.randn(outs, ins, generator=gen, device="cuda"), w8, co3.F8_SQUARE) == co3.OK
    x8, z8 = room(rows, cols), room(rows, cols)
    y, z = torch.empty(rows, to, device="cuda"), torch.empty(rows, to, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert co3.co3_f8_linear(x, x8, w8, b, y, transposed) == co3.OK
    last = torch.zeros_like(y)
    for _ in range(3):
        x.copy_(new())
        y.fill_(math.nan)
        z.fill_(math.nan)
        graph.replay()
        assert co3.co3_f8_linear(x, z8, w8, b, z, transposed) == co3.OK
        torch.cuda.synchronize()
        assert torch.isfinite(y).all() and torch.equal(y, z) and not torch.equal(y, last)
        u, v = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
        assert co3.co3_f8_unpack(x8, u) == co3.OK and co3.co3_f8_unpack(z8, v) == co3.OK
        torch.cuda.synchronize()
        assert torch.equal(u, v)
        last.copy_(y)


def test_activation_beyond_32_bit_offsets():
    """The first and last rows of a long matrix, forward and backward in place, against the definition and the same rows alone."""
    rows, cols, tail = 70000, 65536, 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    ends = (slice(0, tail), slice(rows - tail, rows))
    for e in ends:
        x[e] = torch.randn(tail, cols, generator=gen, device="cuda").bfloat16()
    kept = [x[e].clone() for e in ends]
    x8, t8 = torch.empty(co3.co3_f8_bytes(rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(co3.co3_f8_bytes(tail, cols), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)
    assert x8.numel() > 1 << 32 and x.numel() > 1 << 32
    assert co3.co3_f8_activation(x, co3.ACT_RELU, y, None, x8) == co3.OK
    assert co3.co3_f8_activation_backward(x, x8, co3.ACT_RELU, x) == co3.OK         # the gradient: x itself, in place
    torch.cuda.synchronize()
    for e, k in zip(ends, kept):
        assert torch.equal(y[e], k.clamp(min=0))
        # what 8 bits round to zero lets nothing through
        v, dx = torch.empty(tail, cols, device="cuda"), torch.empty_like(k)
        assert co3.co3_f8_pack(k, t8) == co3.OK and co3.co3_f8_unpack(t8, v) == co3.OK
        assert co3.co3_f8_activation_backward(k, t8, co3.ACT_RELU, dx) == co3.OK
        torch.cuda.synchronize()
        assert torch.equal(x[e], torch.where(v > 0, k, torch.zeros_like(k))) and torch.equal(x[e], dx)
        assert (x[e] > 0).float().mean() > 0.4
    assert (y[tail:-tail] == 0).all() and (x[tail:-tail] == 0).all()


@pytest.mark.parametrize("rows", [4, 300, 3000])
def test_forks_and_joins(rows):
    """Weights packed on one stream, the product on another that waits for it, the weight gradient on the first again: plain and captured."""
    ins, outs = 512, 1024
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, w, dy = (torch.randn(*s, generator=gen, device="cuda") for s in ((rows, ins), (outs, ins), (rows, outs)))
    x2, w2, dy2 = (torch.empty_like(t) for t in (x, w, dy))
    x8, w8 = (torch.empty(co3.co3_f8_bytes(*s), dtype=torch.uint8, device="cuda") for s in ((rows, ins), (outs, ins, co3.F8_SQUARE)))
    y, g = torch.empty(rows, outs, device="cuda"), torch.zeros(outs * ins + outs, device="cuda")
    ws = torch.empty(co3.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            w2.copy_(w * 2)
            assert co3.co3_f8_pack(w2, w8, co3.F8_SQUARE) == co3.OK
            dy2.copy_(dy)
        x2.copy_(x)
        main.wait_stream(side)
        assert co3.co3_f8_linear(x2, x8, w8, None, y) == co3.OK
        side.wait_stream(main)
        with torch.cuda.stream(side):
            assert co3.co3_f8_weight_gradient(dy2, x8, ins, g, g[outs * ins:], 1, 0, ws) == co3.OK
        main.wait_stream(side)

    # one after the other on one stream
    assert co3.co3_f8_pack(w * 2, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, None, y) == co3.OK
    assert co3.co3_f8_weight_gradient(dy, x8, ins, g, g[outs * ins:], 1, 0, ws) == co3.OK
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, g)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for run in (graph.replay, step) * 10:
        for t in (y, g, w8, x8):
            t.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(g, want[1])
