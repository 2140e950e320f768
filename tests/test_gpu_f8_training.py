"""A client's forward and backward pass through layer norm, linear layers on 8-bit blocks and an activation, as a session and the
example run them: every gradient against the formula in 64 bits on what the calls before it left, the whole captured into a
graph, and the session's refusals."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import values
from paper_2204_08211_b200.session import Co3Session

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "layer_norm_muon.py")
    spec = importlib.util.spec_from_file_location("layer_norm_muon_8", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_of_every_client(example):
    """Each step on the tensors that the steps before it left, so that no value next to a border of the format counts twice.
    fp32 sums of at most 256 terms: 2^-14 of the largest term's sum leaves room; layer norm's own gradients are tested elsewhere."""
    ex, task = example, example.Task(clients=3, rows=40, eight_bits=True)
    task.layer(task.params, ex.BIAS1).normal_(0, 0.1)
    task.layer(task.params, ex.BIAS2).normal_(0, 0.1)
    loss = task.passes()
    torch.cuda.synchronize()
    assert (task.sess.f8_result()["status"] == co3.OK).all()
    w1, w2 = (values(task.matrix(k), True) for k in (ex.W1, ex.W2))
    y1, y2, d, dx2 = (values(t) for t in (task.y1, task.y2, task.d, task.dx2))
    near = lambda got, want, size: ((got.double().cpu() - want).abs() <= 2.0 ** -14 * size.abs().max() + 0 * want).all()
    pre = y1 @ w1.T
    assert near(task.h, pre.clamp(min=0), pre)
    logits = y2 @ w2.T + task.layer(task.params, ex.B2).double().cpu()
    assert abs(loss.item() - torch.nn.functional.cross_entropy(logits, task.labels.cpu()).item()) <= 1e-4
    assert near(task.dy2, d @ w2, d @ w2) and near(task.dy1, dx2 @ w1, dx2 @ w1)
    assert ((task.dx2 != 0).cpu() <= (pre > -2.0 ** -14 * pre.abs().max())).all()          # nothing passes where the activation was off
    split = lambda t: t.double().cpu().view(3, 40, -1)
    for k, dy, x in ((ex.W2, split(task.d), split(y2)), (ex.W1, split(task.dx2), split(y1))):
        want, size = dy.transpose(1, 2) @ x, dy.abs().transpose(1, 2) @ x.abs()
        assert near(task.per_client(k), want, size)
    assert near(task.per_client(ex.B2), split(task.d).sum(1), split(task.d).abs().sum(1))


def test_close_to_the_32_bit_passes(example):
    """The same model in 32 bits: values of three bits behind the leading one are off by at most 2^-4 each, 2^-5.5 in the mean square, and a
    gradient passes through at most six of them one after the other or side by side: a quarter of a layer's norm is far outside."""
    tasks = [example.Task(clients=4, rows=64, eight_bits=e) for e in (False, True)]
    tasks[1].params.copy_(tasks[0].params)
    losses = [t.passes().item() for t in tasks]
    assert abs(losses[0] - losses[1]) <= 0.05 * abs(losses[0])
    for k in range(7):
        a, b = (t.per_client(k).double().flatten(1) for t in tasks)
        assert ((a - b).norm(dim=1) <= 0.25 * a.norm(dim=1) + 1e-9).all(), k


def test_rounds(example):
    """The rounds with compression and the server's step run, and no call reports an error."""
    task = example.Task(clients=4, rows=32, eight_bits=True)
    for _ in range(3):
        loss = task.round()
        task.check()
    assert torch.isfinite(loss)


@pytest.mark.parametrize("type_", [torch.float32, torch.bfloat16])
def test_two_layers_with_gelu_captured(type_):
    """linear - GELU straight into the next operand - linear, and back, captured and replayed on new inputs: the bits of the plain run."""
    clients, rows, ins, hidden, outs = 5, 100, 200, 520, 150
    n = clients * rows
    sess = Co3Session([hidden * ins, hidden, outs * hidden, outs], [(4, 3, 0, 1.0, 1.0)] * 4, clients, 0.9)
    gen = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    params = 0.1 * randn(sess.n_elem)
    f8 = sess.new_f8
    w1, w2 = f8(hidden, ins, co3.F8_SQUARE), f8(outs, hidden, co3.F8_SQUARE)
    x8, h8, a8, d8, e8 = f8(n, ins), f8(n, hidden), f8(n, hidden), f8(n, outs), f8(n, hidden)
    x, dy = randn(n, ins).to(type_), (0.01 * randn(n, outs)).to(type_)
    h, y, da, dx = (torch.empty(n, k, dtype=type_, device="cuda") for k in (hidden, outs, hidden, ins))
    grads = sess.new_client_buffer()
    ws = torch.empty(max(sess.new_linear_workspace(rows, o, i).numel() for o, i in ((hidden, ins), (outs, hidden))), dtype=torch.uint8, device="cuda")

    def step():
        sess.pack_weights(params, 0, (hidden, ins), w1)
        sess.pack_weights(params, 2, (outs, hidden), w2)
        sess.linear(x, x8, w1, params, 1, h)
        assert co3.co3_f8_activation(h, co3.ACT_GELU, None, a8, h8) == co3.OK
        sess.linear(None, a8, w2, params, 3, y, cols=hidden)
        sess.linear_backward(dy, d8, a8, w2, 2, 3, (outs, hidden), da, grads, ws)
        assert co3.co3_f8_activation_backward(da, h8, co3.ACT_GELU, da) == co3.OK
        sess.linear_backward(da, e8, x8, w1, 0, 1, (hidden, ins), dx, grads, ws)

    step()
    torch.cuda.synchronize()
    a, hv = torch.empty(n, hidden, device="cuda"), torch.empty(n, hidden, device="cuda")
    assert co3.co3_f8_unpack(a8, a) == co3.OK and co3.co3_f8_unpack(h8, hv) == co3.OK
    torch.cuda.synchronize()
    # y, and the gradients of both layers, on what the calls left
    want = a.double() @ values(params[hidden * ins + hidden:][:outs * hidden].view(outs, hidden), True).cuda().T + params[-outs:].double()
    assert (y.double() - want).abs().max() <= (2.0 ** -8 if type_ == torch.bfloat16 else 2.0 ** -14) * want.abs().max()
    for u in range(clients):
        r = slice(u * rows, (u + 1) * rows)
        g = sess.client_view(grads, u)
        at = np.cumsum([0, hidden * ins, hidden, outs * hidden, outs])
        xv = values(x[r]).cuda()
        for k, d, v in ((2, dy[r].double(), a[r].double()), (0, da[r].double(), xv)):
            want, size = d.T @ v, d.abs().T @ v.abs()
            assert ((g[at[k]:at[k + 1]].double().view(want.shape) - want).abs() <= 2.0 ** -16 * size).all()
            assert ((g[at[k + 1]:at[k + 2]].double() - d.sum(0)).abs() <= 2.0 ** -16 * d.abs().sum(0)).all()
    # the captured run
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(randn(n, ins))
    dy.copy_(0.01 * randn(n, outs))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (y, dx, grads)]
    for t in (y, dx, grads):
        t.zero_()
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(t, g) for t, g in zip((y, dx, grads), got))
    assert (sess.f8_result()["status"] == co3.OK).all()


def test_two_graphs_of_one_session_on_two_streams():
    """Graphs with their own workspaces and blocks do not disturb one another."""
    clients, rows, ins, outs = 2, 300, 400, 300
    sess = Co3Session([outs * ins, outs], [(4, 3, 0, 1.0, 1.0)] * 2, clients, 0.9)
    params = 0.1 * torch.randn(sess.n_elem, device="cuda")
    w8 = sess.new_f8(outs, ins, co3.F8_SQUARE)
    sess.pack_weights(params, 0, (outs, ins), w8)
    sides = []
    for k in range(2):
        n = clients * rows
        x, dy = torch.randn(n, ins, device="cuda"), torch.randn(n, outs, device="cuda")
        t = dict(x=x, dy=dy, x8=sess.new_f8(n, ins), d8=sess.new_f8(n, outs), y=torch.empty(n, outs, device="cuda"), dx=torch.empty(n, ins, device="cuda"),
                 grads=sess.new_client_buffer(), ws=sess.new_linear_workspace(rows, outs, ins))

        def step(t=t):
            sess.linear(t["x"], t["x8"], w8, params, 1, t["y"])
            sess.linear_backward(t["dy"], t["d8"], t["x8"], w8, 0, 1, (outs, ins), t["dx"], t["grads"], t["ws"])
        step()
        torch.cuda.synchronize()
        want = [t[k].clone() for k in ("y", "dx", "grads")]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        sides.append((t, want, g, torch.cuda.Stream()))
    for _ in range(20):
        for t, _, g, s in sides:
            with torch.cuda.stream(s):
                for k in ("y", "dx", "grads"):
                    t[k].zero_()
                g.replay()
        torch.cuda.synchronize()
        for t, want, _, _ in sides:
            assert all(torch.equal(t[k], w) for k, w in zip(("y", "dx", "grads"), want))


def test_session_refuses_layers_of_another_shape():
    sess = Co3Session([12, 3], [(4, 3, 0, 1.0, 1.0)] * 2, 1, 0.9)
    params, grads = torch.zeros(sess.n_elem, device="cuda"), sess.new_client_buffer()
    x, dy, y = torch.zeros(5, 4, device="cuda"), torch.zeros(5, 3, device="cuda"), torch.zeros(5, 3, device="cuda")
    x8, w8, ws = sess.new_f8(5, 4), sess.new_f8(3, 4, co3.F8_SQUARE), sess.new_linear_workspace(5, 3, 4)
    with pytest.raises(RuntimeError):
        sess.pack_weights(params, 1, (3, 5), w8)                               # no such view
    with pytest.raises(ValueError):
        sess.linear(x, x8, w8, params, 0, y)
    for weight, bias, shape in ((1, None, (3, 4)), (0, 0, (3, 4)), (0, 1, (4, 3)), (0, 1, (2, 6))):
        with pytest.raises(ValueError):
            sess.linear_backward(dy, None, x8, w8, weight, bias, shape, None, grads, ws)


FIRST_CALLS = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_2204_08211_b200 as co3
room = lambda r, c, k=co3.F8_ROWS: torch.empty(co3.co3_f8_bytes(r, c, k), dtype=torch.uint8, device="cuda")
cases = []
for rows, ins, outs in ((3, 300, 500), (200, 300, 500), (3000, 512, 2304)):
    x, dy, w = torch.randn(rows, ins, device="cuda"), torch.randn(rows, outs, device="cuda").bfloat16(), torch.randn(outs, ins, device="cuda")
    t = dict(x=x, dy=dy, w=w, x8=room(rows, ins), d8=room(rows, outs), w8=room(outs, ins, co3.F8_SQUARE), y=torch.empty(rows, outs, device="cuda"),
             dx=torch.empty(rows, ins, device="cuda"), g=torch.empty(outs * ins + outs, device="cuda"),
             ws=torch.empty(co3.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins), dtype=torch.uint8, device="cuda"))
    cases.append((ins, outs, t))

def run():
    for ins, outs, t in cases:
        assert co3.co3_f8_pack(t["w"], t["w8"], co3.F8_SQUARE) == co3.OK
        assert co3.co3_f8_linear(t["x"], t["x8"], t["w8"], None, t["y"]) == co3.OK
        assert co3.co3_f8_linear(t["dy"], t["d8"], t["w8"], None, t["dx"], True) == co3.OK
        assert co3.co3_f8_weight_gradient(t["dy"], t["x8"], ins, t["g"], t["g"][outs * ins:], 1, outs * ins + outs, t["ws"]) == co3.OK

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
graph.replay()
torch.cuda.synchronize()
kept = [[t[k].clone() for k in ("y", "dx", "g")] for _, _, t in cases]
run()
torch.cuda.synchronize()
for (_, _, t), want in zip(cases, kept):
    for k, v in zip(("y", "dx", "g"), want):
        assert torch.isfinite(v).all() and torch.equal(t[k], v), k
print("captured")
"""


def test_first_calls_of_a_process_can_be_captured():
    """What the calls ask the device for once (attributes, clusters at once, the driver's tensor maps) is allowed while a stream is captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", FIRST_CALLS, root], capture_output=True, text=True, timeout=120)
    assert p.returncode == 0 and "captured" in p.stdout, p.stderr[-2000:]
