"""The example that runs layer norm, compression and the orthogonalised step together."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3
from paper_2204_08211_b200.session import Co3Session

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "layer_norm_muon.py")
    spec = importlib.util.spec_from_file_location("layer_norm_muon", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def model(example, task, params):
    """The same model in 64 bits: one loss per client."""
    x = task.x.double()
    at = np.concatenate([[0], np.cumsum(task.sess.sizes)])
    w = [params[at[k]:at[k + 1]] if task.shapes[k] is None else params[at[k]:at[k + 1]].view(task.shapes[k]) for k in range(7)]
    h = torch.nn.functional.layer_norm(x, x.shape[1:], w[example.GAIN1], w[example.BIAS1], 1e-5) @ w[example.W1].T
    h = h.relu()
    h = torch.nn.functional.layer_norm(h, h.shape[1:], w[example.GAIN2], w[example.BIAS2], 1e-5) @ w[example.W2].T
    loss = torch.nn.functional.cross_entropy(h + w[example.B2], task.labels, reduction="none")
    return loss.view(task.clients, task.rows).mean(1)


def test_gradients_of_every_client(example):
    """Against automatic differentiation in 64 bits.  The passes are fp32 (matrix products with fp32 inputs, no reduced
    precision): a chain of two products and two norms, each with sums of at most 256 terms, is good to some 256 units of
    2^-24 of a layer's largest gradient; 2^-12 leaves room for rows whose spread is small against their mean."""
    task = example.Task(clients=3, rows=40)
    task.layer(task.params, example.BIAS1).normal_(0, 0.1)
    task.layer(task.params, example.BIAS2).normal_(0, 0.1)
    task.layer(task.params, example.GAIN2).normal_(1, 0.1)
    loss = task.passes()
    p = task.params.double().requires_grad_()
    want = model(example, task, p)
    assert abs(loss.item() - want.mean().item()) <= 1e-5
    for u in range(3):
        (g,) = torch.autograd.grad(want[u], p, retain_graph=True)
        got = task.sess.client_view(task.grads, u)
        for k in range(7):
            a, b = task.layer(got, k).double(), task.layer(g, k)
            assert (a - b).abs().max() <= 2.0 ** -12 * b.abs().max(), (u, k)


def test_one_round_is_the_chain_of_its_calls(example):
    """The average the server steps with, decoded again; the step against the formula in 64 bits."""
    task = example.Task(clients=4)
    before = task.params.clone()
    task.round(lr=0.02, weight_decay=0.01)
    torch.cuda.synchronize()
    task.check()
    avg = task.sess.avg.double().cpu()
    f = lambda v: float(np.float32(v))
    for k, shape in enumerate(task.shapes):
        at = sum(task.sess.sizes[:k])
        g = avg[at:at + task.sess.sizes[k]]
        u = g + f(0.95) * g                                    # the momentum starts at zero: buf = g
        if shape is not None:
            x = u.view(shape)
            x = x.T if shape[0] > shape[1] else x
            x = x / (x.norm() + 1e-7)
            for _ in range(5):
                s = x @ x.T
                x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
            u = (x.T if shape[0] > shape[1] else x).reshape(-1) * f(max(1.0, shape[0] / shape[1]) ** 0.5)
        old = task.layer(before, k).double().cpu()
        want = (1.0 - f(0.02) * f(0.01)) * old - f(0.02) * u
        assert (task.layer(task.params, k).double().cpu() - want).norm() <= 1e-5 * (f(0.02) * u).norm() + 2.0 ** -23 * old.norm()


def test_training_lowers_the_loss(example):
    task = example.Task()
    first = task.round().item()
    for _ in range(59):
        last = task.round()
    task.check()
    assert last.item() < 0.5 * first


def test_session_refuses_shapes_that_do_not_fit():
    sess = Co3Session([12, 5], [(4, 3, 0, 1.0, 1.0)] * 2, 1, 0.9)
    with pytest.raises(ValueError):
        sess.setup_muon([(5, 3), None])
    with pytest.raises(ValueError):
        sess.setup_muon([(4, 3)])
    x = torch.zeros(4, 12, device="cuda")
    with pytest.raises(ValueError):
        sess.layer_norm_backward(x, x, sess.avg, 0, 1, x, x, None, sess.new_client_buffer(), sess.workspace)
