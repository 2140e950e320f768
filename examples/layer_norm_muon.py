"""Rounds of federated training with layer norm at the clients and orthogonalised updates at the server.

Every client holds its own rows of a synthetic classification task (inputs of its own offset and spread, labels of one
hidden teacher).  The model, a parameter vector of seven layers:

    LN(gain, bias) -> W1 (hidden x inputs) -> ReLU -> LN(gain, bias) -> W2 (classes x hidden) -> + b2 -> cross entropy

One round: the clients' forward and backward passes (co3_layer_norm, co3_layer_norm_backward; the linear layers are
plain matrix products) write one gradient vector per client, co3_fit_scale and co3_model_weights fit this round's
formats and codes, co3_encode compresses with error memory, co3_decode_aggregate averages, co3_muon_update steps.

    python examples/layer_norm_muon.py [--rounds N] [--clients U] [--rows B]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import co3_inputs as ci                                                    # noqa: E402
import paper_2204_08211_b200 as co3                                        # noqa: E402
from paper_2204_08211_b200.session import Co3Session                       # noqa: E402

GAIN1, BIAS1, W1, GAIN2, BIAS2, W2, B2 = range(7)


class Task:
    """The data, the parameters and the clients' passes."""

    def __init__(self, clients=8, rows=64, inputs=96, hidden=160, classes=10, decay=0.9, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
        self.shapes = [None, None, (hidden, inputs), None, None, (classes, hidden), None]
        sizes = [inputs, inputs, hidden * inputs, hidden, hidden, classes * hidden, classes]
        self.sess = Co3Session(sizes, [(4, 3, 0, 1.0, 1.0)] * 7, clients, decay)
        self.sess.setup_muon(self.shapes)
        self.clients, self.rows = clients, rows

        clean = randn(clients, rows, inputs)
        self.labels = (clean.view(-1, inputs) @ randn(inputs, classes)).argmax(1)
        self.x = (clean * (0.5 + 2.0 * torch.rand(clients, 1, 1, device="cuda", generator=gen))
                  + 3.0 * randn(clients, 1, 1)).view(-1, inputs)
        self.params = torch.zeros(self.sess.n_elem, device="cuda")
        for k, scale in ((W1, inputs ** -0.5), (W2, hidden ** -0.5)):
            self.layer(self.params, k).copy_(randn(sizes[k]) * scale)
        for k in (GAIN1, GAIN2):
            self.layer(self.params, k).fill_(1.0)

        n = clients * rows
        self.y1, self.dy1 = (torch.empty(n, inputs, device="cuda") for _ in range(2))
        self.y2, self.dx2 = (torch.empty(n, hidden, device="cuda") for _ in range(2))
        self.stats = [torch.empty(n, device="cuda") for _ in range(4)]
        self.workspace = self.sess.new_layer_norm_workspace(rows, max(inputs, hidden))
        self.grads, self.mems = self.sess.new_client_buffer(), self.sess.new_client_buffer()
        log_tab, self.beta0, self.dbeta = ci.scale_log_table([(4, 3)])
        self.log_tab = torch.from_numpy(log_tab).cuda()
        self.fit = torch.empty(7, 4, dtype=torch.float64, device="cuda")

    def layer(self, vec, k):
        at = sum(self.sess.sizes[:k])
        return vec[at:at + self.sess.sizes[k]]

    def matrix(self, k):
        return self.layer(self.params, k).view(self.shapes[k])

    def per_client(self, k):
        """[clients][...] view of layer k of the gradient vectors."""
        at = sum(self.sess.sizes[:k])
        rows = self.grads.view(self.clients, self.sess.stride)[:, at:at + self.sess.sizes[k]]
        return rows if self.shapes[k] is None else rows.view(self.clients, *self.shapes[k])

    def passes(self):
        """Forward and backward pass of every client; returns the mean loss, leaves the gradients in self.grads."""
        s, (mean1, rstd1, mean2, rstd2) = self.sess, self.stats
        s.layer_norm(self.x, self.params, GAIN1, BIAS1, self.y1, mean1, rstd1)
        h = (self.y1 @ self.matrix(W1).T).relu_()
        s.layer_norm(h, self.params, GAIN2, BIAS2, self.y2, mean2, rstd2)
        logits = self.y2 @ self.matrix(W2).T + self.layer(self.params, B2)
        loss = torch.nn.functional.cross_entropy(logits, self.labels)

        split = lambda t: t.view(self.clients, self.rows, -1)
        d = torch.softmax(logits, 1)
        d[torch.arange(len(d), device="cuda"), self.labels] -= 1.0
        d /= self.rows                                        # every client's loss is the mean over its rows
        self.per_client(W2).copy_(split(d).transpose(1, 2) @ split(self.y2))
        self.per_client(B2).copy_(split(d).sum(1))
        s.layer_norm_backward(d @ self.matrix(W2), h, self.params, GAIN2, BIAS2, mean2, rstd2, self.dx2, self.grads,
                              self.workspace)
        d1 = self.dx2 * (h > 0)
        self.per_client(W1).copy_(split(d1).transpose(1, 2) @ split(self.y1))
        s.layer_norm_backward(d1 @ self.matrix(W1), self.x, self.params, GAIN1, BIAS1, mean1, rstd1, None, self.grads,
                              self.workspace)
        return loss

    def round(self, lr=0.02, weight_decay=0.0):
        loss = self.passes()
        s = self.sess
        s.fit_scales(self.grads, self.mems, self.log_tab, self.beta0, self.dbeta, stats_out=self.fit)
        s.set_codes_from_model_device(self.fit)
        s.encode(self.grads, self.mems)
        s.decode_aggregate()
        s.muon_update(self.params, lr, weight_decay)
        return loss

    def check(self):
        """Raises if any call of the last round reported an error (synchronises)."""
        for what, res in (("encode", self.sess.encode_results()), ("decode", self.sess.decode_result()),
                          ("update", self.sess.muon_result())):
            if (res["status"] != co3.OK).any():
                raise RuntimeError("%s: status %s" % (what, res["status"]))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--clients", type=int, default=8)
    ap.add_argument("--rows", type=int, default=64)
    a = ap.parse_args()
    task = Task(a.clients, a.rows)
    for t in range(a.rounds):
        loss = task.round()
        if t % 10 == 0 or t == a.rounds - 1:
            task.check()
            bits = task.sess.encode_results()["payload_bits"].sum() / (a.clients * task.sess.n_elem)
            print("round %3d  loss %.4f  %.2f bits per gradient element" % (t, loss.item(), bits))


if __name__ == "__main__":
    main()
