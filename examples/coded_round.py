"""Data-parallel training of a two-layer network with the whole round on the library's operators:

  master   codes the weights in 8 bits, one scale for each output channel (the broadcast of Algorithm 1);
  workers  multiply with the codes, forwards and backwards; each one's weight gradients are a row of `grad`;
  round    error feedback, top-r, k-of-r messages and their average, per tensor (RTopK.step_segmented);
  master   momentum and the orthogonal update of each weight matrix, straight from the dense average.

The data are synthetic: every worker draws inputs, a fixed teacher network gives the targets.

  python examples/coded_round.py [--rounds 60] [--workers 4]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_10761_b200 as rt  # noqa: E402


class Network:
    """Two weight matrices as views of one flat vector, so that a gradient row and the average match it."""

    def __init__(self, n_in, n_hidden, n_out, gen):
        self.shapes = [(n_hidden, n_in), (n_out, n_hidden)]
        sizes = [a * b for a, b in self.shapes]
        self.offsets = [0, sizes[0], sizes[0] + sizes[1]]
        self.d = self.offsets[-1]
        self.flat = torch.empty(self.d, device="cuda")
        for w in self.views(self.flat):
            w.copy_(torch.randn(w.shape, generator=gen, device="cuda") / math.sqrt(w.shape[1]))

    def views(self, flat):
        return [flat[o:o + a * b].view(a, b) for o, (a, b) in zip(self.offsets, self.shapes)]


def train(rounds=60, workers=4, tokens=256, n_in=192, n_hidden=320, n_out=160, density=0.05, eta=0.02, mu=0.9, seed=0):
    """The mean loss over the workers of every round."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = [torch.randn(s, generator=gen, device="cuda") / math.sqrt(s[1]) for s in ((n_hidden, n_in), (n_out, n_hidden))]
    net = Network(n_in, n_hidden, n_out, gen)
    weights = net.views(net.flat)
    velocity = torch.zeros(net.d, device="cuda")

    ld = -(-net.d // 8) * 8
    grad = torch.zeros((workers, ld), device="cuda")
    residual = torch.zeros((workers, ld), device="cuda")
    average = torch.zeros(ld, device="cuda")
    seg_k = [max(1, int(density * a * b / workers)) for a, b in net.shapes]
    seg_r = [workers * k for k in seg_k]                  # k / r = 1 / n
    msg_idx = torch.zeros((workers, sum(seg_k)), dtype=torch.int32, device="cuda")
    msg_val = torch.zeros((workers, sum(seg_k)), device="cuda")

    exchange = rt.RTopK(d_max=net.d, W_max=workers, r_max=sum(seg_r), k_max=sum(seg_k), segments_max=2)
    matrices = rt.MatrixContext(max([rt.orthogonalize_scratch(1, a, b) for a, b in net.shapes] +
                                    [rt.coded_scratch(tokens, a, b) for a, b in net.shapes]))
    coded = [rt.CodedWeights(a, b, transposed=i > 0) for i, (a, b) in enumerate(net.shapes)]
    losses = []
    for t in range(rounds):
        for w, c in zip(weights, coded):
            matrices.code_weights(w, c)
        loss = torch.zeros((), device="cuda")
        for i in range(workers):
            x = torch.randn((tokens, n_in), generator=gen, device="cuda")
            target = torch.relu(x @ teacher[0].t()) @ teacher[1].t()
            pre, y = torch.empty((tokens, n_hidden), device="cuda"), torch.empty((tokens, n_out), device="cuda")
            matrices.coded_product(x, coded[0], pre)
            h = torch.relu(pre)
            matrices.coded_product(h, coded[1], y)
            loss += (y - target).square().mean() / workers
            dy = (y - target) * (2.0 / y.numel())
            dw = net.views(grad[i])
            dh = torch.empty_like(h)
            matrices.coded_gradients(dy, h, coded[1], dh, dw[1])
            matrices.coded_gradients(dh * (pre > 0), x, coded[0], dw=dw[0])
        exchange.step_segmented(grad, residual, net.d, net.offsets, seg_r, seg_k, seed, t, msg_idx, msg_val, average)
        for g, v, w in zip(net.views(average), net.views(velocity), weights):
            matrices.orthogonal_update(g, v, w, eta, mu, scale=math.sqrt(max(1.0, w.shape[0] / w.shape[1])))
        losses.append(loss)
    exchange.poll_status()
    matrices.poll_status()
    exchange.close()
    matrices.close()
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    for t, v in enumerate(train(a.rounds, a.workers)):
        if t % 10 == 0 or t + 1 == a.rounds:
            print(f"round {t:4d}  loss {v:.4f}")
