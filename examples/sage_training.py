"""Training a GraphSAGE network with pre-norm residual layers on sampled mini-batches, start to end on one GPU.

    python examples/sage_training.py [--steps 60] [--int8]

Every layer l takes the residual stream of its block's source rows and gives that of its destinations:

    s = x + r                      x: the layer's input, r: the stream so far          mqg_rms_norm
    y = s / rms(s) * g             and y in 8 bits, one scale per row
    a = mean of the neighbours' y  read from the 8-bit rows                            mqg_sage_mean_aggregate_q8
    z = relu([y | a] W^T)          the next layer's x; its r is s of the destinations  (torch)

and the logits are norm(s) C^T.  The backward goes the same way back (the rounding to 8 bits is taken as the identity):
mqg_sage_mean_aggregate_backward for a, mqg_rms_norm_backward for y and the stream; W takes a step by its momentum's orthogonal
factor (mqg_muon_step).  Sampling and the features' gather are the library's, too.  Nothing on the way waits for the host:
the rows of a mini-batch are counted on the device, and what lies past them is zero.

The graph, the features and the labels (a fixed linear function of a node's features and its neighbours' mean) are made up.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_04707_amd import mqg, synth  # noqa: E402


class Sage:
    def __init__(self, ctx, dim, classes, layers, type8=torch.float8_e4m3fn, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ctx, self.dim, self.type8 = ctx, dim, type8
        self.weights = [torch.randn((dim, 2 * dim), generator=gen, device="cuda") / (2 * dim) ** 0.5 for _ in range(layers)]
        self.momenta = [torch.zeros_like(w) for w in self.weights]
        self.gains = [torch.ones(dim, device="cuda") for _ in range(layers + 1)]
        self.classifier = torch.randn((classes, dim), generator=gen, device="cuda") / dim ** 0.5
        ctx.reserve_layer(norm_dim=dim, num_mats=1, rows=dim, cols=2 * dim)

    def _norm(self, layer, x, residual, num_rows, quantised):
        s, y = torch.zeros_like(x), torch.zeros_like(x)
        q = torch.zeros(x.shape, dtype=self.type8, device="cuda") if quantised else None
        scale = torch.zeros((x.shape[0], 1), device="cuda") if quantised else None
        mqg.mqg_rms_norm(self.ctx, x, self.gains[layer], residual=residual, sum_out=s, y=y, q=q, q_scale=scale, num_rows=num_rows)
        return s, y, q, scale

    def forward(self, blocks, x):
        """x: [cap_src of block 0, dim].  Returns the logits of the seeds and what the backward reads."""
        kept, residual = [], None
        for l, w in enumerate(self.weights):
            rows = blocks.bounds[l][0]
            s, y, q, scale = self._norm(l, x, residual, blocks.sizes[l, 1:2], True)
            both = torch.zeros((rows, 2 * self.dim), device="cuda")
            both[:, :self.dim] = y[:rows]
            both[:, self.dim:] = self._mean(blocks, l, q, scale, rows)
            both *= self._live(blocks, l, rows)
            z = torch.relu(both @ w.t())
            kept.append((s, both, z))
            x, residual = z, s[:rows]
        s, y, _, _ = self._norm(len(self.weights), x, residual, blocks.sizes[-1, 0:1], False)
        return y @ self.classifier.t(), (kept, s, y)

    def _mean(self, blocks, l, q, scale, rows):
        out = torch.zeros((rows, self.dim), device="cuda")
        mqg.mqg_sage_mean_aggregate_q8(self.ctx, blocks, l, q, scale, out)
        return out

    @staticmethod
    def _live(blocks, l, rows):
        """1 for the block's destinations, 0 for the rows past them (they hold the sources that follow)."""
        return (torch.arange(rows, device="cuda") < blocks.sizes[l, 0]).unsqueeze(1)

    def backward(self, blocks, grad_logits, state):
        """Gradients: {"weights": [...], "gains": [...], "classifier": ..., "x": of the input rows}."""
        kept, s, y = state
        grads = {"weights": [None] * len(self.weights), "gains": [torch.zeros_like(g) for g in self.gains], "classifier": grad_logits.t() @ y}
        stream = torch.zeros_like(s)
        mqg.mqg_rms_norm_backward(self.ctx, grad_logits @ self.classifier, s, self.gains[-1], stream, grad_weight=grads["gains"][-1],
                                  num_rows=blocks.sizes[-1, 0:1])
        for l in reversed(range(len(self.weights))):
            s, both, z = kept[l]
            rows = blocks.bounds[l][0]
            grad_z = stream * (z > 0)
            grads["weights"][l] = grad_z.t() @ both
            grad_both = grad_z @ self.weights[l]
            grad_y, grad_s, grad_x = torch.zeros_like(s), torch.zeros_like(s), torch.zeros_like(s)
            mqg.mqg_sage_mean_aggregate_backward(self.ctx, blocks, l, grad_both[:, self.dim:], grad_y)
            grad_y[:rows] += grad_both[:, :self.dim]
            grad_s[:rows] = stream
            mqg.mqg_rms_norm_backward(self.ctx, grad_y, s, self.gains[l], grad_x, grad_weight=grads["gains"][l], grad_sum=grad_s,
                                      num_rows=blocks.sizes[l, 1:2])
            stream = grad_x
        grads["x"] = stream
        return grads

    def step(self, grads, lr):
        for w, m, g in zip(self.weights, self.momenta, grads["weights"]):
            mqg.mqg_muon_step(self.ctx, g, m, w, lr=lr, weight_decay=0.01)
        for gain, g in zip(self.gains, grads["gains"]):
            gain -= lr * g
        self.classifier -= 10 * lr * grads["classifier"]


class Data:
    """A power-law graph, features and labels; mini-batches of it as input rows, blocks and labels."""

    def __init__(self, nodes=20_000, edges=300_000, dim=64, classes=8, batch=512, fanouts=(8, 5), seed=0):
        rp, ci = synth.chung_lu_graph(nodes, edges, seed=seed, max_degree=600)
        self.feats = synth.node_features(nodes, dim, seed=seed + 1)
        gen = torch.Generator().manual_seed(seed + 2)
        count = (rp[1:] - rp[:-1]).clamp(min=1).unsqueeze(1)
        sums = torch.zeros_like(self.feats).index_add_(0, torch.repeat_interleave(torch.arange(nodes), rp[1:] - rp[:-1]), self.feats[ci.long()])
        self.labels = (self.feats @ torch.randn((dim, classes), generator=gen) + sums / count @ torch.randn((dim, classes), generator=gen)).argmax(1).cuda()
        self.graph = mqg.Graph(rp.cuda(), ci.cuda())
        self.batch, self.fanouts, self.dim, self.classes = batch, list(fanouts), dim, classes
        self.ctx = mqg.Context(self.graph, batch, self.fanouts)
        self.blocks = mqg.Blocks(self.graph, batch, self.fanouts)
        self.cache = mqg.Cache(self.graph, self.feats.pin_memory(), nodes // 5)
        mqg.mqg_build_cache(self.ctx, self.graph, self.cache)
        self.seeds = [s.cuda() for s in synth.seed_batches(nodes, batch, nodes // batch, seed=seed + 3, dtype=ci.dtype)]

    def sample(self, k):
        seeds = self.seeds[k % len(self.seeds)]
        mqg.mqg_sample_blocks(self.ctx, self.graph, seeds, self.fanouts, k, self.blocks)
        x = torch.zeros((self.blocks.bounds[0][1], self.dim), device="cuda")
        mqg.mqg_gather_features(self.ctx, self.cache, self.blocks.src_ids[0], self.blocks.sizes[0, 1:2], x)
        return x, self.blocks, self.labels[seeds.long()]


def train(steps, type8=torch.float8_e4m3fn, lr=0.02, tell=None):
    """Losses of the steps."""
    data = Data()
    net = Sage(data.ctx, data.dim, data.classes, len(data.fanouts), type8)
    losses = []
    for k in range(steps):
        x, blocks, labels = data.sample(k)
        logits, state = net.forward(blocks, x)
        chance = torch.softmax(logits, 1)
        losses.append(-torch.log(chance.gather(1, labels.unsqueeze(1))).mean())
        grad = (chance - torch.nn.functional.one_hot(labels, data.classes)) / data.batch
        net.step(net.backward(blocks, grad, state), lr)
        if tell and k % 10 == 9:
            tell(k + 1, float(losses[-1]))
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--int8", action="store_true", help="hidden rows in int8 instead of e4m3")
    args = ap.parse_args()
    began = time.perf_counter()
    train(args.steps, torch.int8 if args.int8 else torch.float8_e4m3fn, tell=lambda k, loss: print(f"step {k}: loss {loss:.4f}", flush=True))
    print(f"{args.steps} steps in {time.perf_counter() - began:.1f} s, the graph's making included")
