"""examples/sage_training.py with layer norm and the AdamW step: its gradients against torch's own on the same blocks, and a step of everything by clipped
gradients against the formulas in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sage_training.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("sage_training", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(net, blocks, x, labels, params):
    """Loss of the same network in 64 bits by torch, hidden rows rounded to 8 bits as the identity's gradient."""
    weights, gains, shifts, classifier = params
    sizes = blocks.host_sizes()
    x = x[:sizes[0][1]]
    residual = None

    def norm(s, g, b):
        d = s - s.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * g + b

    for l, w in enumerate(weights):
        nd, ns, nnz, _ = sizes[l]
        s = x if residual is None else x + residual
        y = norm(s, gains[l], shifts[l])
        scale = (y.detach().abs().amax(1, keepdim=True) / 448.0).clamp(min=2.0 ** -126)
        q = (y.detach() / scale).float().to(net.type8).double() * scale
        values = y + (q - y).detach()
        ptr, idx = blocks.indptr[l][:nd + 1].long(), blocks.indices[l][:nnz].long()
        row = torch.repeat_interleave(torch.arange(nd, device="cuda"), ptr[1:] - ptr[:-1])
        mean = torch.zeros((nd, y.shape[1]), dtype=torch.float64, device="cuda").index_add(0, row, values[idx]) / (ptr[1:] - ptr[:-1]).clamp(min=1).unsqueeze(1)
        x, residual = torch.relu(torch.cat([y[:nd], mean], 1) @ w.t()), s[:nd]
    logits = norm(x + residual, gains[-1], shifts[-1]) @ classifier.t()
    return logits, torch.nn.functional.cross_entropy(logits, labels)


@pytest.mark.parametrize("optimiser", ["adamw", "adamw8"])
def test_gradients_and_a_step(example, optimiser):
    data = example.Data(nodes=4000, edges=60_000, dim=32, classes=5, batch=96, fanouts=(6, 4))
    net = example.Sage(data.ctx, data.dim, data.classes, 2, layer_norm=True, optimiser=optimiser)
    gen = torch.Generator().manual_seed(1)
    for t in net.gains + net.shifts:
        t.add_(0.2 * torch.randn(t.shape, generator=gen).cuda())
    x, blocks, labels = data.sample(3)
    logits, state = net.forward(blocks, x)
    grads = net.backward(blocks, (torch.softmax(logits, 1) - torch.nn.functional.one_hot(labels, data.classes)) / data.batch, state)
    leaf = lambda t: t.detach().double().requires_grad_()  # noqa: E731
    params = ([leaf(w) for w in net.weights], [leaf(g) for g in net.gains], [leaf(b) for b in net.shifts], leaf(net.classifier))
    x64 = leaf(x)
    want, loss = reference(net, blocks, x64, labels, params)
    loss.backward()

    # a value at the border of two 8-bit values may fall to either side: a sixteenth of a row's largest value at most, in one of ten thousand
    # or so; a neighbour's mean over a handful of rows passes it on, so that norms differ by 1e-3 at the very most
    def near(got, ref):
        assert float((got.double() - ref).norm()) <= 2e-3 * float(ref.norm()), float((got.double() - ref).norm() / ref.norm())
    near(logits, want.detach())
    near(grads["classifier"], params[3].grad)
    for l in range(2):
        near(grads["weights"][l], params[0][l].grad)
    for l in range(3):
        near(grads["gains"][l], params[1][l].grad)
        near(grads["shifts"][l], params[2][l].grad)
    ns = blocks.host_sizes()[0][1]
    near(grads["x"][:ns], x64.grad[:ns])
    assert bool((grads["x"][ns:] == 0).all())

    # the step, from these gradients: the first one, whose moments are (1 - beta) g and (1 - beta) g^2
    tensors = net.weights + net.gains + net.shifts + [net.classifier]
    all_grads = [g.double() for g in grads["weights"] + grads["gains"] + grads["shifts"] + [grads["classifier"]]]
    before = [t.double() for t in tensors]
    total = math.sqrt(sum(float((g * g).sum()) for g in all_grads))
    factor = min(1.0, 1.0 / total)
    net.step(grads, 0.02)
    torch.cuda.synchronize()
    for t, w, g, decay in zip(tensors, before, all_grads, [1.0] * 2 + [0.0] * 6 + [1.0]):
        g = g * factor
        ref = w * (1 - 0.02 * 0.01 * decay) - 0.02 * g / (g.abs() + 1e-8)
        # the weight's rounding and that of its kept part, and the step's: 20 roundings of a step of at most 0.02
        assert bool(((t.double() - ref).abs() <= 2.0 ** -24 * (2 * ref.abs() + 20 * 0.02)).all())


@pytest.mark.parametrize("optimiser", ["muon", "adamw", "adamw8"])
def test_it_trains(example, optimiser):
    losses = example.train(12, layer_norm=True, optimiser=optimiser)
    assert len(losses) == 12 and all(math.isfinite(x) for x in losses)
