"""The calls of a layer together, as examples/sage_training.py has them: gradients against torch's own on the same blocks, and a loss that falls."""
import importlib.util
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


def reference(net, blocks, x, labels, classes, params):
    """Loss of the same network in 64 bits by torch, hidden rows rounded to 8 bits as the identity's gradient."""
    weights, gains, classifier = params
    sizes = blocks.host_sizes()
    x = x[:sizes[0][1]]
    residual = None
    top = 127.0 if net.type8 == torch.int8 else 448.0

    def norm(s, g):
        return s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6) * g

    for l, w in enumerate(weights):
        nd, ns, nnz, _ = sizes[l]
        s = x if residual is None else x + residual
        y = norm(s, gains[l])
        scale = (y.detach().abs().amax(1, keepdim=True) / top).clamp(min=2.0 ** -126)
        q = (y.detach() / scale).float()
        q = (q.round() if net.type8 == torch.int8 else q.to(net.type8)).double() * scale
        values = y + (q - y).detach()
        ptr, idx = blocks.indptr[l][:nd + 1].long(), blocks.indices[l][:nnz].long()
        row = torch.repeat_interleave(torch.arange(nd, device="cuda"), ptr[1:] - ptr[:-1])
        mean = torch.zeros((nd, y.shape[1]), dtype=torch.float64, device="cuda").index_add(0, row, values[idx]) / (ptr[1:] - ptr[:-1]).clamp(min=1).unsqueeze(1)
        x, residual = torch.relu(torch.cat([y[:nd], mean], 1) @ w.t()), s[:nd]
    logits = norm(x + residual, gains[-1]) @ classifier.t()
    return logits, torch.nn.functional.cross_entropy(logits, labels)


@pytest.mark.parametrize("type8", [torch.float8_e4m3fn, torch.int8])
def test_gradients_of_a_step(example, type8):
    data = example.Data(nodes=4000, edges=60_000, dim=32, classes=5, batch=96, fanouts=(6, 4))
    net = example.Sage(data.ctx, data.dim, data.classes, 2, type8)
    x, blocks, labels = data.sample(3)
    logits, state = net.forward(blocks, x)
    grads = net.backward(blocks, (torch.softmax(logits, 1) - torch.nn.functional.one_hot(labels, data.classes)) / data.batch, state)
    leaf = lambda t: t.detach().double().requires_grad_()  # noqa: E731
    params = ([leaf(w) for w in net.weights], [leaf(g) for g in net.gains], leaf(net.classifier))
    x64 = leaf(x)
    want, loss = reference(net, blocks, x64, labels, data.classes, params)
    loss.backward()
    # a value at the border of two 8-bit values may fall to either side: a sixteenth (e4m3) or a 127th of a row's largest value, in one of
    # ten thousand or so; a neighbour's mean over a handful of rows passes it on, so that norms differ by 1e-3 at the very most
    def near(got, ref):
        assert float((got.double() - ref).norm()) <= 2e-3 * float(ref.norm()), float((got.double() - ref).norm() / ref.norm())
    near(logits, want.detach())
    near(grads["classifier"], params[2].grad)
    for l in range(2):
        near(grads["weights"][l], params[0][l].grad)
    for l in range(3):
        near(grads["gains"][l], params[1][l].grad)
    ns = blocks.host_sizes()[0][1]
    near(grads["x"][:ns], x64.grad[:ns])
    assert bool((grads["x"][ns:] == 0).all())


def test_the_loss_falls(example):
    losses = example.train(60)
    assert all(x == x for x in losses)
    assert sum(losses[:5]) / 5 > 1.5 and sum(losses[-5:]) / 5 < 0.75 * sum(losses[:5]) / 5
