"""Recorded steps of a layer and the scratch that they were recorded with, on a context whose scratch is replaced by a larger one afterwards."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


def context(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


class Step:
    """The norm's backward and a step of weights that needs scratch, on buffers of its own."""

    def __init__(self, mqg, seed, rows, cols, n=3000, dim=96):
        gen = torch.Generator().manual_seed(seed)
        self.mqg = mqg
        self.grad, self.weight = (torch.randn((rows, cols), generator=gen).cuda() for _ in range(2))
        self.momentum = torch.zeros_like(self.grad)
        self.s, self.gy = (torch.randn((n, dim), generator=gen).cuda() for _ in range(2))
        self.gx, self.gw = torch.zeros_like(self.s), torch.zeros(dim, device="cuda")

    def __call__(self, ctx):
        self.mqg.mqg_rms_norm_backward(ctx, self.gy, self.s, None, self.gx, grad_weight=self.gw)
        self.mqg.mqg_muon_step(ctx, self.grad, self.momentum, self.weight, lr=0.05)

    def outputs(self):
        return self.gx, self.gw, self.momentum, self.weight


def test_replays_after_the_scratch_was_outgrown(mqg):
    ctx, eager = context(mqg), context(mqg)
    # scratch of each context: the first step's, then that of the second one, then a still larger one
    ctx.reserve_layer(norm_dim=96, num_mats=1, rows=256, cols=602)
    steps, twins, graphs = [], [], []
    side = torch.cuda.Stream()
    for seed, (rows, cols) in enumerate([(256, 602), (700, 1300)]):
        steps.append(Step(mqg, seed, rows, cols))
        twins.append(Step(mqg, seed, rows, cols))
        torch.cuda.synchronize()
        ctx.reserve_layer(norm_dim=96, num_mats=1, rows=rows, cols=cols)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            steps[-1](ctx)
    big = torch.randn((3, 1100, 1500), device="cuda")
    for k in range(4):
        mqg.mqg_orthogonalize(ctx, big, torch.empty_like(big))          # eager on the same context: larger scratch, then the same again
        room = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]    # whoever took freed memory would read this
        torch.cuda.synchronize()
        for step, twin, graph in zip(steps, twins, graphs):
            for t in (step, twin):
                t.grad.add_(0.1 * k)
                t.s.add_(0.05 * k)
            graph.replay()
            twin(eager)
            torch.cuda.synchronize()
            for got, want in zip(step.outputs(), twin.outputs()):
                assert torch.equal(got, want), k
        del room


def test_what_is_kept_and_what_is_given_back(mqg):
    gib = 12 * 8192 * 8192 + 8 * 8192 * 8192                            # scratch of one matrix of 8,192 x 8,192
    for recorded in (False, True):
        ctx = context(mqg)
        step = Step(mqg, 1, 256, 602)
        ctx.reserve_layer(norm_dim=96, num_mats=1, rows=8192, cols=8192)
        if recorded:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                step(ctx)
        else:
            step(ctx)
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        ctx.reserve_layer(num_mats=2, rows=8192, cols=8192)
        used = before - torch.cuda.mem_get_info()[0]
        want = gib * (2 if recorded else 1)
        assert abs(used - want) < (64 << 20), (recorded, used, want)
        del ctx
        torch.cuda.synchronize()


def test_the_products_refuse_to_allocate_while_recorded(mqg):
    ctx = context(mqg)
    step = Step(mqg, 2, 256, 602)
    out = torch.empty_like(step.grad)
    torch.cuda.synchronize()
    for call in (lambda: mqg.mqg_orthogonalize(ctx, step.grad, out), lambda: mqg.mqg_muon_step(ctx, step.grad, step.momentum, step.weight, lr=0.1)):
        with pytest.raises(mqg.MqgError) as refused:
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=torch.cuda.Stream()):
                call()
        assert refused.value.code == mqg.MQG_ERR_UNSUPPORTED and "mqg_ctx_reserve_layer" in str(refused.value)
        torch.cuda.synchronize()


def test_reserving_more_waits_for_steps_on_another_stream(mqg):
    """A step that is still on its way on a stream of its own (which the default stream does not wait for) when its scratch is replaced."""
    ctx, eager = context(mqg), context(mqg)
    step, twin = Step(mqg, 3, 1100, 1500), Step(mqg, 3, 1100, 1500)
    twin(eager)
    ctx.reserve_layer(norm_dim=96, num_mats=1, rows=1100, cols=1500)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    done = torch.cuda.Event()
    with torch.cuda.stream(side):
        for _ in range(3):                                 # (other work before it, so that it is on its way for a while)
            mqg.mqg_orthogonalize(ctx, step.grad, torch.empty_like(step.grad))
        step(ctx)
        done.record()
    ctx.reserve_layer(num_mats=2, rows=1100, cols=1500)
    assert done.query()                                    # nothing that had the old scratch is left
    torch.cuda.synchronize()
    for got, want in zip(step.outputs(), twin.outputs()):
        assert torch.equal(got, want)


def test_matrices_of_one_workgroup_need_no_scratch(mqg):
    """Nothing is set aside for them, and nothing has to be: their steps are recorded on a context without scratch."""
    ctx = context(mqg)
    torch.cuda.synchronize()
    for rows, cols in ((32, 512), (512, 32), (64, 256), (96, 160), (160, 96), (1, 1)):
        before = torch.cuda.mem_get_info()[0]
        ctx.reserve_layer(num_mats=65_535, rows=rows, cols=cols)
        assert before - torch.cuda.mem_get_info()[0] < (8 << 20)
        gen = torch.Generator().manual_seed(rows)
        grad, weight = (torch.randn((2, rows, cols), generator=gen).cuda() for _ in range(2))
        momentum, eager = torch.zeros_like(weight), (torch.zeros_like(weight), weight.clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            mqg.mqg_muon_step(ctx, grad, momentum, weight, lr=0.1)
        for k in range(3):
            graph.replay()
            mqg.mqg_muon_step(ctx, grad, *eager, lr=0.1)
            torch.cuda.synchronize()
            assert torch.equal(weight, eager[1]) and torch.equal(momentum, eager[0]), k
    # the next larger ones do
    for rows, cols in ((33, 512), (64, 257), (96, 161), (97, 97)):
        other = context(mqg)
        grad = torch.randn((rows, cols), device="cuda")
        out = torch.empty_like(grad)
        torch.cuda.synchronize()
        with pytest.raises(mqg.MqgError):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=torch.cuda.Stream()):
                mqg.mqg_orthogonalize(other, grad, out)
        torch.cuda.synchronize()
        other.reserve_layer(num_mats=1, rows=rows, cols=cols)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            mqg.mqg_orthogonalize(other, grad, out)
        want = torch.empty_like(grad)
        mqg.mqg_orthogonalize(ctx, grad, want)
        for _ in range(2):
            out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        del graph
