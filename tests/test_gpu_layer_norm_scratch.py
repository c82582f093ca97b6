"""What mqg_ctx_reserve_layer takes for the norms' backward: no more than the header says, and enough for every call of up to that many columns while a stream is recorded."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MIB = 1 << 20


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


def context(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


@pytest.mark.parametrize("dim", [1024, 2048, 4096, 8192, 12_000, 16_384])
def test_room(mqg, dim):
    limit = 8 * dim << 10 if dim <= 2048 else max(16 * MIB, 2 * dim << 10)
    contexts = [context(mqg) for _ in range(9)]
    contexts[0].reserve_layer(norm_dim=dim)                                # the allocator's own beginning
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    for c in contexts[1:]:
        c.reserve_layer(norm_dim=dim)
    used = (before - torch.cuda.mem_get_info()[0]) / 8
    assert used <= limit + 2 * MIB, (used / MIB, limit / MIB)              # (the allocator's pages are 2 MiB)


# widths at the ends of every layout
BORDERS = [1, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 512, 513, 768, 769, 1024, 1025, 1536, 2048, 2049, 4096, 4097, 8192, 8193, 16_384]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_reserved_for_every_width_and_number_of_rows(mqg, dtype):
    side = torch.cuda.Stream()
    for dim in BORDERS:
        ctx, eager = context(mqg), context(mqg)
        ctx.reserve_layer(norm_dim=dim)
        for width in {dim, max(d for d in BORDERS if d < dim) if dim > 1 else 1, dim // 2 + 1}:
            for rows in (3, 256, 257, 5000, 70_000 if width <= 256 else 5001):
                gen = torch.Generator(device="cuda").manual_seed(width)
                s, gy = (torch.randn((rows, width), generator=gen, device="cuda").to(dtype) for _ in range(2))
                out = [[torch.zeros_like(s), torch.zeros(width, device="cuda"), torch.zeros(width, device="cuda"), torch.zeros_like(s), torch.zeros(width, device="cuda")]
                       for _ in range(2)]

                def call(c, o):
                    mqg.mqg_layer_norm_backward(c, gy, s, None, o[0], grad_weight=o[1], grad_bias=o[2])
                    mqg.mqg_rms_norm_backward(c, gy, s, None, o[3], grad_weight=o[4])

                torch.cuda.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    call(ctx, out[0])
                graph.replay()
                call(eager, out[1])
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(*out)), (dim, width, rows)
