"""The operators of a layer between two aggregations, over the sizes that a training program calls them at, for timing.

``run`` computes them in plain torch operations in 32 bits, or, where ``own`` is true, through the public entry points of
``paper_2601_04707_amd.mqg``.  ``exact`` states them in 64 bits.

Kinds of cases
    norm    root-mean-square norm of hidden rows, with the residual's addition, as rows and / or in 8 bits with scales
    grad    its backward: gradients of the rows and of the norm's weight
    mean8   the mean aggregation of a block whose source rows are held in 8 bits with scales
    orth    a stack of updates orthogonalised by Newton-Schulz products
    muon    the weights' step around it: momentum, orthogonalised update, decay

Sizes are those of the workloads of ``paper_2601_04707_amd.synth`` (blocks, feature widths, a layer's weights over a row and its
neighbours' mean) and generic ones of wider models.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
COEFFS = (3.4445, -4.775, 2.0315)
NORM_EPS, ORTH_EPS = 1e-6, 1e-7
STEPS = 5
LR, BETA, DECAY = 0.02, 0.95, 0.01
LEAST_SCALE = 2.0 ** -126


def listed():
    return [
        # hidden rows of a small graph's mini-batch: latency
        {"name": "norm_tiny", "kind": "norm", "rows": 256, "dim": 64, "pad": 0, "dtype": "f32", "residual": True, "out": "rows", "group": 0},
        # one row of a wide model, as answering a single request gives it, quantised by groups for the product after it
        {"name": "norm_one_row", "kind": "norm", "rows": 1, "dim": 8192, "pad": 0, "dtype": "bf16", "residual": True, "out": "rows+e4m3", "group": 128},
        # input rows of a dense graph's mini-batch, an odd width in padded rows
        {"name": "norm_medium", "kind": "norm", "rows": 109_000, "dim": 602, "pad": 6, "dtype": "f32", "residual": True, "out": "rows", "group": 0},
        # hidden rows of a large batch, to be read in 8 bits by the next block's aggregation
        {"name": "norm_stress", "kind": "norm", "rows": 295_000, "dim": 256, "pad": 0, "dtype": "f16", "residual": True, "out": "e4m3", "group": 0},
        # the backward of a small batch, of a large one, and of wide rows
        {"name": "grad_tiny", "kind": "grad", "rows": 1_400, "dim": 64, "pad": 0, "dtype": "f32", "residual": True},
        {"name": "grad_stress", "kind": "grad", "rows": 295_000, "dim": 256, "pad": 0, "dtype": "f16", "residual": True},
        {"name": "grad_wide", "kind": "grad", "rows": 8_192, "dim": 8_192, "pad": 0, "dtype": "bf16", "residual": True},
        # the aggregations that read 8-bit rows: long rows of odd width, and the outermost block of a large batch
        {"name": "mean8_medium", "kind": "mean8", "rows": 10_200, "fanout": 25, "sources": 109_000, "dim": 602, "pad": 6, "dtype": "f32",
         "type8": "e4m3", "group": 0},
        {"name": "mean8_stress", "kind": "mean8", "rows": 295_000, "fanout": 15, "sources": 1_350_000, "dim": 256, "pad": 0, "dtype": "f16",
         "type8": "e4m3", "group": 0},
        # one layer's weights: 256 hidden units over a row of 602 features and its neighbours' mean
        {"name": "muon_layer", "kind": "muon", "mats": 1, "rows": 256, "cols": 1_204, "dtype": "f32"},
        # a stack of square weights, gradients in 16 bits
        {"name": "orth_stack", "kind": "orth", "mats": 24, "rows": 1_024, "cols": 1_024, "dtype": "bf16"},
        # a wide model's weights, taller than wide
        {"name": "muon_large", "kind": "muon", "mats": 1, "rows": 8_192, "cols": 4_096, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "grad", "grad", "mean8", "mean8", "orth", "muon"])
    case = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if kind in ("orth", "muon"):
        case["rows"], case["cols"], case["mats"] = _log(rng, 16, 4096), _log(rng, 16, 4096), rng.choice([1, 1, 2, _log(rng, 2, 16)])
        if rng.random() < 0.5:                         # multiples of 16, as most layers have
            case["rows"], case["cols"] = -(-case["rows"] // 16) * 16, -(-case["cols"] // 16) * 16
        while case["mats"] > 1 and work(case)["flops"] > 5e11:
            case["mats"] -= 1
        return case
    case["dim"] = _log(rng, 16, 8192 if kind != "mean8" else 1024)
    case["pad"] = rng.choice([0, -case["dim"] % 16, rng.randint(1, 9)])
    if kind == "mean8":
        case["rows"], case["fanout"] = _log(rng, 100, 295_000), _log(rng, 3, 40)
        while case["rows"] * case["fanout"] * case["dim"] > 4 * 10 ** 8:
            case["rows"] = max(100, case["rows"] * 2 // 3)
            case["fanout"] = max(3, case["fanout"] - 1)
        case["sources"] = case["rows"] * min(case["fanout"], rng.choice([1, 2, 5]))
        case["type8"], case["group"] = rng.choice(["e4m3", "int8"]), rng.choice([0, 0, 32, 64, 128])
        return case
    case["rows"] = rng.choice([_log(rng, 1, 64), _log(rng, 64, 300_000), _log(rng, 64, 300_000)])
    while case["rows"] * case["dim"] > 7 * 10 ** 7:
        case["rows"] = max(1, case["rows"] * 2 // 3)
    case["residual"] = rng.random() < 0.7
    if kind == "norm":
        case["out"], case["group"] = rng.choice(["rows", "e4m3", "rows+e4m3", "int8"]), rng.choice([0, 0, 32, 64, 128])
        if "8" not in case["out"] and "3" not in case["out"]:
            case["group"] = 0
    return case


# ---- inputs ---------------------------------------------------------------------------------------

def _groups(case):
    return -(-case["dim"] // case["group"]) if case["group"] else 1


def _rows(gen, rows, dim, pad, dtype, spread=0.0):
    """Normal rows in a buffer with `pad` more columns; `spread`: their sizes differ, and one in fifty is zero (no unit was active)."""
    buf = torch.zeros((rows, dim + pad), dtype=dtype, device="cuda")
    x = torch.randn((rows, dim), generator=gen, device="cuda")
    if spread:
        size = torch.exp(spread * torch.randn((rows, 1), generator=gen, device="cuda"))
        alive = torch.rand((rows, 1), generator=gen, device="cuda") > 0.02
        x *= size * alive
    buf[:, :dim] = x.to(dtype)
    return buf[:, :dim]


def _empty(rows, dim, pad, dtype):
    return torch.zeros((rows, dim + pad), dtype=dtype, device="cuda")[:, :dim]


_CONTEXT = []


def _context():
    """The context that a training program keeps: one per stream (here of a graph of two nodes: none of these calls reads the graph)."""
    if not _CONTEXT:
        from paper_2601_04707_amd import mqg
        graph = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
        _CONTEXT.append((mqg, mqg.Context(graph, 1, [1])))
    return _CONTEXT[0]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    st = {"case": case}
    if kind in ("orth", "muon"):
        m, r, c = case["mats"], case["rows"], case["cols"]
        # a gradient of a few strong directions and noise; momentum of earlier steps; weights of a fresh layer's size
        strong = torch.randn((m, r, 8), generator=gen, device="cuda") @ torch.randn((m, 8, c), generator=gen, device="cuda")
        st["grad"] = (1e-3 * (strong + torch.randn((m, r, c), generator=gen, device="cuda"))).to(dtype)
        del strong
        if kind == "muon":
            st["momentum"] = 1e-2 * torch.randn((m, r, c), generator=gen, device="cuda")
            st["weight"] = torch.randn((m, r, c), generator=gen, device="cuda") / math.sqrt(c)
        else:
            st["out"] = torch.zeros((m, r, c), dtype=dtype, device="cuda")
    elif kind == "mean8":
        d, f, s, dim = case["rows"], case["fanout"], case["sources"], case["dim"]
        # some destinations have fewer neighbours than the fanout, some none; a few sources are met far more often than the others
        count = torch.where(torch.rand(d, generator=gen, device="cuda") < 0.1, torch.randint(0, f + 1, (d,), generator=gen, device="cuda"), f)
        st["indptr"] = torch.zeros(d + 1, dtype=torch.int32, device="cuda")
        st["indptr"][1:] = torch.cumsum(count, 0)
        nnz = int(st["indptr"][-1])
        at = torch.rand(max(nnz, 1), generator=gen, device="cuda")
        st["indices"] = (s * at ** 2).to(torch.int64).clamp(max=s - 1).to(torch.int32)
        st["sizes"] = torch.tensor([d, s, nnz, 0], dtype=torch.int64, device="cuda")
        groups, width = _groups(case), case["group"] or dim
        x = torch.zeros((s, groups * width), device="cuda")
        x[:, :dim] = _rows(gen, s, dim, 0, torch.float32, spread=0.3)
        x = x.view(s, groups, width)
        scale = (x.abs().amax(2) / (448 if case["type8"] == "e4m3" else 127)).clamp(min=LEAST_SCALE)
        q = (x / scale.unsqueeze(2)).view(s, groups * width)[:, :dim]
        st["q"] = _empty(s, dim, case["pad"], torch.float8_e4m3fn if case["type8"] == "e4m3" else torch.int8)
        st["q"].copy_((q if case["type8"] == "e4m3" else q.round()).to(st["q"].dtype))
        st["scale"] = scale
        st["out"] = _empty(d, dim, case["pad"], dtype)
        if own:
            mqg, _ = _context()
            st["blocks"] = mqg.BlockView(st["indptr"], st["indices"], st["sizes"], s)
    else:
        rows, dim, pad = case["rows"], case["dim"], case["pad"]
        st["weight"] = 1 + 0.1 * torch.randn(dim, generator=gen, device="cuda")
        st["x"] = _rows(gen, rows, dim, pad, dtype, spread=0.5)
        if kind == "norm":
            st["residual"] = _rows(gen, rows, dim, pad, dtype, spread=0.5) if case["residual"] else None
            st["sum"] = _empty(rows, dim, pad, dtype) if case["residual"] else None
            st["y"] = _empty(rows, dim, pad, dtype) if "rows" in case["out"] else None
            kind8 = torch.float8_e4m3fn if "e4m3" in case["out"] else torch.int8 if "int8" in case["out"] else None
            st["q"] = _empty(rows, dim, -dim % 16, kind8) if kind8 else None
            st["scale"] = torch.zeros((rows, _groups(case)), device="cuda") if kind8 else None
        else:
            st["grad_y"] = _rows(gen, rows, dim, pad, dtype)
            st["grad_sum"] = _rows(gen, rows, dim, pad, dtype) if case["residual"] else None
            st["grad_x"] = _empty(rows, dim, pad, dtype)
            st["grad_weight"] = torch.zeros(dim, device="cuda")
    return st


# ---- one pass -------------------------------------------------------------------------------------

def _values(q, scale, group):
    """What an 8-bit tensor stands for: itself where it is a floating type, with its scales beside it; integers times their scales."""
    if q.dtype != torch.int8:
        return q
    width = group or q.shape[1]
    return (q.to(torch.float32) * scale.repeat_interleave(width, 1)[:, :q.shape[1]]).to(torch.float16)


def _plain_norm(st, case):
    s = st["x"].float()
    if case["residual"]:
        s = s + st["residual"].float()
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + NORM_EPS) * st["weight"]
    out = {}
    if case["residual"]:
        out["sum"] = st["sum"].copy_(s)
    if st["y"] is not None:
        out["y"] = st["y"].copy_(y)
    if st["q"] is not None:
        rows, dim, groups, width = case["rows"], case["dim"], _groups(case), case["group"] or case["dim"]
        y = torch.nn.functional.pad(y, (0, groups * width - dim)).view(rows, groups, width)
        e4m3 = st["q"].dtype != torch.int8
        out["scale"] = (y.abs().amax(2) / (448 if e4m3 else 127)).clamp(min=LEAST_SCALE)
        q = (y / out["scale"].unsqueeze(2)).view(rows, groups * width)[:, :dim]
        out["q"] = _values(st["q"].copy_((q if e4m3 else q.round()).to(st["q"].dtype)), out["scale"], case["group"])
    return out


def _plain_grad(st, case):
    s, g = st["x"].float(), st["grad_y"].float()
    r = torch.rsqrt(s.square().mean(1, keepdim=True) + NORM_EPS)
    gw = g * st["weight"]
    gx = r * gw - s * (r ** 3 * (gw * s).mean(1, keepdim=True))
    if case["residual"]:
        gx = gx + st["grad_sum"].float()
    return {"grad_x": st["grad_x"].copy_(gx), "grad_weight": (g * s * r).sum(0)}


def _plain_mean8(st, case):
    width = case["group"] or case["dim"]
    rows = st["q"].to(torch.float32) * st["scale"].repeat_interleave(width, 1)[:, :case["dim"]]
    first, count = st["indptr"][:-1].long(), (st["indptr"][1:] - st["indptr"][:-1]).long()
    at = torch.arange(case["fanout"], device="cuda")
    there = at < count[:, None]
    source = st["indices"][(first[:, None] + at).clamp(max=st["indices"].numel() - 1)].long()
    total = (rows[source] * there.unsqueeze(2)).sum(1)
    return {"out": st["out"].copy_(total / count.clamp(min=1)[:, None])}


def _plain_orthogonal(u):
    """The stack's orthogonalised matrices."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + ORTH_EPS)
    a, b, c = COEFFS
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_muon(st, case):
    g = st["grad"].float()
    m = st["momentum"].mul_(BETA).add_(g)
    o = _plain_orthogonal(g + BETA * m)
    scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
    w = st["weight"].mul_(1 - LR * DECAY).add_(o, alpha=-LR * scale)
    return {"weight": w, "momentum": m}


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind == "orth":
            return {"out": st["out"].copy_(_plain_orthogonal(st["grad"].float()))}
        return {"norm": _plain_norm, "grad": _plain_grad, "mean8": _plain_mean8, "muon": _plain_muon}[kind](st, case)
    mqg, ctx = _context()
    if kind == "norm":
        mqg.mqg_rms_norm(ctx, st["x"], st["weight"], residual=st["residual"], sum_out=st["sum"], y=st["y"], q=st["q"], q_scale=st["scale"],
                         group=case["group"], eps=NORM_EPS)
        out = {k: st[k] for k in ("sum", "y", "scale") if st[k] is not None}
        if st["q"] is not None:
            out["q"] = _values(st["q"], st["scale"], case["group"])
        return out
    if kind == "grad":
        mqg.mqg_rms_norm_backward(ctx, st["grad_y"], st["x"], st["weight"], st["grad_x"], grad_weight=st["grad_weight"],
                                  grad_sum=st["grad_sum"], eps=NORM_EPS)
        return {"grad_x": st["grad_x"], "grad_weight": st["grad_weight"]}
    if kind == "mean8":
        mqg.mqg_sage_mean_aggregate_q8(ctx, st["blocks"], 0, st["q"], st["scale"], st["out"], group=case["group"])
        return {"out": st["out"]}
    if kind == "orth":
        mqg.mqg_orthogonalize(ctx, st["grad"], st["out"], steps=STEPS, coeffs=COEFFS, eps=ORTH_EPS)
        return {"out": st["out"]}
    mqg.mqg_muon_step(ctx, st["grad"], st["momentum"], st["weight"], lr=LR, beta=BETA, nesterov=True, weight_decay=DECAY,
                      scale=math.sqrt(max(1.0, case["rows"] / case["cols"])), steps=STEPS, coeffs=COEFFS, eps=ORTH_EPS)
    return {"weight": st["weight"], "momentum": st["momentum"]}


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("orth", "muon"):
        n, k, m = min(case["rows"], case["cols"]), max(case["rows"], case["cols"]), case["mats"]
        flops = m * STEPS * (n * n * k + n ** 3 + 2 * n * n * k)       # of symmetric products one half
        return {"bytes": m * n * k * (size + (16 if case["kind"] == "muon" else size)), "flops": flops}
    cells = case["rows"] * case["dim"]
    if case["kind"] == "mean8":
        edges = case["rows"] * case["fanout"]
        met = min(edges, case["sources"])
        return {"bytes": met * (case["dim"] + 4 * _groups(case)) + 4 * edges + 4 * case["rows"] + cells * size, "flops": 2 * edges * case["dim"]}
    if case["kind"] == "norm":
        moved = cells * size * (1 + (2 if case["residual"] else 0) + ("rows" in case["out"]))
        if case["out"] != "rows":
            moved += cells + 4 * case["rows"] * _groups(case)
        return {"bytes": moved + 4 * case["dim"], "flops": 6 * cells}
    return {"bytes": cells * size * (4 if case["residual"] else 3) + 8 * case["dim"], "flops": 12 * cells}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_round8(v, e4m3):
    """To nearest, ties to even, in the 8-bit type's values: integers, or three bits after the leading one down to exponent -6."""
    if not e4m3:
        return torch.round(v).clamp(-127, 127)
    _, e = torch.frexp(v)
    unit = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return (torch.round(v / unit) * unit).clamp(-448, 448)


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    kind = case["kind"]
    if kind == "norm":
        s = st["x"].to(f64)
        if case["residual"]:
            s += st["residual"].to(f64)
        rms = ((s * s).sum(1) / case["dim"] + NORM_EPS).sqrt()
        y = s / rms[:, None] * st["weight"].to(f64)
        out = {}
        if case["residual"]:
            out["sum"] = s
        if st["y"] is not None:
            out["y"] = y
        if st["q"] is not None:
            e4m3 = "e4m3" in case["out"]
            width = case["group"] or case["dim"]
            parts = torch.split(y, width, 1)
            most = torch.stack([p.abs().max(1).values for p in parts], 1)
            out["scale"] = torch.clamp(most / (448.0 if e4m3 else 127.0), min=LEAST_SCALE)
            q = [_exact_round8(p / out["scale"][:, i, None], e4m3) for i, p in enumerate(parts)]
            if not e4m3:
                q = [p * out["scale"][:, i, None] for i, p in enumerate(q)]
            out["q"] = torch.cat(q, 1)
        return out
    if kind == "grad":
        s, g, w = st["x"].to(f64), st["grad_y"].to(f64), st["weight"].to(f64)
        rms = ((s * s).sum(1) / case["dim"] + NORM_EPS).sqrt()[:, None]
        unit = s / rms
        gw = g * w
        gx = (gw - unit * ((gw * unit).sum(1) / case["dim"])[:, None]) / rms
        if case["residual"]:
            gx += st["grad_sum"].to(f64)
        return {"grad_x": gx, "grad_weight": (g * unit).sum(0)}
    if kind == "mean8":
        ptr = st["indptr"].long()
        count = ptr[1:] - ptr[:-1]
        nnz = int(ptr[-1])
        row = torch.repeat_interleave(torch.arange(case["rows"], device="cuda"), count)
        width = case["group"] or case["dim"]
        group = torch.arange(case["dim"], device="cuda") // width
        total = torch.zeros((case["rows"], case["dim"]), dtype=f64, device="cuda")
        for e0 in range(0, nnz, 1 << 19):
            src = st["indices"][e0:min(nnz, e0 + (1 << 19))].long()
            total.index_add_(0, row[e0:e0 + src.numel()], st["q"].view(torch.int8)[src].view(st["q"].dtype).to(f64) * st["scale"].to(f64)[src][:, group])
        return {"out": total / count.clamp(min=1)[:, None]}
    g = st["grad"].to(f64)
    m = BETA * st["momentum"].to(f64) + g if kind == "muon" else None
    update = g + BETA * m if kind == "muon" else g
    results = []
    a, b, c = COEFFS
    for u in update:
        u = u / (torch.linalg.vector_norm(u) + ORTH_EPS)
        for _ in range(STEPS):
            # on the left or on the right, whichever Gram matrix is the smaller: the polynomial is the same
            gram = u @ u.T if u.shape[0] <= u.shape[1] else u.T @ u
            poly = b * gram + c * gram @ gram
            u = a * u + (poly @ u if u.shape[0] <= u.shape[1] else u @ poly)
        results.append(u)
    o = torch.stack(results)
    if kind == "orth":
        return {"out": o}
    scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
    return {"weight": st["weight"].to(f64) * (1 - LR * DECAY) - LR * scale * o, "momentum": m}
