"""Layer norm with its backward, and the AdamW step over many tensors with the norm of their gradients before it, for timing.

``run`` computes them in plain torch operations in 32 bits, or, where ``own`` is true, through the public entry points of
``paper_2601_04707_amd.mqg``.  ``exact`` states them in 64 bits.

Kinds of cases
    layer   layer norm of hidden rows, with the residual's addition, as rows and / or in 8 bits with scales
    grad    its backward: gradients of the rows, of the weight and of the bias
    adamw   a step of all tensors of a network, moments in 32 bits or in 8 with a scale per 128; `clip`: before it the norm of all
            gradients, and the factor that clips them

Rows are those of the blocks of the workloads of ``paper_2601_04707_amd.synth`` and generic ones of wider models.  A network is a
stack of layers, each a matrix over a row and its neighbours' mean, its bias and the norm's weight and bias, and a classifier.
All weights lie in one buffer, and so do the moments, the copies and the gradients: `packed`, one tensor right after the other, as
buckets that ranks reduce have them, or each at a multiple of 256 bytes.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
NORM_EPS = 1e-5
LEAST_SCALE = 2.0 ** -126
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 7
BLOCK = 128                       # elements of a tensor that share the scale of an 8-bit moment
LEAST_ROOT = 2.0 ** -9            # the least 8-bit value above zero


def listed():
    return [
        # hidden rows of a small graph's mini-batch: latency
        {"name": "layer_tiny", "kind": "layer", "rows": 256, "dim": 64, "pad": 0, "dtype": "f32", "residual": True, "out": "rows", "group": 0},
        # one row of a wide model, as answering a single request gives it, quantised by groups for the product after it
        {"name": "layer_one_row", "kind": "layer", "rows": 1, "dim": 8192, "pad": 0, "dtype": "bf16", "residual": True, "out": "rows+e4m3", "group": 128},
        # input rows of a dense graph's mini-batch, an odd width in padded rows
        {"name": "layer_medium", "kind": "layer", "rows": 109_000, "dim": 602, "pad": 6, "dtype": "f32", "residual": True, "out": "rows", "group": 0},
        # hidden rows of a large batch, to be read in 8 bits by the next block's aggregation
        {"name": "layer_stress", "kind": "layer", "rows": 295_000, "dim": 256, "pad": 0, "dtype": "f16", "residual": True, "out": "e4m3", "group": 0},
        # the backward of a small batch, of a large one, and of wide rows
        {"name": "grad_tiny", "kind": "grad", "rows": 1_400, "dim": 64, "pad": 0, "dtype": "f32", "residual": True},
        {"name": "grad_stress", "kind": "grad", "rows": 295_000, "dim": 256, "pad": 0, "dtype": "f16", "residual": True},
        {"name": "grad_wide", "kind": "grad", "rows": 8_192, "dim": 8_192, "pad": 0, "dtype": "bf16", "residual": True},
        # a small network's step with clipped gradients: latency
        {"name": "adamw_tiny", "kind": "adamw", "layers": 2, "dim": 64, "classes": 41, "weight": "f32", "dtype": "f32", "copy": "", "bits": 32, "clip": True,
         "packed": False},
        # many tensors of odd sizes one right after the other, moments in 8 bits, clipped gradients
        {"name": "adamw_many", "kind": "adamw", "layers": 60, "dim": 301, "classes": 47, "weight": "f32", "dtype": "f32", "copy": "", "bits": 8, "clip": True,
         "packed": True},
        # a wide model's step: gradients in 16 bits, the weights' copy in 16 bits for the next forward
        {"name": "adamw_wide", "kind": "adamw", "layers": 12, "dim": 2_048, "classes": 172, "weight": "f32", "dtype": "bf16", "copy": "bf16", "bits": 32,
         "clip": False, "packed": False},
        # the same with clipped gradients
        {"name": "adamw_wide_clip", "kind": "adamw", "layers": 12, "dim": 2_048, "classes": 172, "weight": "f32", "dtype": "bf16", "copy": "bf16", "bits": 32,
         "clip": True, "packed": False},
        # the same with moments in 8 bits
        {"name": "adamw_wide_8bit", "kind": "adamw", "layers": 12, "dim": 2_048, "classes": 172, "weight": "f32", "dtype": "bf16", "copy": "bf16", "bits": 8,
         "clip": False, "packed": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layer", "layer", "grad", "grad", "adamw", "adamw", "adamw"])
    case = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if kind == "adamw":
        case["layers"], case["dim"], case["classes"] = _log(rng, 1, 100), _log(rng, 16, 2_048), _log(rng, 2, 1_000)
        if rng.random() < 0.5:
            case["dim"] = -(-case["dim"] // 16) * 16       # as most layers have
        while case["layers"] > 1 and _count(case) > 9 * 10 ** 7:
            case["layers"] = case["layers"] * 2 // 3
        case["weight"] = rng.choice(["f32", "f32", "f32", case["dtype"]])
        case["copy"] = rng.choice(["", "bf16", "f16"]) if case["weight"] == "f32" else ""
        case["bits"], case["clip"], case["packed"] = rng.choice([32, 8, 8]), rng.random() < 0.4, rng.random() < 0.5
        return case
    case["dim"] = _log(rng, 16, 8192)
    case["pad"] = rng.choice([0, -case["dim"] % 16, rng.randint(1, 9)])
    case["rows"] = rng.choice([_log(rng, 1, 64), _log(rng, 64, 300_000), _log(rng, 64, 300_000)])
    while case["rows"] * case["dim"] > 7 * 10 ** 7:
        case["rows"] = max(1, case["rows"] * 2 // 3)
    case["residual"] = rng.random() < 0.7
    if kind == "layer":
        case["out"], case["group"] = rng.choice(["rows", "e4m3", "rows+e4m3", "int8"]), rng.choice([0, 0, 32, 64, 128])
        if case["out"] == "rows":
            case["group"] = 0
    return case


# ---- inputs ---------------------------------------------------------------------------------------

def _groups(case):
    return -(-case["dim"] // case["group"]) if case["group"] else 1


def _rows(gen, rows, dim, pad, dtype, spread=0.0):
    """Normal rows in a buffer with `pad` more columns; `spread`: their sizes and means differ, and one in fifty is zero (no unit was active)."""
    buf = torch.zeros((rows, dim + pad), dtype=dtype, device="cuda")
    x = torch.randn((rows, dim), generator=gen, device="cuda")
    if spread:
        x += 0.5 * torch.randn((rows, 1), generator=gen, device="cuda")
        size = torch.exp(spread * torch.randn((rows, 1), generator=gen, device="cuda"))
        alive = torch.rand((rows, 1), generator=gen, device="cuda") > 0.02
        x *= size * alive
    buf[:, :dim] = x.to(dtype)
    return buf[:, :dim]


def _empty(rows, dim, pad, dtype):
    return torch.zeros((rows, dim + pad), dtype=dtype, device="cuda")[:, :dim]


def _shapes(case):
    dim = case["dim"]
    return [(dim, 2 * dim), (dim,), (dim,), (dim,)] * case["layers"] + [(case["classes"], dim), (case["classes"],)]


def _count(case):
    return sum(math.prod(s) for s in _shapes(case))


def _quantised(x):
    """e4m3 values and the scales of blocks of 128 of a tensor in its order, nothing above zero below the least value."""
    flat = torch.nn.functional.pad(x.reshape(-1), (0, -x.numel() % BLOCK)).view(-1, BLOCK)
    scale = (flat.abs().amax(1) / 448).clamp(min=LEAST_SCALE)
    return (flat / scale.unsqueeze(1)).view(-1)[:x.numel()].view(x.shape), scale


def _places(sizes, step):
    """Where each of the tensors of these sizes begins in one buffer, at multiples of `step` elements, and the buffer's size."""
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // step) * step)
    return at


def _views(buf, shapes, places):
    return [buf[a:a + math.prod(s)].view(s) for s, a in zip(shapes, places)]


def _tensors(st, case, gen):
    """A network's gradients, weights, moments and what takes the weights' copy; st[k] is a buffer, st["list"][k] its tensors."""
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    blocks = [(-(-n // BLOCK),) for n in sizes]
    eight = case["bits"] == 8
    places, scale_places = _places(sizes, 1 if case["packed"] else 256), _places([b[0] for b in blocks], 1)
    state = torch.float8_e4m3fn if eight else torch.float32
    types = {"grad": DTYPES[case["dtype"]], "weight": DTYPES[case["weight"]], "m": state, "v": state}
    if case["copy"]:
        types["copy"] = DTYPES[case["copy"]]
    st["list"] = {}
    for k, t in types.items():
        st[k] = torch.zeros(places[-1], dtype=t, device="cuda")
        st["list"][k] = _views(st[k], shapes, places)
    if eight:
        for k in ("m_scale", "v_scale"):
            st[k] = torch.zeros(scale_places[-1], device="cuda")
            st["list"][k] = _views(st[k], blocks, scale_places)
    of = st["list"]
    for i, shape in enumerate(shapes):
        # gradients whose sizes differ from unit to unit, some of which were never active
        unit = 1e-2 * torch.exp(torch.randn((shape[0], 1), generator=gen, device="cuda"))
        unit *= torch.rand((shape[0], 1), generator=gen, device="cuda") > 0.02
        unit = unit if len(shape) == 2 else unit.view(-1)
        of["grad"][i].copy_(unit * torch.randn(shape, generator=gen, device="cuda"))
        wide = shape[-1] if len(shape) == 2 else 1
        of["weight"][i].copy_(torch.randn(shape, generator=gen, device="cuda") / math.sqrt(wide))
        # what a few steps of such gradients leave
        m = 0.3 * unit * torch.randn(shape, generator=gen, device="cuda")
        v = 5e-3 * unit * unit * (0.5 + torch.rand(shape, generator=gen, device="cuda"))
        if eight:
            q, scale = _quantised(m)
            of["m"][i].copy_(q)
            of["m_scale"][i].copy_(scale)
            q, scale = _quantised(v.sqrt())
            of["v"][i].copy_(torch.where(q > 0, q.clamp(min=LEAST_ROOT), q))
            of["v_scale"][i].copy_(scale)
        else:
            of["m"][i].copy_(m)
            of["v"][i].copy_(v)
    st["norm"], st["scale"] = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")


def _most_norm(case):
    """The largest norm that is let through: about a third of what these gradients have."""
    return 1e-2 * math.sqrt(_count(case))


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
    if kind == "adamw":
        _tensors(st, case, gen)
        if own:                                            # the list of tensors that a program makes once
            mqg, _ = _context()
            of = st["list"]
            st["params"] = mqg.Params(of["weight"], of["grad"], m=of["m"], v=of["v"], m_scale=of.get("m_scale"), v_scale=of.get("v_scale"),
                                      copies=of.get("copy"))
        return st
    rows, dim, pad = case["rows"], case["dim"], case["pad"]
    st["weight"] = 1 + 0.1 * torch.randn(dim, generator=gen, device="cuda")
    st["bias"] = 0.1 * torch.randn(dim, generator=gen, device="cuda")
    st["x"] = _rows(gen, rows, dim, pad, dtype, spread=0.5)
    if kind == "layer":
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
        st["grad_weight"], st["grad_bias"] = torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
    return st


# ---- one pass -------------------------------------------------------------------------------------

def _values(q, scale, group):
    """What an 8-bit tensor stands for: itself where it is a floating type, with its scales beside it; integers times their scales."""
    if q.dtype != torch.int8:
        return q
    width = group or q.shape[1]
    return (q.to(torch.float32) * scale.repeat_interleave(width, 1)[:, :q.shape[1]]).to(torch.float16)


def _plain_layer(st, case):
    s = st["x"].float()
    if case["residual"]:
        s = s + st["residual"].float()
    d = s - s.mean(1, keepdim=True)
    y = d * torch.rsqrt(d.square().mean(1, keepdim=True) + NORM_EPS) * st["weight"] + st["bias"]
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
    d = s - s.mean(1, keepdim=True)
    r = torch.rsqrt(d.square().mean(1, keepdim=True) + NORM_EPS)
    unit = d * r
    gw = g * st["weight"]
    gx = r * (gw - gw.mean(1, keepdim=True) - unit * (gw * unit).mean(1, keepdim=True))
    if case["residual"]:
        gx = gx + st["grad_sum"].float()
    return {"grad_x": st["grad_x"].copy_(gx), "grad_weight": (g * unit).sum(0), "grad_bias": g.sum(0)}


def _plain_norm(grads, most):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt().float().view(1)
    return {"norm": norm, "scale": (most / norm).clamp(max=1)}


def _plain_adamw(st, case):
    of, eight = st["list"], case["bits"] == 8
    out = _plain_norm(of["grad"], _most_norm(case)) if case["clip"] else {}
    for i, (weight, grad, m, v) in enumerate(zip(of["weight"], of["grad"], of["m"], of["v"])):
        g = grad.float()
        if case["clip"]:
            g = g * out["scale"]
        if eight:
            n = g.numel()
            m_old = m.float().view(-1) * of["m_scale"][i].repeat_interleave(BLOCK)[:n]
            root = v.float().view(-1) * of["v_scale"][i].repeat_interleave(BLOCK)[:n]
            m_new = BETA1 * m_old.view(g.shape) + (1 - BETA1) * g
            v_new = BETA2 * root.square().view(g.shape) + (1 - BETA2) * g * g
        else:
            m_new = m.mul_(BETA1).add_(g, alpha=1 - BETA1)
            v_new = v.mul_(BETA2).add_(g * g, alpha=1 - BETA2)
        root = v_new.sqrt()
        step = m_new / (1 - BETA1 ** STEP) / (root / math.sqrt(1 - BETA2 ** STEP) + ADAM_EPS)
        w = weight.float() * (1 - LR * DECAY) - LR * step
        weight.copy_(w)
        if case["copy"]:
            of["copy"][i].copy_(w)
        if eight:
            q, scale = _quantised(m_new)
            m.copy_(q)
            of["m_scale"][i].copy_(scale)
            q, scale = _quantised(root)
            v.copy_(torch.where(q > 0, q.clamp(min=LEAST_ROOT), q))
            of["v_scale"][i].copy_(scale)
    return {**out, **_stepped(st)}


def _stepped(st):
    return {k: st[k] for k in ("weight", "m", "v", "copy", "m_scale", "v_scale") if k in st}


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"layer": _plain_layer, "grad": _plain_grad, "adamw": _plain_adamw}[kind](st, case)
    mqg, ctx = _context()
    if kind == "layer":
        mqg.mqg_layer_norm(ctx, st["x"], st["weight"], st["bias"], residual=st["residual"], sum_out=st["sum"], y=st["y"], q=st["q"],
                           q_scale=st["scale"], group=case["group"], eps=NORM_EPS)
        out = {k: st[k] for k in ("sum", "y", "scale") if st[k] is not None}
        if st["q"] is not None:
            out["q"] = _values(st["q"], st["scale"], case["group"])
        return out
    if kind == "grad":
        mqg.mqg_layer_norm_backward(ctx, st["grad_y"], st["x"], st["weight"], st["grad_x"], grad_weight=st["grad_weight"], grad_bias=st["grad_bias"],
                                    grad_sum=st["grad_sum"], eps=NORM_EPS)
        return {"grad_x": st["grad_x"], "grad_weight": st["grad_weight"], "grad_bias": st["grad_bias"]}
    out = {}
    if case["clip"]:
        mqg.mqg_grad_norm(ctx, st["params"], max_norm=_most_norm(case), norm=st["norm"], scale=st["scale"])
        out = {"norm": st["norm"], "scale": st["scale"]}
    mqg.mqg_adamw_step(ctx, st["params"], lr=LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                       grad_scale=st["scale"] if case["clip"] else None)
    return {**out, **_stepped(st)}


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    size = SIZES[case["dtype"]]
    if case["kind"] == "adamw":
        n = _count(case)
        moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        # clipped gradients are read twice: no element can step before the norm is known
        grads = size * (2 if case["clip"] else 1)
        return {"bytes": n * (grads + 2 * SIZES[case["weight"]] + (2 if case["copy"] else 0) + moments), "flops": (18 if case["clip"] else 16) * n}
    cells = case["rows"] * case["dim"]
    if case["kind"] == "layer":
        moved = cells * size * (1 + (2 if case["residual"] else 0) + ("rows" in case["out"]))
        if case["out"] != "rows":
            moved += cells + 4 * case["rows"] * _groups(case)
        return {"bytes": moved + 8 * case["dim"], "flops": 8 * cells}
    return {"bytes": cells * size * (4 if case["residual"] else 3) + 12 * case["dim"], "flops": 16 * cells}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_round8(v, e4m3):
    """To nearest, ties to even, in the 8-bit type's values: integers, or three bits after the leading one down to exponent -6."""
    if not e4m3:
        return torch.round(v).clamp(-127, 127)
    _, e = torch.frexp(v)
    unit = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return (torch.round(v / unit) * unit).clamp(-448, 448)


def _exact_moment(x, least):
    """8-bit values and scales, block after block of the tensor; values above zero have at least `least`."""
    flat = x.reshape(-1)
    whole = flat.numel() // BLOCK * BLOCK
    most = [flat[:whole].view(-1, BLOCK).abs().max(1).values] if whole else []
    if whole < flat.numel():
        most.append(flat[whole:].abs().max().view(1))
    scale = torch.clamp(torch.cat(most) / 448.0, min=LEAST_SCALE)
    of = scale[torch.arange(flat.numel(), device=flat.device) // BLOCK]
    q = _exact_round8(flat / of, True)
    if least:
        q = torch.where((flat > 0) & (q < least), torch.full_like(q, least), q)
    return q.view(x.shape), scale


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    kind = case["kind"]
    if kind == "layer":
        s = st["x"].to(f64)
        if case["residual"]:
            s += st["residual"].to(f64)
        mean = s.sum(1, keepdim=True) / case["dim"]
        std = (((s - mean) ** 2).sum(1, keepdim=True) / case["dim"] + NORM_EPS).sqrt()
        y = (s - mean) / std * st["weight"].to(f64) + st["bias"].to(f64)
        out = {}
        if case["residual"]:
            out["sum"] = s
        if st["y"] is not None:
            out["y"] = y
        if st["q"] is not None:
            e4m3 = "e4m3" in case["out"]
            parts = torch.split(y, case["group"] or case["dim"], 1)
            most = torch.stack([p.abs().max(1).values for p in parts], 1)
            out["scale"] = torch.clamp(most / (448.0 if e4m3 else 127.0), min=LEAST_SCALE)
            q = [_exact_round8(p / out["scale"][:, i, None], e4m3) for i, p in enumerate(parts)]
            if not e4m3:
                q = [p * out["scale"][:, i, None] for i, p in enumerate(q)]
            out["q"] = torch.cat(q, 1)
        return out
    if kind == "grad":
        s, g, w = st["x"].to(f64), st["grad_y"].to(f64), st["weight"].to(f64)
        mean = s.sum(1, keepdim=True) / case["dim"]
        std = (((s - mean) ** 2).sum(1, keepdim=True) / case["dim"] + NORM_EPS).sqrt()
        unit = (s - mean) / std
        gw = g * w
        gx = (gw - (gw.sum(1, keepdim=True) + unit * (gw * unit).sum(1, keepdim=True)) / case["dim"]) / std
        if case["residual"]:
            gx += st["grad_sum"].to(f64)
        return {"grad_x": gx, "grad_weight": (g * unit).sum(0), "grad_bias": g.sum(0)}
    of = st["list"]
    out = {k: torch.zeros(st[k].shape, dtype=f64, device="cuda") for k in _stepped(st)}
    factor = 1.0
    if case["clip"]:
        total = float(torch.dot(st["grad"].to(f64), st["grad"].to(f64)))                  # (zeros between the tensors)
        factor = min(1.0, _most_norm(case) / math.sqrt(total))
        out["norm"] = torch.tensor([math.sqrt(total)], dtype=f64, device="cuda")
        out["scale"] = torch.tensor([factor], dtype=f64, device="cuda")
    for i, g in enumerate(of["grad"]):
        g, m, v, w = factor * g.to(f64), of["m"][i].to(f64), of["v"][i].to(f64), of["weight"][i].to(f64)

        def put(key, value):
            start = of[key][i].storage_offset()
            out[key][start:start + value.numel()] = value.reshape(-1)

        if case["bits"] == 8:
            block = torch.arange(g.numel(), device="cuda").view(g.shape) // BLOCK
            m *= of["m_scale"][i].to(f64)[block]
            v = (v * of["v_scale"][i].to(f64)[block]) ** 2
        m += (1 - BETA1) * (g - m)
        v += (1 - BETA2) * (g * g - v)
        step = m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS)
        w = w - LR * DECAY * w - LR * step
        put("weight", w)
        if case["copy"]:
            put("copy", w)
        if case["bits"] == 8:
            for key, x, least in (("m", m, 0.0), ("v", v.sqrt(), LEAST_ROOT)):
                q, scale = _exact_moment(x, least)
                put(key, q)
                put(key + "_scale", scale)
        else:
            put("m", m)
            put("v", v)
    return out
