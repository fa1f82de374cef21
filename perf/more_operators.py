"""Cases of the gated feed-forward block and of the Muon step.

Every case is one call of a training or serving step.  Where ``own`` is false, ``run`` computes the
operators from elementary torch operations in 32 bits, rounded once at the end; where it is true, it makes
the calls that a user makes of ``paper_2201_06227_b200.ops``.

  gated forward     g = x w_gate^T + b_gate;  u = x w_up^T + b_up;  y = (act(g) * u) w_down^T + b_down + residual
  gated backward    dh = dy w_down;  dg = dh * u * act'(g);  du = dh * act(g);  dx = dg w_gate + du w_up;
                    dw_gate = dg^T x;  dw_up = du^T x;  dw_down = dy^T (act(g) * u);  db = the columns' sums
  Muon              m = beta m + (1 - beta) g;  t = beta m + (1 - beta) g (Nesterov) or m;  X = t / max(|t|, eps);
                    five times X = a X + (b A + c A^2) X with A = X X^T;  p = p (1 - lr wd) - lr scale X,
                    for every matrix of a model whose module is not frozen

The sizes are those of the named workloads of the package (hidden size 1024, 27 blocks of 16, 32 and 64
channels), twice them, and odd ones between; a gated block's hidden size is the usual 8/3 of the width, rounded
up to a multiple of 256.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
NS_A, NS_B, NS_C, NS_STEPS = 3.4445, -4.7750, 2.0315, 5
LR, BETA, EPS = 1e-4, 0.95, 1e-7


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one token of a decoder: the whole cost is reading the three weights and the launches
        dict(name="gated_token", op="gated_forward", type="bf16", rows=1, inp=1024, hidden=2816, out=1024, act="silu",
             bias=False, residual=True, save=False),
        # a small batch of sequences while decoding
        dict(name="gated_batch", op="gated_forward", type="bf16", rows=48, inp=1024, hidden=2816, out=1024, act="silu",
             bias=False, residual=True, save=False),
        # a training step's tokens through a 1024-wide block, with what its backward pass needs
        dict(name="gated_train", op="gated_forward", type="bf16", rows=16384, inp=1024, hidden=2816, out=1024, act="silu",
             bias=False, residual=True, save=True),
        # a block of twice the width over a long prompt, nothing kept
        dict(name="gated_prompt", op="gated_forward", type="bf16", rows=16384, inp=2048, hidden=5632, out=2048, act="gelu_tanh",
             bias=False, residual=True, save=False),
        # nothing a multiple of anything, biases everywhere
        dict(name="gated_odd", op="gated_forward", type="f16", rows=333, inp=519, hidden=1001, out=517, act="gelu",
             bias=True, residual=True, save=True),
        # the gradients of the training step's block
        dict(name="gated_back", op="gated_backward", type="bf16", rows=16384, inp=1024, hidden=2816, out=1024, act="silu",
             bias=False),
        # a ragged batch through a small block, biases everywhere
        dict(name="gated_back_odd", op="gated_backward", type="f16", rows=777, inp=515, hidden=1333, out=519, act="gelu_tanh",
             bias=True),
        # the matrices of a 24-block, 1024-wide decoder, bf16 weights with 32-bit masters, a third of its blocks frozen
        dict(name="muon_decoder", op="muon", type="bf16", master=True, model="decoder", hidden=1024, modules=24, frozen=8,
             nesterov=True),
        # two blocks of twice the width with gated feed-forwards, weights without masters
        dict(name="muon_gated", op="muon", type="bf16", master=False, model="gated", hidden=2048, modules=2, frozen=0,
             nesterov=True),
        # the 54 convolutions of a 27-block residual network of 16, 32 and 64 channels
        dict(name="muon_small", op="muon", type="f32", master=False, model="residual", hidden=64, modules=27, frozen=5,
             nesterov=False),
        # nothing a multiple of anything
        dict(name="muon_odd", op="muon", type="f16", master=True, model="decoder", hidden=333, modules=2, frozen=1,
             nesterov=True),
    ]


def _spread(rng, low, high):
    """A whole number of low..high, spread over the logarithm; odd ones and multiples of 64 among them."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    shape = rng.randrange(3)
    if shape == 0:
        n = max(low, n // 64 * 64)
    elif shape == 1:
        n |= 1
    return min(max(n, low), high)


def draw(rng):
    op = rng.choice(["gated_forward", "gated_backward", "muon"])
    acts = ["silu", "gelu_tanh", "gelu", "relu", "none"]
    if op != "muon":
        inp, hidden = _spread(rng, 16, 2048), _spread(rng, 16, 5632)
        out = inp if rng.random() < 0.7 else _spread(rng, 16, 2048)
        most = 16384 * 2048 * 5632 if op == "gated_forward" else 16384 * 1024 * 5632
        rows = _spread(rng, 1, max(1, min(32768, most // (max(inp, out) * hidden))))
        case = dict(op=op, type=rng.choice(["bf16", "bf16", "f16"]), rows=rows, inp=inp, hidden=hidden, out=out,
                    act=rng.choice(acts), bias=rng.random() < 0.4)
        if op == "gated_forward":
            case.update(residual=rng.random() < 0.7, save=rng.random() < 0.5)
        return case
    model = rng.choice(["decoder", "gated", "residual"])
    hidden = _spread(rng, 8, 128) if model == "residual" else _spread(rng, 64, 1024)
    modules = rng.randint(1, 24 if model == "residual" else max(1, min(24, int(16 * (1024 / hidden) ** 3))))
    dtype = rng.choice(["f32", "bf16", "f16"])
    return dict(op=op, type=dtype, master=dtype != "f32" and rng.random() < 0.5, model=model, hidden=hidden, modules=modules,
                frozen=rng.randint(0, modules - 1), nesterov=rng.random() < 0.7)


# ----------------------------------------------------------------------------- what a program has in hand

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(20220622 + int(seed))
    return g


def _matrices(case):
    """{(rows, cols): the module of every matrix of that shape} of the model."""
    h, shapes = case["hidden"], {}
    for k in range(case["modules"]):
        if case["model"] == "decoder":       # four projections and the two hidden products
            block = 4 * [(h, h)] + [(4 * h, h), (h, 4 * h)]
        elif case["model"] == "gated":       # four projections and the three products of a gated block
            wide = -(-8 * h // 768) * 256 if h % 256 == 0 else 8 * h // 3
            block = 4 * [(h, h)] + [(wide, h), (wide, h), (h, wide)]
        else:                                # two 3 x 3 convolutions, wider in later thirds
            c = max(1, h >> max(0, 2 - 3 * k // case["modules"]))
            block = 2 * [(c, 9 * c)]
        for shape in block:
            shapes.setdefault(shape, []).append(k)
    return shapes


def _scale(shape):
    return 0.2 * math.sqrt(max(shape))       # an update whose values are as large as AdamW's usually are


def _muon_state(case, seed):
    g, t = _gen(seed), TYPES[case["type"]]
    shapes = _matrices(case)
    s = dict(case=case, shapes=list(shapes), modules=list(shapes.values()), params=[], grads=[], m=[], masters=[], live=[])
    for (rows, cols), modules in shapes.items():
        n = len(modules)
        p = torch.randn(n, rows, cols, generator=g, device=DEVICE).mul_(1.0 / math.sqrt(min(rows, cols)))
        # gradients of a few strong directions over noise, their size different from matrix to matrix
        rank = max(1, min(rows, cols) // 16)
        strong = torch.randn(n, rows, rank, generator=g, device=DEVICE) @ torch.randn(n, rank, cols, generator=g, device=DEVICE)
        size = 1e-3 * torch.exp(torch.randn(n, 1, 1, generator=g, device=DEVICE))
        grad = (strong / math.sqrt(rank) + torch.randn(n, rows, cols, generator=g, device=DEVICE)) * size
        m = (0.5 * grad + 0.2 * size * torch.randn(n, rows, cols, generator=g, device=DEVICE))
        s["params"].append(p.to(t))
        s["grads"].append(grad.to(t))
        s["m"].append(m)
        s["masters"].append(p if case["master"] else None)
        s["live"].append(torch.tensor([i for i, k in enumerate(modules) if k >= case["frozen"]], dtype=torch.int64, device=DEVICE))
    s["frozen"] = (torch.arange(case["modules"], device=DEVICE) < case["frozen"]).to(torch.uint8)
    s["grad_scale"] = torch.full((1,), 0.5, device=DEVICE)
    return s


def prepare(case, seed):
    if case["op"] == "muon":
        s = _muon_state(case, seed)
        if own:   # the optimizer's handle: its table of matrices lives as long as the model does
            from paper_2201_06227_b200 import ops
            masters = [m for stack in s["masters"] for m in stack] if case["master"] else None
            s["muon"] = ops.Muon([p for stack in s["params"] for p in stack], [g for stack in s["grads"] for g in stack],
                                 [m for stack in s["m"] for m in stack], masters=masters, weight_decay=0.1, scale="rms",
                                 modules=[k for modules in s["modules"] for k in modules])
        return s
    g, t = _gen(seed), TYPES[case["type"]]
    rows, inp, hidden, out = case["rows"], case["inp"], case["hidden"], case["out"]

    def rand(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale).to(t)

    s = dict(case=case, x=rand(rows, inp), w_gate=rand(hidden, inp, scale=inp ** -0.5), w_up=rand(hidden, inp, scale=inp ** -0.5),
             w_down=rand(out, hidden, scale=hidden ** -0.5))
    if case["op"] == "gated_forward":
        for k, n in (("b_gate", hidden), ("b_up", hidden), ("b_down", out)):
            s[k] = rand(n, scale=0.1) if case["bias"] else None
        s["residual"] = rand(rows, out) if case["residual"] else None
    else:
        s["dy"] = rand(rows, out, scale=1.0 / 64)
        s["g"] = (s["x"].float() @ s["w_gate"].float().t()).to(t)
        s["u"] = (s["x"].float() @ s["w_up"].float().t()).to(t)
    if own:   # the handle and its workspace, kept for the whole run
        from paper_2201_06227_b200 import ops
        s["ops"] = ops.Ops(ops.egeria_gated_workspace_bytes(rows, inp, hidden, out))
    return s


# ----------------------------------------------------------------------------- one pass

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def run(s):
    case = s["case"]
    return {"gated_forward": _gated_forward, "gated_backward": _gated_backward, "muon": _muon}[case["op"]](s, case)


def _gated_forward(s, case):
    if own:
        return s["ops"].egeria_gated_forward(s["x"], s["w_gate"], s["w_up"], s["w_down"], b_gate=s["b_gate"], b_up=s["b_up"],
                                             b_down=s["b_down"], act=case["act"], residual=s["residual"], save=case["save"])
    t, x = s["x"].dtype, s["x"].float()
    g, u = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    if case["bias"]:
        g, u = g + s["b_gate"].float(), u + s["b_up"].float()
    y = (_act(g, case["act"]) * u) @ s["w_down"].float().t()
    if case["bias"]:
        y = y + s["b_down"].float()
    if case["residual"]:
        y = y + s["residual"].float()
    return (y.to(t), g.to(t), u.to(t)) if case["save"] else y.to(t)


def _gated_backward(s, case):
    if own:
        return s["ops"].egeria_gated_backward(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"], s["g"], s["u"], act=case["act"],
                                              need_db=case["bias"])
    t, dy, x, g, u = s["dy"].dtype, s["dy"].float(), s["x"].float(), s["g"].float(), s["u"].float()
    dh, a = dy @ s["w_down"].float(), _act(g, case["act"])
    dg, du = dh * u * _slope(g, case["act"]), dh * a
    dx = dg @ s["w_gate"].float() + du @ s["w_up"].float()
    db = dict(db_gate=dg.sum(0).to(t), db_up=du.sum(0).to(t), db_down=dy.sum(0).to(t)) if case["bias"] else \
        dict(db_gate=None, db_up=None, db_down=None)
    return dict(dx=dx.to(t), dw_gate=(dg.t() @ x).to(t), dw_up=(du.t() @ x).to(t), dw_down=(dy.t() @ (a * u)).to(t), **db)


def _muon(s, case):
    if own:
        s["muon"].egeria_muon_step(LR, beta=BETA, nesterov=case["nesterov"], eps=EPS, grad_scale=s["grad_scale"], frozen=s["frozen"])
    else:
        for shape, live, params, grads, moments, masters in zip(s["shapes"], s["live"], s["params"], s["grads"], s["m"], s["masters"]):
            g = grads[live].float() * s["grad_scale"]
            m = BETA * moments[live] + (1.0 - BETA) * g
            t = BETA * m + (1.0 - BETA) * g if case["nesterov"] else m
            x = t / torch.sqrt((t * t).sum((1, 2), keepdim=True)).clamp(min=EPS)
            x = x.transpose(1, 2) if shape[0] > shape[1] else x
            for _ in range(NS_STEPS):
                a = x @ x.transpose(1, 2)
                x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
            x = x.transpose(1, 2) if shape[0] > shape[1] else x
            p = (params if masters is None else masters)[live].float()
            p = p * (1.0 - LR * 0.1) - LR * _scale(shape) * x
            moments[live] = m
            params[live] = p.to(params.dtype)
            if masters is not None:
                masters[live] = p
    return dict(params=s["params"], m=s["m"], masters=s["masters"] if case["master"] else None)


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "muon":
        size = flops = 0
        for (rows, cols), modules in _matrices(case).items():
            n, low, high = sum(k >= case["frozen"] for k in modules), min(rows, cols), max(rows, cols)
            size += n * rows * cols
            # A and A^2 are symmetric: half of each is enough
            flops += n * NS_STEPS * (low * low * high + low ** 3 + 2 * low * low * high)
        each = BYTES[case["type"]] * (2 if case["master"] else 3) + (8 if case["master"] else 0) + 8
        return {"bytes": size * each, "flops": flops}
    r, i, h, o, b = case["rows"], case["inp"], case["hidden"], case["out"], BYTES[case["type"]]
    weights = 2 * h * i + o * h
    if case["op"] == "gated_forward":
        n = r * i + weights + r * o * (1 + case["residual"]) + 2 * r * h * case["save"] + (2 * h + o) * case["bias"]
        return {"bytes": n * b, "flops": 2 * r * weights}
    return {"bytes": (r * o + 2 * r * i + 2 * r * h + 2 * weights + (2 * h + o) * case["bias"]) * b, "flops": 4 * r * weights}


# ----------------------------------------------------------------------------- the definition in 64 bits

def _exact_act(z, act):
    """Value and slope of the activation."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    v = z if act == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
    dv = 1.0 if act == "silu" else math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
    p = 1 / (1 + torch.exp(-v))
    return z * p, p + z * dv * p / (1 + torch.exp(v))


def exact(case, seed):
    global own
    before, own = own, False        # the inputs alone, without a handle
    s = prepare(case, seed)
    own = before
    if case["op"] == "muon":
        return _exact_muon(s, case)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "gated_forward":
        g, u = (torch.einsum("ri,hi->rh", d["x"], d[w]) + (d[b] if b in d else 0.0) for w, b in (("w_gate", "b_gate"), ("w_up", "b_up")))
        y = torch.einsum("rh,oh->ro", _exact_act(g, case["act"])[0].mul_(u), d["w_down"]) + d.get("b_down", 0.0) + d.get("residual", 0.0)
        return (y, g, u) if case["save"] else y
    value, slope = _exact_act(d["g"], case["act"])
    dh = torch.einsum("ro,oh->rh", d["dy"], d["w_down"])
    both = torch.stack([dh * d["u"] * slope, dh * value])
    dx = torch.einsum("krh,khi->ri", both, torch.stack([d["w_gate"], d["w_up"]]))
    dw_gate, dw_up = torch.einsum("krh,ri->khi", both, d["x"])
    dw_down = torch.einsum("ro,rh->oh", d["dy"], value * d["u"])
    sums = torch.einsum("krh->kh", both) if case["bias"] else (None, None)
    return dict(dx=dx, dw_gate=dw_gate, dw_up=dw_up, dw_down=dw_down, db_gate=sums[0], db_up=sums[1],
                db_down=torch.einsum("ro->o", d["dy"]) if case["bias"] else None)


def _exact_muon(s, case):
    out = dict(params=[], m=[], masters=[] if case["master"] else None)
    for i, (rows, cols) in enumerate(s["shapes"]):
        p = s["params"][i].double() if s["masters"][i] is None else s["masters"][i].double()
        m, at = s["m"][i].double(), s["live"][i]
        g = torch.index_select(s["grads"][i], 0, at).double() * s["grad_scale"].double()
        mean = torch.lerp(g, m[at], BETA)
        t = torch.lerp(g, mean, BETA) if case["nesterov"] else mean
        m[at] = mean
        x = t / torch.linalg.vector_norm(t, dim=(1, 2), keepdim=True).clamp(min=EPS)
        # the polynomial from the side of the shorter axis, which is the same matrix
        left = rows <= cols
        for _ in range(NS_STEPS):
            gram = torch.einsum("nij,nkj->nik", x, x) if left else torch.einsum("nji,njk->nik", x, x)
            factor = torch.baddbmm(NS_B * gram, gram, gram, alpha=NS_C)
            factor.diagonal(dim1=1, dim2=2).add_(NS_A)
            x = torch.bmm(factor, x) if left else torch.bmm(x, factor)
        moved = p.clone()
        moved[at] = (1 - LR * 0.1) * p[at] - (LR * 0.2 * math.sqrt(max(rows, cols))) * x
        out["m"].append(m)
        # (a frozen matrix keeps the weights that it has, which need not be its master's rounding)
        kept = s["params"][i].double()
        kept[at] = moved[at]
        out["params"].append(kept)
        if case["master"]:
            out["masters"].append(moved)
    return out
