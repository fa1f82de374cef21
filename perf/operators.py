"""Cases of the training operators: linear layers, residual norms and the AdamW step.

Every case is one call of a training or serving step.  Where ``own`` is false, ``run`` computes
the operators from elementary torch operations in 32 bits, rounded once at the end; where it is
true, it makes the calls that a user makes of ``paper_2201_06227_b200.ops``.

  linear forward    z = x w^T + bias;  y = act(z) + residual
  linear backward   dz = dy * act'(z);  dx = (dz w) * act_in'(z_in);  dw = dz^T x;  db = sum_rows dz
  norm forward      y = alpha x + gate * N_post(f);  h = N_pre(y)
  norm backward     the gradients of x, f, the gate and the norms' weights and biases
  AdamW             one step of many tensors; moments in 32 bits, or in 8 with a scale per 256 values

The sizes are those of the named workloads of the package (hidden sizes 768 and 1024, 4096 =
32 x 128 and 65536 = 256 x 256 tokens, the 16/32/64-channel blocks of a CIFAR residual network)
and odd ones between.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                     # values that share one scale of an 8-bit moment
BETA1, BETA2, ADAM_EPS, LR = 0.9, 0.999, 1e-8, 3e-4
NORM_EPS = 1e-5


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one token of a decoder: the whole cost is reading the weights and the launch
        dict(name="linear_token", op="linear_forward", type="bf16", rows=1, inp=1024, out=4096, act="gelu_tanh",
             bias=True, residual=False, save_z=False),
        # the hidden product of a 1024-wide block over 256 x 256 tokens, with what its backward pass needs
        dict(name="linear_hidden", op="linear_forward", type="bf16", rows=65536, inp=1024, out=4096, act="gelu_tanh",
             bias=True, residual=False, save_z=True),
        # an output projection of a 768-wide encoder over 32 x 128 tokens, added to the stream
        dict(name="linear_project", op="linear_forward", type="bf16", rows=4096, inp=768, out=768, act="none",
             bias=True, residual=True, save_z=False),
        # nothing a multiple of anything: row pitches that no tile load takes as they are
        dict(name="linear_odd", op="linear_forward", type="f16", rows=333, inp=1001, out=519, act="silu",
             bias=True, residual=True, save_z=True),
        # backward of a block's second product; its input came out of the first product's activation
        dict(name="linear_back", op="linear_backward", type="bf16", rows=16384, inp=4096, out=1024, act="none",
             act_in="gelu_tanh", bias=True),
        # a ragged batch through a small projection with its activation
        dict(name="linear_back_odd", op="linear_backward", type="f16", rows=777, inp=515, out=1001, act="gelu",
             act_in="none", bias=True),
        # one block boundary of the 1024-wide decoder: norm, gate, add and the next block's norm
        dict(name="norm_stream", op="norm_forward", type="bf16", kind="layer", rows=65536, cols=1024, post=True, pre=True,
             gate_rows=0, affine=True, alpha=1.0),
        # the same for one token per sequence while decoding
        dict(name="norm_token", op="norm_forward", type="bf16", kind="rms", rows=8, cols=1024, post=True, pre=True,
             gate_rows=0, affine=True, alpha=1.0),
        # its gradients, the gate given per sequence of 256 tokens
        dict(name="norm_back", op="norm_backward", type="bf16", kind="rms", rows=65536, cols=1024, post=True, pre=True,
             gate_rows=256, affine=True, alpha=1.0),
        # a 24-block, 1024-wide decoder with 32-bit moments, a third of its blocks frozen
        dict(name="adamw_decoder", op="adamw", bits=32, type="bf16", master=True, model="decoder", hidden=1024, modules=24,
             frozen=8),
        # the same model with 8-bit moments and nothing frozen
        dict(name="adamw_decoder_8", op="adamw", bits=8, type="bf16", master=False, model="decoder", hidden=1024, modules=24,
             frozen=0),
        # a 27-block residual network of 16, 32 and 64 channels: hundreds of tiny tensors
        dict(name="adamw_small", op="adamw", bits=32, type="f32", master=False, model="residual", hidden=64, modules=27,
             frozen=9),
    ]


def _spread(rng, low, high):
    """A whole number of low..high, spread over the logarithm; odd ones and multiples of 64 among them."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    shape = rng.randrange(3)
    if shape == 0:
        n = max(low, n // 64 * 64)
    elif shape == 1:
        n |= 1
    n = min(max(n, low), high)
    return n - 2 if n == 3072 else n


def draw(rng):
    op = rng.choice(["linear_forward", "linear_backward", "norm_forward", "norm_backward", "adamw"])
    kind = rng.choice(["bf16", "bf16", "f16"])
    acts = ["none", "relu", "gelu", "gelu_tanh", "silu"]
    if op == "linear_forward":
        inp, out = _spread(rng, 16, 4096), _spread(rng, 16, 4096)
        rows = _spread(rng, 1, min(65536, 65536 * 1024 * 4096 // (inp * out)))
        return dict(op=op, type=kind, rows=rows, inp=inp, out=out, act=rng.choice(acts), bias=rng.random() < 0.8,
                    residual=rng.random() < 0.5, save_z=rng.random() < 0.5)
    if op == "linear_backward":
        inp, out = _spread(rng, 16, 4096), _spread(rng, 16, 4096)
        rows = _spread(rng, 1, min(32768, 32768 * 1024 * 4096 // (inp * out)))
        return dict(op=op, type=kind, rows=rows, inp=inp, out=out, act=rng.choice(acts), act_in=rng.choice(acts),
                    bias=rng.random() < 0.8)
    if op in ("norm_forward", "norm_backward"):
        cols = _spread(rng, 64, 8192)
        rows = _spread(rng, 1, 65536 * 1024 // cols)
        return dict(op=op, type=rng.choice(["bf16", "bf16", "f16", "f32"]), kind=rng.choice(["layer", "rms"]),
                    rows=min(rows, 65536), cols=cols, post=rng.random() < 0.7, pre=rng.random() < 0.8,
                    gate_rows=rng.choice([-1, 0, 1, 256]), affine=rng.random() < 0.8, alpha=rng.choice([1.0, 0.5, 1.25]))
    model = rng.choice(["decoder", "residual"])
    hidden = _spread(rng, 64, 1024) if model == "decoder" else _spread(rng, 8, 128)
    hidden += hidden == 768
    modules = rng.randint(1, 24)
    dtype = rng.choice(["f32", "bf16", "f16"])
    return dict(op=op, bits=rng.choice([8, 32]), type=dtype, master=dtype != "f32" and rng.random() < 0.5, model=model,
                hidden=hidden, modules=modules, frozen=rng.randint(0, modules - 1))


# ----------------------------------------------------------------------------- what a program has in hand

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(20220106 + int(seed))
    return g


def _tensor_sizes(case):
    """(number of values, module, weight decay) of every tensor of the model."""
    h, sizes = case["hidden"], []
    for m in range(case["modules"]):
        if case["model"] == "decoder":
            # four projections, the two hidden products; biases and norms without decay
            for n, wd in (4 * [(h * h, 0.1), (h, 0.0)] +
                          [(4 * h * h, 0.1), (4 * h, 0.0), (4 * h * h, 0.1)] + 5 * [(h, 0.0)]):
                sizes.append((n, m, wd))
        else:
            # two 3 x 3 convolutions and two norms, wider in later thirds
            c = max(1, h >> max(0, 2 - 3 * m // case["modules"]))
            for n, wd in ((9 * c * c, 1e-2), (c, 0.0), (c, 0.0), (9 * c * c, 1e-2), (c, 0.0), (c, 0.0)):
                sizes.append((n, m, wd))
    return sizes


def _adamw_state(case, seed):
    g, t = _gen(seed), TYPES[case["type"]]
    sizes = _tensor_sizes(case)
    first, total = [], 0
    for n, _, _ in sizes:       # every tensor starts on a multiple of 256 of its flat buffer
        first.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    counts = torch.tensor([n for n, _, _ in sizes], device=DEVICE)
    padded = (counts + BLOCK - 1) // BLOCK * BLOCK
    ends = torch.cumsum(padded, 0) - padded + counts
    real = torch.arange(total, device=DEVICE) < torch.repeat_interleave(ends, padded, output_size=total)

    def values(scale):
        return torch.randn(total, generator=g, device=DEVICE).mul_(real).mul_(scale)

    weights = values(0.02)
    # gradients whose size differs from value to value over a few orders, as rows of a layer's do
    spread = torch.exp(2.0 * torch.randn(total // BLOCK, 1, generator=g, device=DEVICE)) * 1e-3
    grads = (values(1.0).view(-1, BLOCK) * spread).view(-1)
    m = values(0.3).view(-1, BLOCK).mul(spread).view(-1)
    v = ((0.2 + torch.rand(total, generator=g, device=DEVICE)).mul_(real).view(-1, BLOCK) * spread * spread).view(-1)
    s = dict(case=case, sizes=sizes, first=first, padded=padded, total=total,
             params=weights.to(t), grads=grads.to(t), masters=weights.clone() if case["master"] else None,
             wd=torch.tensor([wd for _, _, wd in sizes], device=DEVICE),
             module=torch.tensor([k for _, k, _ in sizes], dtype=torch.int64, device=DEVICE),
             steps=torch.tensor([100 + k % 7 for k in range(len(sizes))], dtype=torch.int32, device=DEVICE),
             frozen=(torch.arange(case["modules"], device=DEVICE) < case["frozen"]).to(torch.uint8),
             grad_scale=torch.full((1,), 0.5, device=DEVICE))
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_codes(m, 127)
        root, s["v_scale"] = _to_codes(v.sqrt(), 255)
        s["m"], s["v"] = s["m"].to(torch.int8), torch.where(v > 0, root.clamp(min=1), root).to(torch.uint8)
    else:
        s["m"], s["v"] = m, v
    return s


def _views(s, flat, block=1):
    """Each tensor's part of a flat buffer (block = 256: of a buffer of scales)."""
    if flat is None:
        return None
    return [flat[a // block:(a + n + block - 1) // block if block > 1 else a + n] for a, (n, _, _) in zip(s["first"], s["sizes"])]


def prepare(case, seed):
    if case["op"] == "adamw":
        s = _adamw_state(case, seed)
        if own:   # the optimizer's handle: its table of tensors lives as long as the model does
            from paper_2201_06227_b200 import ops
            s["adamw"] = ops.AdamW(_views(s, s["params"]), _views(s, s["grads"]), _views(s, s["m"]), _views(s, s["v"]),
                                   s["steps"], masters=_views(s, s["masters"]),
                                   m_scales=_views(s, s.get("m_scale"), BLOCK), v_scales=_views(s, s.get("v_scale"), BLOCK),
                                   weight_decay=[wd for _, _, wd in s["sizes"]], modules=[k for _, k, _ in s["sizes"]])
        return s
    g, t = _gen(seed), TYPES[case["type"]]

    def rand(*shape, scale=1.0, base=0.0, kind=t):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale).add_(base).to(kind)

    s = dict(case=case)
    if case["op"].startswith("linear"):
        rows, inp, out = case["rows"], case["inp"], case["out"]
        s["w"] = rand(out, inp, scale=1.0 / math.sqrt(inp))
        if case["op"] == "linear_forward":
            s["x"] = rand(rows, inp)
            s["bias"] = rand(out, scale=0.1) if case["bias"] else None
            s["residual"] = rand(rows, out) if case["residual"] else None
        else:
            s["dy"] = rand(rows, out, scale=1.0 / 64)
            s["z"] = rand(rows, out) if case["act"] != "none" else None
            s["z_in"] = rand(rows, inp) if case["act_in"] != "none" else None
            s["x"] = _act(s["z_in"].float(), case["act_in"]).to(t) if s["z_in"] is not None else rand(rows, inp)
        if own:   # the handle and its workspace, kept for the whole training run
            from paper_2201_06227_b200 import ops
            s["ops"] = ops.Ops(ops.egeria_linear_workspace_bytes(rows, inp, out))
        return s
    rows, cols = case["rows"], case["cols"]
    s["f"] = rand(rows, cols, scale=2.0, base=0.1)
    if case["op"] == "norm_forward":
        s["x"] = rand(rows, cols)
    else:
        s["y"] = rand(rows, cols, scale=1.5)
        s["dy"] = rand(rows, cols, scale=1.0 / 64)
        s["dh"] = rand(rows, cols, scale=1.0 / 64) if case["pre"] else None
        s["stats"] = torch.cat([_stats(s["f"].float(), case["kind"]), _stats(s["y"].float(), case["kind"])], 1)
    for k in ("pre", "post"):
        s["w_" + k] = rand(cols, scale=0.1, base=1.0) if case[k] and case["affine"] else None
        s["b_" + k] = rand(cols, scale=0.1) if case[k] and case["affine"] and case["kind"] == "layer" else None
    groups = 0 if case["gate_rows"] < 0 else 1 if case["gate_rows"] == 0 else -(-rows // case["gate_rows"])
    s["gate"] = rand(groups, cols, scale=0.3, base=0.5) if groups else None
    if own:
        from paper_2201_06227_b200 import ops
        s["ops"] = ops.Ops(ops.egeria_norm_workspace_bytes(rows, cols))
    return s


# ----------------------------------------------------------------------------- the calls

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"linear_forward": _linear_forward, "linear_backward": _linear_backward, "norm_forward": _norm_forward,
            "norm_backward": _norm_backward, "adamw": _adamw}[case["op"]](s, case)


def _run_own(s, case):
    if case["op"] == "linear_forward":
        return s["ops"].egeria_linear_forward(s["x"], s["w"], bias=s["bias"], act=case["act"], residual=s["residual"],
                                              save_z=case["save_z"])
    if case["op"] == "linear_backward":
        return s["ops"].egeria_linear_backward(s["dy"], s["x"], s["w"], z=s["z"], act=case["act"], z_in=s["z_in"],
                                               act_in=case["act_in"], need_db=case["bias"])
    if case["op"] == "norm_forward":
        return s["ops"].egeria_norm_forward(s["x"], s["f"], gate=s["gate"], gate_rows=max(case["gate_rows"], 0),
                                            w_post=s["w_post"], b_post=s["b_post"], w_pre=s["w_pre"], b_pre=s["b_pre"],
                                            kind=case["kind"], post=case["post"], pre=case["pre"], alpha=case["alpha"],
                                            eps=NORM_EPS)
    if case["op"] == "norm_backward":
        return s["ops"].egeria_norm_backward(s["dy"], s["dh"], s["y"], s["f"], s["stats"], gate=s["gate"],
                                             gate_rows=max(case["gate_rows"], 0), w_post=s["w_post"], b_post=s["b_post"],
                                             w_pre=s["w_pre"], b_pre=s["b_pre"], kind=case["kind"], post=case["post"],
                                             pre=case["pre"], alpha=case["alpha"])
    s["adamw"].egeria_adamw_step(LR, BETA1, BETA2, ADAM_EPS, grad_scale=s["grad_scale"], frozen=s["frozen"])
    return _adamw_outputs(s, case)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        k = 2.0 * math.sqrt(2.0 / math.pi)
        p = torch.sigmoid(k * (z + 0.044715 * z * z * z))
        return p + z * p * (1.0 - p) * k * (1.0 + 3.0 * 0.044715 * z * z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * (1.0 - p)
    return torch.ones_like(z)


def _linear_forward(s, case):
    t = s["x"].dtype
    z = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        z += s["bias"].float()
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(t), z.to(t)) if case["save_z"] else y.to(t)


def _linear_backward(s, case):
    t = s["x"].dtype
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(s["z"].float(), case["act"])
    dx = dz @ s["w"].float()
    if s["z_in"] is not None:
        dx = dx * _act_slope(s["z_in"].float(), case["act_in"])
    dw = dz.t() @ s["x"].float()
    return dx.to(t), dw.to(t), dz.sum(0).to(t) if case["bias"] else None


def _stats(a, kind):
    """Mean (0 for the root-mean-square norm) and 1 / deviation of every row."""
    mean = a.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(a[:, :1])
    return torch.cat([mean, 1.0 / torch.sqrt(((a - mean) ** 2).mean(1, keepdim=True) + NORM_EPS)], 1)


def _gate(s, case):
    """The gate of every row, as it broadcasts over [rows, cols]."""
    if s["gate"] is None:
        return torch.ones(1, 1, device=DEVICE)
    if case["gate_rows"] == 0:
        return s["gate"].float()
    return torch.repeat_interleave(s["gate"].float(), case["gate_rows"], 0)[:case["rows"]]


def _affine(a, w, b):
    if w is not None:
        a = a * w.float()
    return a if b is None else a + b.float()


def _norm_forward(s, case):
    t = s["x"].dtype
    f, blank = s["f"].float(), torch.zeros(case["rows"], 2, device=DEVICE)
    post = pre = blank
    if case["post"]:
        post = _stats(f, case["kind"])
        f = _affine((f - post[:, :1]) * post[:, 1:], s["w_post"], s["b_post"])
    y = case["alpha"] * s["x"].float() + _gate(s, case) * f
    h = None
    if case["pre"]:
        pre = _stats(y, case["kind"])
        h = _affine((y - pre[:, :1]) * pre[:, 1:], s["w_pre"], s["b_pre"]).to(t)
    return y.to(t), h, torch.cat([post, pre], 1)


def _norm_rows(d, hat, inv, w, kind):
    """The gradient of a norm's input from that of its output."""
    if w is not None:
        d = d * w.float()
    lean = d.mean(1, keepdim=True) if kind == "layer" else 0.0
    return inv * (d - lean - hat * (d * hat).mean(1, keepdim=True))


def _norm_backward(s, case):
    t, st = s["y"].dtype, s["stats"]
    total, out = s["dy"].float(), dict(dx=None, df=None, dgate=None, dw_post=None, db_post=None, dw_pre=None, db_pre=None)
    if case["pre"]:
        hat, dh = (s["y"].float() - st[:, 2:3]) * st[:, 3:4], s["dh"].float()
        total = total + _norm_rows(dh, hat, st[:, 3:4], s["w_pre"], case["kind"])
        out["dw_pre"] = (dh * hat).sum(0).to(t) if s["w_pre"] is not None else None
        out["db_pre"] = dh.sum(0).to(t) if s["b_pre"] is not None else None
    out["dx"] = (case["alpha"] * total).to(t)
    dn, f = total * _gate(s, case), s["f"].float()
    if case["post"]:
        hat = (f - st[:, 0:1]) * st[:, 1:2]
        out["df"] = _norm_rows(dn, hat, st[:, 1:2], s["w_post"], case["kind"]).to(t)
        out["dw_post"] = (dn * hat).sum(0).to(t) if s["w_post"] is not None else None
        out["db_post"] = dn.sum(0).to(t) if s["b_post"] is not None else None
        f = _affine(hat, s["w_post"], s["b_post"])
    else:
        out["df"] = dn.to(t)
    if s["gate"] is not None:
        f = total * f
        if case["gate_rows"] == 0:
            out["dgate"] = f.sum(0, keepdim=True).to(t)
        else:
            group = torch.arange(case["rows"], device=DEVICE) // case["gate_rows"]
            out["dgate"] = torch.zeros_like(s["gate"], dtype=torch.float32).index_add_(0, group, f).to(t)
    return out


def _to_codes(a, most):
    """8-bit codes: the size of a value is (code / most)^2 of the largest size in its block of 256."""
    a = a.view(-1, BLOCK)
    scale = a.abs().amax(1, keepdim=True)
    code = torch.round(most * torch.sqrt(a.abs() / torch.where(scale > 0, scale, torch.ones_like(scale))))
    return (torch.sign(a) * code).view(-1), scale.view(-1)


def _from_codes(code, scale, most):
    c = code.float().view(-1, BLOCK)
    return (c * c.abs() * (scale.view(-1, 1) / (most * most))).view(-1)


def _adamw(s, case):
    each = lambda v: torch.repeat_interleave(v, s["padded"], output_size=s["total"])  # noqa: E731
    live_tensor = s["frozen"][s["module"]] == 0
    live = each(live_tensor)
    s["steps"] += live_tensor.to(torch.int32)
    step = s["steps"].double()
    fix1, fix2 = (1.0 - BETA1 ** step).float(), (1.0 - BETA2 ** step).float()
    g = s["grads"].float() * s["grad_scale"]
    small = case["bits"] == 8
    m = _from_codes(s["m"], s["m_scale"], 127) if small else s["m"]
    v = _from_codes(s["v"], s["v_scale"], 255) ** 2 if small else s["v"]
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    del g
    p = s["masters"] if s["masters"] is not None else s["params"].float()
    moved = p * (1.0 - LR * each(s["wd"])) - each(LR / fix1) * m / (torch.sqrt(v) * each(1.0 / torch.sqrt(fix2)) + ADAM_EPS)
    moved = torch.where(live, moved, p)
    s["params"].copy_(torch.where(live, moved.to(s["params"].dtype), s["params"]))
    if s["masters"] is not None:
        s["masters"].copy_(moved)
    if small:
        blocks = live.view(-1, BLOCK)[:, 0]
        code, scale = _to_codes(m, 127)
        s["m"].copy_(torch.where(live, code.to(torch.int8), s["m"]))
        s["m_scale"].copy_(torch.where(blocks, scale, s["m_scale"]))
        code, scale = _to_codes(torch.sqrt(v), 255)
        code = torch.where(v > 0, code.clamp(min=1), code)
        s["v"].copy_(torch.where(live, code.to(torch.uint8), s["v"]))
        s["v_scale"].copy_(torch.where(blocks, scale, s["v_scale"]))
    else:
        s["m"].copy_(torch.where(live, m, s["m"]))
        s["v"].copy_(torch.where(live, v, s["v"]))
    return _adamw_outputs(s, case)


def _adamw_outputs(s, case):
    out = dict(params=s["params"], steps=s["steps"])
    if s["masters"] is not None:
        out["masters"] = s["masters"]
    if case["bits"] == 8:
        # what the codes stand for; a code of eight bits is worth no more digits than bfloat16 has
        out["m"] = s["m"].float().view(-1, BLOCK)
        out["m"] = (out["m"] * out["m"].abs() * (s["m_scale"] / 127.0 ** 2).view(-1, 1)).to(torch.bfloat16)
        out["v"] = s["v"].float().view(-1, BLOCK)
        out["v"] = (out["v"] ** 4 * (s["v_scale"] / 255.0 ** 2).view(-1, 1) ** 2).to(torch.bfloat16)
        out["m_scale"], out["v_scale"] = s["m_scale"], s["v_scale"]
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "linear_forward":
        r, i, o, b = case["rows"], case["inp"], case["out"], BYTES[case["type"]]
        n = r * i + o * i + r * o * (1 + case["residual"] + case["save_z"]) + o * case["bias"]
        return {"bytes": n * b, "flops": 2 * r * i * o}
    if case["op"] == "linear_backward":
        r, i, o, b = case["rows"], case["inp"], case["out"], BYTES[case["type"]]
        n = r * o * (1 + (case["act"] != "none")) + r * i * (2 + (case["act_in"] != "none")) + 2 * o * i + o * case["bias"]
        return {"bytes": n * b, "flops": 4 * r * i * o}
    if case["op"] in ("norm_forward", "norm_backward"):
        r, c, b = case["rows"], case["cols"], BYTES[case["type"]]
        weights = (case["pre"] + case["post"]) * case["affine"] * (2 if case["kind"] == "layer" else 1)
        gates = 0 if case["gate_rows"] < 0 else 1 if case["gate_rows"] == 0 else -(-r // case["gate_rows"])
        if case["op"] == "norm_forward":
            return {"bytes": r * c * b * (3 + case["pre"]) + c * b * (weights + gates) + 16 * r, "flops": 16 * r * c}
        return {"bytes": r * c * b * (4 + 2 * case["pre"]) + 2 * c * b * (weights + gates) + 16 * r, "flops": 30 * r * c}
    live = sum(n for n, m, _ in _tensor_sizes(case) if m >= case["frozen"])
    each = BYTES[case["type"]] * (2 if case["master"] else 3) + (8 if case["master"] else 0)
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": int(live * (each + moments)), "flops": 15 * live}


# ----------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"].startswith("linear"):
        return _exact_linear(d, case)
    if case["op"].startswith("norm"):
        return _exact_norm(d, case)
    return _exact_adamw(d, case)


def _exact_act(z, act):
    """Value and slope of the activation."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        half = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * half, half + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    u = z if act == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
    du = 1.0 if act == "silu" else math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
    p = 1 / (1 + torch.exp(-u))
    return z * p, p + z * du * p / (1 + torch.exp(u))


def _exact_linear(d, case):
    if case["op"] == "linear_forward":
        z = torch.einsum("ri,oi->ro", d["x"], d["w"])
        z = z if d["bias"] is None else z + d["bias"]
        y = _exact_act(z, case["act"])[0] + (0.0 if d["residual"] is None else d["residual"])
        return (y, z) if case["save_z"] else y
    dz = d["dy"] if d["z"] is None else d["dy"] * _exact_act(d["z"], case["act"])[1]
    dx = torch.einsum("ro,oi->ri", dz, d["w"])
    if d["z_in"] is not None:
        dx *= _exact_act(d["z_in"], case["act_in"])[1]
    return dx, torch.einsum("ro,ri->oi", dz, d["x"]), torch.einsum("ro->o", dz) if case["bias"] else None


def _exact_norm(d, case):
    layer, rows, cols = case["kind"] == "layer", case["rows"], case["cols"]
    if d["gate"] is None:
        gate, group = torch.ones(1, cols, dtype=torch.float64, device=DEVICE), None
    else:
        group = torch.arange(rows, device=DEVICE) // case["gate_rows"] if case["gate_rows"] else torch.zeros(rows, dtype=torch.int64, device=DEVICE)
        gate = d["gate"][group] if case["gate_rows"] else d["gate"]
    one, none = torch.ones(cols, dtype=torch.float64, device=DEVICE), torch.zeros(cols, dtype=torch.float64, device=DEVICE)
    w = {k: one if d["w_" + k] is None else d["w_" + k] for k in ("pre", "post")}
    b = {k: none if d["b_" + k] is None else d["b_" + k] for k in ("pre", "post")}
    if case["op"] == "norm_forward":
        def normed(a, k):
            mean = a.sum(1, keepdim=True) / cols * layer
            inv = ((a - mean).square().sum(1, keepdim=True) / cols + NORM_EPS).rsqrt()
            return (a - mean) * inv * w[k] + b[k], mean, inv
        zero = torch.zeros(rows, 1, dtype=torch.float64, device=DEVICE)
        f, mean, inv = normed(d["f"], "post") if case["post"] else (d["f"], zero, zero)
        y = torch.addcmul(case["alpha"] * d["x"], gate, f)
        h, mean_y, inv_y = normed(y, "pre") if case["pre"] else (None, zero, zero)
        return y, h, torch.hstack([mean, inv, mean_y, inv_y])

    def through(g, a, mean, inv):
        """Gradient of a row's input from g, that of its normalised values: the projection off 1 and off them."""
        hat = (a - mean) * inv
        along = torch.einsum("rc,rc->r", g, hat)[:, None] / cols
        return (g - hat * along - (g.sum(1, keepdim=True) / cols if layer else 0.0)) * inv, hat

    out = dict(dx=None, df=None, dgate=None, dw_post=None, db_post=None, dw_pre=None, db_pre=None)
    st, total = d["stats"], d["dy"]
    if case["pre"]:
        through_y, hat = through(d["dh"] * w["pre"], d["y"], st[:, 2:3], st[:, 3:4])
        total = total + through_y
        out["dw_pre"] = torch.einsum("rc,rc->c", d["dh"], hat) if d["w_pre"] is not None else None
        out["db_pre"] = torch.einsum("rc->c", d["dh"]) if d["b_pre"] is not None else None
    out["dx"], dn, made = total * case["alpha"], total * gate, d["f"]
    if case["post"]:
        out["df"], hat = through(dn * w["post"], d["f"], st[:, 0:1], st[:, 1:2])
        out["dw_post"] = torch.einsum("rc,rc->c", dn, hat) if d["w_post"] is not None else None
        out["db_post"] = torch.einsum("rc->c", dn) if d["b_post"] is not None else None
        made = hat * w["post"] + b["post"]
    else:
        out["df"] = dn
    if group is not None:
        out["dgate"] = torch.zeros_like(d["gate"]).index_add_(0, group, total * made)
    return out


def _exact_adamw(d, case):
    size = d["padded"]
    live = ~d["frozen"].bool()[d["module"]]
    steps = d["steps"] + live
    full = lambda v: torch.repeat_interleave(v, size, output_size=d["total"])  # noqa: E731
    on = full(live)
    g = d["grads"] * d["grad_scale"]
    if case["bits"] == 8:
        m0 = torch.sign(d["m"].double()) * ((d["m"].double() / 127) ** 2).view(-1, BLOCK).mul(d["m_scale"].view(-1, 1)).view(-1)
        v0 = ((d["v"].double() / 255) ** 2).view(-1, BLOCK).mul(d["v_scale"].view(-1, 1)).view(-1).square()
    else:
        m0, v0 = d["m"], d["v"]
    m = torch.lerp(g, m0, BETA1)
    v = torch.lerp(g.square(), v0, BETA2)
    p = d["masters"] if d["masters"] is not None else d["params"]
    t = steps.double()
    change = (m / full(1 - BETA1 ** t)) / ((v / full(1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    new = torch.where(on, p - LR * (change + full(d["wd"]) * p), p)
    out = dict(params=torch.where(on, new, d["params"]), steps=steps)
    del change
    if d["masters"] is not None:
        out["masters"] = new
    if case["bits"] == 32:
        out["m"], out["v"] = torch.where(on, m, m0), torch.where(on, v, v0)
        return out

    def kept(a, most):
        rows = a.view(-1, BLOCK)
        top = rows.abs().amax(1, keepdim=True)
        code = torch.round(torch.sqrt(rows.abs() / top.clamp(min=1e-300)) * most)
        code = torch.where((rows != 0) & (most == 255), code.clamp(min=1), code)
        return torch.sign(rows) * (code / most) ** 2 * top, top.view(-1)

    alive = on.view(-1, BLOCK)[:, :1]
    m8, top_m = kept(m, 127)
    v8, top_v = kept(v.sqrt(), 255)
    out["m"] = torch.where(alive, m8, m0.view(-1, BLOCK))
    out["v"] = torch.where(alive, v8.square(), v0.view(-1, BLOCK))
    out["m_scale"] = torch.where(alive.view(-1), top_m, d["m_scale"])
    out["v_scale"] = torch.where(alive.view(-1), top_v, d["v_scale"])
    return out
