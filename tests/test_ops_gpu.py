"""GPU parity of the training operators against plain implementations in 64 bits.

Tolerances come from the arithmetic, not from what was seen: an output of p bits is rounded once
(u = 2^-8 for bfloat16, 2^-11 for float16, 2^-24 for float32), a sum of n products in 32 bits is off by at most
(n + 8) 2^-23 times the sum of the products' sizes, and an activation is off by 2^-15 of its value (the
approximate exponential).  Each bound is evaluated element by element, in 64 bits.
"""
import math

import pytest
import torch

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}  # below: absolute error
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def rand(*shape, dtype=torch.bfloat16, seed=0, scale=1.0, base=0.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(1234 + seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale + base).to(dtype)


def close(got, ref, tol, what=""):
    got = got.double()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - ref).abs() / tol).max()):.2f} times the bound, "
                           f"first at {bad.nonzero()[0].tolist()}")


def act64(z, act):
    """Value and slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(8 / math.pi)
    u, du = (z, torch.ones_like(z)) if act == "silu" else (c * (z + 0.044715 * z ** 3), c * (1 + 3 * 0.044715 * z ** 2))
    p = torch.sigmoid(u)
    return z * p, p + z * du * p * torch.sigmoid(-u)


def handle(rows, inp, out):
    return ops.Ops(ops.egeria_linear_workspace_bytes(rows, inp, out), DEV)


def check_forward(o, x, w, bias, act, residual, save_z, out=None):
    base = None if residual is None else residual.clone()
    got = o.egeria_linear_forward(x, w, bias=bias, act=act, residual=residual, save_z=save_z, out=out)
    y, z = got if save_z else (got, None)
    t, k = x.dtype, x.shape[1]
    xd, wd = x.double(), w.double()
    zr = xd @ wd.t()
    size = xd.abs() @ wd.abs().t()
    if bias is not None:
        zr, size = zr + bias.double(), size + bias.double().abs()
    err = (k + 8) * 2.0 ** -23 * size
    yr = act64(zr, act)[0]
    if z is not None:
        close(z, zr, U[t] * zr.abs() + err + TINY[t], "z")
    tol = 1.2 * err + 2.0 ** -15 * yr.abs()     # no activation is steeper than 1.13
    if base is not None:
        yr = yr + base.double()
        tol = tol + 2.0 ** -23 * yr.abs()
    close(y, yr, U[t] * yr.abs() + tol + TINY[t], "y")


def check_backward(o, dy, x, w, z, act, z_in, act_in, **need):
    dx, dw, db = o.egeria_linear_backward(dy, x, w, z=z, act=act, z_in=z_in, act_in=act_in, **need)
    t, (rows, n) = dy.dtype, dy.shape
    g = dy.double()
    rounded = 0.0
    if act != "none":
        g = g * act64(z.double(), act)[1]
        rounded = U[t] + 2.0 ** -14       # dz as the products' operand, and the slope's own error
    if dx is not None:
        wd = w.double()
        ref, size = g @ wd, g.abs() @ wd.abs()
        tol = (rounded + (n + 8) * 2.0 ** -23) * size + TINY[t] * wd.abs().sum(0)
        if act_in != "none":
            slope = act64(z_in.double(), act_in)[1]
            ref, tol = ref * slope, tol * slope.abs() + 2.0 ** -14 * (ref * slope).abs() + 2.0 ** -20 * ref.abs()
        close(dx, ref, U[t] * ref.abs() + tol + TINY[t], "dx")
    if dw is not None:
        xd = x.double()
        ref, size = g.t() @ xd, g.abs().t() @ xd.abs()
        close(dw, ref, U[t] * ref.abs() + (rounded + (rows + 8) * 2.0 ** -23) * size + TINY[t] * (1 + xd.abs().sum(0)), "dw")
    if db is not None:
        ref, size = g.sum(0), g.abs().sum(0)
        close(db, ref, U[t] * ref.abs() + ((rows + 8) * 2.0 ** -23 + 2.0 ** -14) * size + TINY[t], "db")
    return dx, dw, db


# ----------------------------------------------------------------------------- linear layers

SIZES = [(1, 64, 64), (2, 8, 1), (3, 1024, 512), (5, 100, 333), (8, 513, 70), (9, 64, 32), (17, 16, 16), (64, 1, 5), (100, 72, 136),
         (128, 256, 256), (129, 1000, 257), (256, 4096, 128), (300, 65, 1032), (333, 1001, 519), (512, 768, 768), (1000, 24, 3000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inp,out", SIZES)
def test_linear_forward(rows, inp, out, dtype):
    o = handle(rows, inp, out)
    s = rows + inp + out
    x, w = rand(rows, inp, dtype=dtype, seed=s), rand(out, inp, dtype=dtype, seed=s + 1, scale=inp ** -0.5)
    b, r = rand(out, dtype=dtype, seed=s + 2), rand(rows, out, dtype=dtype, seed=s + 3)
    check_forward(o, x, w, b, ACTS[s % 5], r, True)
    check_forward(o, x, w, None, "none", None, False)
    o.check_device_status()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [4, 200])
def test_linear_activations_over_a_wide_range(act, rows):
    o = handle(rows, 128, 512)
    x, w = rand(rows, 128, seed=1, scale=3.0), rand(512, 128, seed=2, scale=0.3)
    check_forward(o, x, w, rand(512, seed=3, scale=4.0), act, None, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inp,out", SIZES)
def test_linear_backward(rows, inp, out, dtype):
    o = handle(rows, inp, out)
    s = rows + inp + out
    dy, x = rand(rows, out, dtype=dtype, seed=s, scale=0.1), rand(rows, inp, dtype=dtype, seed=s + 1)
    w = rand(out, inp, dtype=dtype, seed=s + 2, scale=inp ** -0.5)
    z, z_in = rand(rows, out, dtype=dtype, seed=s + 3, scale=2.0), rand(rows, inp, dtype=dtype, seed=s + 4, scale=2.0)
    check_backward(o, dy, x, w, z, ACTS[s % 5], z_in, ACTS[(s + 2) % 5])
    check_backward(o, dy, x, w, None, "none", None, "none")
    o.check_device_status()


@pytest.mark.parametrize("rows,inp,out", [(4096, 768, 768), (2048, 1024, 4096), (16384, 256, 512)])
def test_linear_larger(rows, inp, out):
    """Whole waves of tiles, split sums and pairs of thread blocks, at sizes the planner sends there."""
    o = handle(rows, inp, out)
    x, w = rand(rows, inp, seed=1), rand(out, inp, seed=2, scale=inp ** -0.5)
    check_forward(o, x, w, rand(out, seed=3), "gelu_tanh", rand(rows, out, seed=4), True)
    check_backward(o, rand(rows, out, seed=5, scale=0.1), x, w, rand(rows, out, seed=6), "gelu_tanh", x, "gelu")
    o.check_device_status()


@pytest.mark.parametrize("dx,dw,db", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 0, 1)])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_linear_backward_of_parts(dx, dw, db, act):
    """A frozen layer needs only dx, the first layer that trains no dx."""
    o = handle(150, 96, 80)
    dy, x, w, z = rand(150, 80, seed=1), rand(150, 96, seed=2), rand(80, 96, seed=3), rand(150, 80, seed=4)
    got = check_backward(o, dy, x if dw or not dx else None, w if dx else None, z if act != "none" else None, act, None, "none",
                         need_dx=bool(dx), need_dw=bool(dw), need_db=bool(db))
    assert [g is not None for g in got] == [bool(dx), bool(dw), bool(db)]


@pytest.mark.parametrize("shift,pitch", [(0, 72), (1, 65), (3, 80), (8, 96), (16, 64)])
@pytest.mark.parametrize("rows", [5, 140])
def test_linear_strides_and_offsets(shift, pitch, rows):
    """Every operand a view with its own offset and row pitch; what lies between the rows stays as it was."""
    inp = out = 64

    def view(seed, n, fill=0.0):
        buf = torch.full((shift + n * pitch + 64,), fill, dtype=torch.bfloat16, device=DEV)
        v = buf[shift:shift + n * pitch].view(n, pitch)[:, :64]
        v.copy_(rand(n, 64, seed=seed, scale=0.3))
        return buf, v

    o = handle(rows, inp, out)
    x, w, r, z = (view(k, n)[1] for k, n in ((1, rows), (2, out), (3, rows), (4, rows)))
    buf, y = view(5, rows, 7.0)
    check_forward(o, x, w, rand(out, seed=6), "silu", r, False, out=y)
    check_backward(o, r, x, w, z, "gelu", z, "silu")
    if pitch > 64:
        gaps = buf[shift:shift + rows * pitch].view(rows, pitch)[:, 64:]
        assert (gaps == 7.0).all()
    assert (buf[:shift] == 7.0).all() and (buf[shift + rows * pitch:] == 7.0).all()


@pytest.mark.parametrize("rows", [3, 200])
def test_linear_adds_onto_the_residual_in_place(rows):
    o = handle(rows, 128, 96)
    x, w, r = rand(rows, 128, seed=1), rand(96, 128, seed=2, scale=0.1), rand(rows, 96, seed=3)
    separate = o.egeria_linear_forward(x, w, residual=r, act="gelu")
    o.egeria_linear_forward(x, w, residual=r, act="gelu", out=r)
    assert torch.equal(r, separate)


def test_linear_no_rows():
    o = handle(0, 32, 16)
    x, w = torch.empty(0, 32, dtype=torch.bfloat16, device=DEV), rand(16, 32)
    assert o.egeria_linear_forward(x, w).shape == (0, 16)
    dx, dw, db = o.egeria_linear_backward(torch.empty(0, 16, dtype=torch.bfloat16, device=DEV), x, w)
    assert dx.shape == (0, 32) and not dw.any() and not db.any()


@pytest.mark.parametrize("rows", [2, 130])
def test_linear_keeps_infinities_and_nans_to_their_rows(rows):
    o = handle(rows, 64, 64)
    x, w = rand(rows, 64, seed=1), rand(64, 64, seed=2)
    x[0, 3], x[1, 5] = float("inf"), float("nan")
    y = o.egeria_linear_forward(x, w).float()
    ref = x.float() @ w.float().t()
    assert torch.isnan(y[1]).all() and torch.isinf(y[0]).all()
    assert torch.equal(torch.sign(y[0]), torch.sign(ref[0]))
    assert torch.isfinite(y[2:]).all()


def test_linear_same_bits_every_time():
    """Split sums are added in a fixed order."""
    o = handle(4000, 256, 256)
    dy, x, w = rand(4000, 256, seed=1), rand(4000, 256, seed=2), rand(256, 256, seed=3)
    first = o.egeria_linear_backward(dy, x, w)
    for _ in range(5):
        for a, b in zip(first, o.egeria_linear_backward(dy, x, w)):
            assert torch.equal(a, b)


def test_linear_gradients_against_differences():
    """The gradients of a scalar of the layer against central differences of the forward call."""
    rows, inp, out = 40, 48, 56
    o = handle(rows, inp, out)
    t = torch.float16
    x, w, b, c = rand(rows, inp, dtype=t, seed=1), rand(out, inp, dtype=t, seed=2, scale=0.15), rand(out, dtype=t, seed=3), rand(rows, out, dtype=t, seed=4)

    def loss(x, w, b):
        return float((o.egeria_linear_forward(x, w, bias=b, act="gelu").double() * c.double()).sum())

    z = o.egeria_linear_forward(x, w, bias=b, act="gelu", save_z=True)[1]
    dx, dw, db = o.egeria_linear_backward(c, x, w, z=z, act="gelu")
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        args = [x, w, b]
        d = rand(*grad.shape, dtype=t, seed=20 + which)
        step = 2.0 ** -4
        up, down = list(args), list(args)
        up[which] = (args[which].double() + step * d.double()).to(t)
        down[which] = (args[which].double() - step * d.double()).to(t)
        real = (up[which].double() - down[which].double())          # the step that the rounded inputs took
        slope = float((grad.double() * real).sum())
        # rounding of rows * out outputs of size ~1 weighted by c, and the third derivative over the step
        noise = 2 * 2.0 ** -11 * math.sqrt(rows * out) * 4 + 0.02 * abs(slope)
        assert abs(loss(*up) - loss(*down) - slope) <= noise + 3.0, (which, loss(*up) - loss(*down), slope)


def test_linear_refusals():
    o = handle(16, 64, 64)
    x, w = rand(16, 64), rand(64, 64)
    with pytest.raises(ValueError):
        o.egeria_linear_forward(x, w, act="tanh")
    with pytest.raises(ValueError):
        o.egeria_linear_forward(x, rand(64, 32))
    with pytest.raises(ValueError):
        o.egeria_linear_forward(x, w, bias=rand(63))
    with pytest.raises(ValueError):
        o.egeria_linear_forward(x, w.t())                     # a row's values are not consecutive
    with pytest.raises(ValueError):
        o.egeria_linear_forward(x.cpu(), w)
    with pytest.raises(ValueError):
        o.egeria_linear_backward(x, x, None)
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_linear_forward(x.float(), w.float())
    assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_linear_backward(x, x, w, act="relu")          # no z
    assert e.value.status == eg.ERR_INVALID_ARG
    small = ops.Ops(device=DEV)
    with pytest.raises(eg.EgeriaError) as e:
        small.egeria_linear_forward(rand(2000, 512), rand(512, 512))
    assert e.value.status == eg.ERR_WORKSPACE


def test_linear_on_another_stream_and_in_a_graph():
    o = handle(300, 128, 128)
    x, w = rand(300, 128, seed=1), rand(128, 128, seed=2)
    want = o.egeria_linear_forward(x, w, act="relu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = o.egeria_linear_forward(x, w, act="relu", stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o.egeria_linear_forward(x, w, act="relu", out=out, stream=torch.cuda.current_stream())
    for k in range(3):
        x.copy_(rand(300, 128, seed=50 + k))
        g.replay()
        replayed = out.clone()
        assert torch.equal(replayed, o.egeria_linear_forward(x, w, act="relu"))


# ----------------------------------------------------------------------------- residual norms

def stats64(a, kind, eps=1e-5):
    mean = a.mean(1, keepdim=True) * (kind == "layer")
    return mean, 1 / torch.sqrt(((a - mean) ** 2).mean(1, keepdim=True) + eps)


def norm64(a, w, b, kind):
    """(normalised with weights, bound of its error over 2^-24 (cols + 64))."""
    mean, inv = stats64(a, kind)
    w = torch.ones(a.shape[1], device=DEV, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    return (a - mean) * inv * w + b, (2 * (a - mean).abs() + mean.abs() + a.abs().mean(1, keepdim=True)) * inv * w.abs() + b.abs()


def gate64(gate, gate_rows, rows):
    if gate is None:
        return 1.0
    return gate.double().view(1, -1) if gate_rows == 0 else gate.double().repeat_interleave(gate_rows, 0)[:rows]


def norm_inputs(rows, cols, dtype, ptype, kind, post, pre, gate_rows, affine, seed):
    s = dict(x=rand(rows, cols, dtype=dtype, seed=seed), f=rand(rows, cols, dtype=dtype, seed=seed + 1, scale=2.0, base=0.3))
    s["gate"] = None if gate_rows is None else rand(1 if gate_rows == 0 else -(-rows // gate_rows), cols, dtype=ptype, seed=seed + 2, base=0.5)
    for k, on in (("post", post), ("pre", pre)):
        s["w_" + k] = rand(cols, dtype=ptype, seed=seed + 3, scale=0.2, base=1.0) if affine and on else None
        s["b_" + k] = rand(cols, dtype=ptype, seed=seed + 4) if affine and on and kind == "layer" else None
    return s


def check_norm(o, s, kind, post, pre, gate_rows, alpha, dtype):
    args = {k: s[k] for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    opts = dict(kind=kind, post=post, pre=pre, alpha=alpha, gate_rows=gate_rows or 0)
    y, h, st = o.egeria_norm_forward(s["x"], s["f"], **args, **opts)
    rows, cols = s["x"].shape
    xd, fd = s["x"].double(), s["f"].double()
    g = gate64(s["gate"], gate_rows, rows)
    n, n_size = norm64(fd, s["w_post"], s["b_post"], kind) if post else (fd, fd.abs())
    yr = alpha * xd + g * n
    c = 2.0 ** -24 * (cols + 64)
    err = c * (abs(alpha) * xd.abs() + (g * n_size).abs())
    close(y, yr, U[dtype] * yr.abs() + err + TINY[dtype], "y")
    if pre:
        hr, h_size = norm64(yr, s["w_pre"], s["b_pre"], kind)
        mean, inv = stats64(yr, kind)
        wp = 1.0 if s["w_pre"] is None else s["w_pre"].double().abs()
        spread = (err + err.mean(1, keepdim=True) * (1 + ((yr - mean) * inv).abs())) * inv * wp * 2
        close(h, hr, U[dtype] * hr.abs() + c * h_size * 4 + spread + TINY[dtype], "h")
    want = torch.cat([*(stats64(fd, kind) if post else [torch.zeros(rows, 1, device=DEV, dtype=torch.float64)] * 2),
                      *(stats64(yr, kind) if pre else [torch.zeros(rows, 1, device=DEV, dtype=torch.float64)] * 2)], 1)
    near = torch.cat([c * fd.abs().mean(1, keepdim=True), 4 * c * want[:, 1:2],
                      c * yr.abs().mean(1, keepdim=True) + err.mean(1, keepdim=True),
                      (4 * c + 2 * err.mean(1, keepdim=True) * want[:, 3:4]) * want[:, 3:4]], 1)
    close(st, want, 2 * near + 1e-30, "stats")
    # backward, from the stored y and statistics
    dy, dh = rand(rows, cols, dtype=dtype, seed=91, scale=0.1), rand(rows, cols, dtype=dtype, seed=92, scale=0.1) if pre else None
    got = o.egeria_norm_backward(dy, dh, y, s["f"], st, **args, **opts)
    sd = st.double()

    def through(d, a, mean, inv, w):
        """(gradient, bound) of a norm's input."""
        hat = (a - mean) * inv
        dw = d if w is None else d * w.double()
        lean = dw.mean(1, keepdim=True) * (kind == "layer")
        along = (dw * hat).mean(1, keepdim=True)
        size = inv * (dw.abs() + dw.abs().mean(1, keepdim=True) + hat.abs() * (dw * hat).abs().mean(1, keepdim=True))
        return inv * (dw - lean - hat * along), size, hat

    tot, tot_err = dy.double(), 0.0
    if pre:
        dhd = dh.double()
        extra, size, hat = through(dhd, y.double(), sd[:, 2:3], sd[:, 3:4], s["w_pre"])
        tot, tot_err = tot + extra, c * 4 * size
        if s["w_pre"] is not None:
            sums(got["dw_pre"], dhd * hat, "dw_pre")
        if s["b_pre"] is not None:
            sums(got["db_pre"], dhd, "db_pre")
    tot_err = tot_err + 2.0 ** -23 * tot.abs()
    close(got["dx"], alpha * tot, U[dtype] * (alpha * tot).abs() + abs(alpha) * tot_err + TINY[dtype], "dx")
    d, d_err = tot * g, (tot_err * g).abs() if not isinstance(g, float) else tot_err
    made, made_size = fd, fd.abs()
    if post:
        ref, size, hat = through(d, fd, sd[:, 0:1], sd[:, 1:2], s["w_post"])
        w = 1.0 if s["w_post"] is None else s["w_post"].double().abs()
        grow = sd[:, 1:2] * ((d_err * w) + (d_err * w).mean(1, keepdim=True) + hat.abs() * (d_err * w * hat.abs()).mean(1, keepdim=True))
        close(got["df"], ref, U[dtype] * ref.abs() + c * 4 * size + grow + TINY[dtype], "df")
        if s["w_post"] is not None:
            sums(got["dw_post"], d * hat, "dw_post", (d_err * hat.abs()).sum(0))
        if s["b_post"] is not None:
            sums(got["db_post"], d, "db_post", d_err.sum(0))
        made = hat * (1.0 if s["w_post"] is None else s["w_post"].double()) + (0.0 if s["b_post"] is None else s["b_post"].double())
        made_size = (hat * w).abs() + (0.0 if s["b_post"] is None else s["b_post"].double().abs())
    else:
        close(got["df"], d, U[dtype] * d.abs() + d_err + 2.0 ** -23 * d.abs() + TINY[dtype], "df")
    if s["gate"] is not None:
        part = tot * made
        part_err = tot_err * made.abs() + 2.0 ** -22 * tot.abs() * made_size     # the branch's value is rounded where its parts cancel
        span = gate_rows or rows
        for k in range(s["gate"].shape[0]):
            rows_k = slice(k * span, (k + 1) * span)
            sums(got["dgate"][k], part[rows_k], f"dgate[{k}]", part_err[rows_k].sum(0))


def sums(got, terms, what, err=0.0):
    ref, size = terms.sum(0), terms.abs().sum(0)
    close(got, ref, U[got.dtype] * ref.abs() + (terms.shape[0] + 64) * 2.0 ** -23 * size + err + TINY[got.dtype], what)


NORM_SIZES = [(1, 1), (1, 64), (3, 7), (5, 256), (2, 257), (33, 512), (40, 1000), (7, 1024), (9, 1025), (150, 768), (64, 2048), (20, 2055), (3, 4096),
              (11, 4104), (2, 8191), (6, 8192), (2500, 72), (5000, 33)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_norm_sizes(rows, cols, dtype):
    o = ops.Ops(ops.egeria_norm_workspace_bytes(rows, cols), DEV)
    kind = "rms" if cols == 1 or (rows + cols) % 2 else "layer"     # one column has no variance for a layer norm
    gate_rows = [0, None, 1, 4, 300][(rows + cols) % 5]
    s = norm_inputs(rows, cols, dtype, torch.float32 if rows % 2 else dtype, kind, True, True, gate_rows, True, seed=rows + cols)
    check_norm(o, s, kind, True, True, gate_rows, 1.0, dtype)
    o.check_device_status()


@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False), (True, True)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("affine", [True, False])
def test_norm_parts(post, pre, kind, affine):
    o = ops.Ops(ops.egeria_norm_workspace_bytes(50, 192), DEV)
    for gate_rows, alpha in ((None, 1.0), (0, 0.5), (7, -1.25)):
        s = norm_inputs(50, 192, torch.bfloat16, torch.bfloat16, kind, post, pre, gate_rows, affine, seed=3)
        check_norm(o, s, kind, post, pre, gate_rows, alpha, torch.bfloat16)


def test_norm_rms_with_biases():
    o = ops.Ops(ops.egeria_norm_workspace_bytes(60, 136), DEV)
    s = norm_inputs(60, 136, torch.float16, torch.float16, "layer", True, True, 9, True, seed=4)
    check_norm(o, s, "rms", True, True, 9, 1.0, torch.float16)


@pytest.mark.parametrize("gate_rows", [1, 2, 3, 17, 256, 999, 1000, 5000])
@pytest.mark.parametrize("rows", [999, 4000])
def test_norm_gate_groups(rows, gate_rows):
    """Groups inside a thread block's rows, cut by their ends, and spanning many."""
    o = ops.Ops(ops.egeria_norm_workspace_bytes(rows, 128), DEV)
    s = norm_inputs(rows, 128, torch.float32, torch.float32, "rms", True, True, gate_rows, True, seed=8)
    args = {k: s[k] for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    opts = dict(kind="rms", gate_rows=gate_rows)
    y, h, st = o.egeria_norm_forward(s["x"], s["f"], **args, **opts)
    dy, dh = rand(rows, 128, dtype=torch.float32, seed=1), rand(rows, 128, dtype=torch.float32, seed=2)
    got = o.egeria_norm_backward(dy, dh, y, s["f"], st, **args, **opts)
    hat = y.double() * st[:, 3:4].double()
    d = dh.double() * s["w_pre"].double()
    tot = dy.double() + st[:, 3:4].double() * (d - hat * (d * hat).mean(1, keepdim=True))
    terms = tot * s["f"].double() * st[:, 1:2].double() * s["w_post"].double()
    group = torch.arange(rows, device=DEV) // gate_rows
    ref = torch.zeros_like(s["gate"], dtype=torch.float64).index_add_(0, group, terms)
    # what t is made of, where its parts cancel
    parts = dy.double().abs() + st[:, 3:4].double() * (d.abs() + hat.abs() * (d * hat).abs().mean(1, keepdim=True))
    made = (s["f"].double() * st[:, 1:2].double() * s["w_post"].double()).abs()
    size = torch.zeros_like(ref).index_add_(0, group, parts * made)
    close(got["dgate"], ref, (min(gate_rows, rows) + 256) * 2.0 ** -22 * size + 1e-30, "dgate")


def test_norm_strides():
    rows, cols = 30, 96
    o = ops.Ops(ops.egeria_norm_workspace_bytes(rows, cols), DEV)
    for shift, pitch in ((0, 104), (1, 97), (8, 96)):
        s = norm_inputs(rows, cols, torch.bfloat16, torch.bfloat16, "layer", True, True, 0, True, seed=5)
        for k in ("x", "f"):
            buf = torch.zeros(shift + rows * pitch, dtype=torch.bfloat16, device=DEV)
            v = buf[shift:].view(rows, pitch)[:, :cols]
            v.copy_(s[k])
            s[k] = v
        check_norm(o, s, "layer", True, True, 0, 1.0, torch.bfloat16)


def test_norm_of_large_offsets_and_constant_rows():
    """A row far from zero keeps its variance; a constant row has none and gives its bias."""
    o = ops.Ops(ops.egeria_norm_workspace_bytes(4, 512), DEV)
    f = rand(4, 512, dtype=torch.float32, seed=1, scale=0.5) + torch.tensor([[0.0], [1000.0], [-3e4], [0.0]], device=DEV)
    f[3] = 5.0
    x = torch.zeros_like(f)
    y, _, st = o.egeria_norm_forward(x, f, pre=False)
    mean, inv = stats64(f.double(), "layer")
    hat = (f.double() - mean) * inv
    close(y[:3], hat[:3], 2.0 ** -24 * 600 * (f.double().abs() * inv)[:3] + 1e-30, "y")
    assert (y[3] == 0).all() and torch.isfinite(st).all()


def test_norm_no_rows_and_nan_rows():
    o = ops.Ops(ops.egeria_norm_workspace_bytes(8, 64), DEV)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    w = rand(64)
    y, h, st = o.egeria_norm_forward(e, e, w_pre=w)
    got = o.egeria_norm_backward(e, e, y, e, st, w_pre=w)
    assert y.shape == (0, 64) and not got["dw_pre"].any()
    x, f = rand(8, 64, seed=1), rand(8, 64, seed=2)
    f[2, 5] = float("nan")
    f[4, 6] = float("inf")
    y, h, st = o.egeria_norm_forward(x, f)
    ok = [0, 1, 3, 5, 6, 7]
    assert torch.isnan(y[2]).all() and torch.isnan(h[4]).any() and torch.isfinite(y[ok]).all() and torch.isfinite(h[ok]).all()


def test_norm_in_place_and_same_bits():
    o = ops.Ops(ops.egeria_norm_workspace_bytes(3000, 128), DEV)
    s = norm_inputs(3000, 128, torch.bfloat16, torch.float32, "layer", True, True, 100, True, seed=2)
    args = {k: s[k] for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    y, h, st = o.egeria_norm_forward(s["x"], s["f"], gate_rows=100, **args)
    dy, dh = rand(3000, 128, seed=1), rand(3000, 128, seed=2)
    first = o.egeria_norm_backward(dy, dh, y, s["f"], st, gate_rows=100, **args)
    for _ in range(3):
        again = o.egeria_norm_backward(dy, dh, y, s["f"], st, gate_rows=100, **args)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_norm_refusals():
    o = ops.Ops(device=DEV)
    x = rand(4, 64)
    with pytest.raises(ValueError):
        o.egeria_norm_forward(x, x, kind="batch")
    with pytest.raises(ValueError):
        o.egeria_norm_forward(x, rand(4, 63))
    with pytest.raises(ValueError):
        o.egeria_norm_forward(x, x, gate=rand(2, 64), gate_rows=1)
    with pytest.raises(ValueError):
        o.egeria_norm_forward(x, x, w_pre=rand(64), w_post=rand(64, dtype=torch.float32))
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_norm_forward(x, x, w_pre=rand(64, dtype=torch.float16))
    assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_norm_forward(rand(2, 8200), rand(2, 8200))
    assert e.value.status == eg.ERR_UNSUPPORTED_SHAPE
    y, h, st = o.egeria_norm_forward(x, x)
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_norm_backward(x, None, y, x, st)              # no dh
    assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_norm_backward(rand(900, 2048), rand(900, 2048), rand(900, 2048), rand(900, 2048),
                               torch.zeros(900, 4, device=DEV))
    assert e.value.status == eg.ERR_WORKSPACE


# ----------------------------------------------------------------------------- AdamW

def model(sizes, dtype, gtype, master, bits, seed=0, shift=0):
    """Tensors, moments and gradients of a model; shift: elements by which every tensor is off its alignment."""
    def off(n, dt, values):
        buf = torch.zeros(n + shift, dtype=dt, device=DEV)
        buf[shift:] = values
        return buf[shift:]

    s = dict(p=[], g=[], m=[], v=[], w=[], ms=[], vs=[])
    for i, n in enumerate(sizes):
        p = rand(n, dtype=torch.float32, seed=seed + 10 * i)
        s["p"].append(off(n, dtype, p.to(dtype)))
        s["w"].append(off(n, torch.float32, p) if master else None)
        s["g"].append(off(n, gtype, rand(n, dtype=gtype, seed=seed + 10 * i + 1, scale=0.1)))
        m = rand(n, dtype=torch.float32, seed=seed + 10 * i + 2, scale=0.05)
        v = rand(n, dtype=torch.float32, seed=seed + 10 * i + 3, scale=0.1) ** 2
        if bits == 32:
            s["m"].append(off(n, torch.float32, m))
            s["v"].append(off(n, torch.float32, v))
        else:
            blocks = -(-n // 256)
            s["m"].append(off(n, torch.int8, torch.randint(-127, 128, (n,), device=DEV)))
            s["v"].append(off(n, torch.uint8, torch.randint(0, 256, (n,), device=DEV)))
            s["ms"].append(torch.rand(blocks, device=DEV) * 0.1 + 0.01)
            s["vs"].append(torch.rand(blocks, device=DEV) * 0.1 + 0.01)
    s["steps"] = torch.tensor([i % 5 for i in range(len(sizes))], dtype=torch.int32, device=DEV)
    return s


def decode(c, scale, most):
    c = c.double()
    return c * c.abs() / most ** 2 * scale.double().repeat_interleave(256)[:c.numel()]


def optimizer(s, bits, **kw):
    more = dict(m_scales=s["ms"], v_scales=s["vs"]) if bits == 8 else {}
    return ops.AdamW(s["p"], s["g"], s["m"], s["v"], s["steps"], masters=s["w"] if s["w"][0] is not None else None, **more, **kw)


def check_adamw(sizes, dtype, gtype, master, bits, shift=0, lr=1e-2, betas=(0.9, 0.99), eps=1e-8, wd=0.1, gs=0.5, frozen=None, modules=None, steps=1):
    s = model(sizes, dtype, gtype, master, bits, shift=shift)
    modules = modules or [-1] * len(sizes)
    a = optimizer(s, bits, weight_decay=wd, modules=modules)
    mask = None if frozen is None else torch.tensor(frozen, dtype=torch.uint8, device=DEV)
    scale = None if gs is None else torch.tensor([gs], device=DEV)
    for _ in range(steps):
        before = {k: [None if t is None else t.clone() for t in s[k]] for k in ("p", "m", "v", "w", "ms", "vs")}
        t0 = s["steps"].clone()
        a.egeria_adamw_step(lr, *betas, eps, grad_scale=scale, frozen=mask)
        for i, n in enumerate(sizes):
            if frozen is not None and modules[i] >= 0 and frozen[modules[i]]:
                assert s["steps"][i] == t0[i]
                assert all(torch.equal(s[k][i], before[k][i]) for k in ("p", "m", "v"))
                continue
            t = int(t0[i]) + 1
            assert s["steps"][i] == t
            g = s["g"][i].double() * (1.0 if gs is None else gs)
            m = before["m"][i].double() if bits == 32 else decode(before["m"][i], before["ms"][i], 127)
            v = before["v"][i].double() if bits == 32 else decode(before["v"][i], before["vs"][i], 255) ** 2
            m_size, v_size = betas[0] * m.abs() + (1 - betas[0]) * g.abs(), betas[1] * v + (1 - betas[1]) * g * g
            m, v = betas[0] * m + (1 - betas[0]) * g, v_size
            p = (before["w"] if master else before["p"])[i].double()
            change = m / (1 - betas[0] ** t) / (torch.sqrt(v / (1 - betas[1] ** t)) + eps)
            ref = p - lr * (wd * p + change)
            # the moments' few roundings reach the step relative to their sizes; root and division add a few more
            err = lr * (change.abs() * 2.0 ** -19 + 16 * 2.0 ** -24 * m_size / (1 - betas[0] ** t) / (torch.sqrt(v / (1 - betas[1] ** t)) + eps))
            if master:
                close(s["w"][i], ref, err + 2.0 ** -22 * p.abs() + 1e-30, f"master {i}")
                assert torch.equal(s["p"][i], s["w"][i].to(dtype))
            close(s["p"][i], ref, U[dtype] * ref.abs() + err + 2.0 ** -22 * p.abs() + TINY[dtype], f"param {i}")
            if bits == 32:
                close(s["m"][i], m, 8 * 2.0 ** -24 * m_size + 1e-37, "m")
                close(s["v"][i], v, 8 * 2.0 ** -24 * v_size + 1e-37, "v")
            elif n:
                for code, sc, val, most, size in ((s["m"][i], s["ms"][i], m, 127, m_size), (s["v"][i], s["vs"][i], v.sqrt(), 255, v.sqrt())):
                    pad = torch.zeros(-n % 256, device=DEV, dtype=torch.float64)
                    top, parts = (torch.cat([q.abs(), pad]).view(-1, 256).amax(1) for q in (val, size))
                    near = 2.0 ** -20 * top + 2.0 ** -21 * parts      # the parts of a moment may cancel
                    close(sc, top, near, "scale")
                    # half a step of the code next to the value: ((c + 1/2)^2 - c^2) / most^2 of the scale, but a code of 1 for any v > 0
                    c, full = code.double().abs(), sc.double().repeat_interleave(256)[:n]
                    step = (c + 0.25) / most ** 2 * full
                    if most == 255:
                        step = torch.where(c == 1, full / most ** 2, step)
                        assert ((c > 0) == (val > 0)).all()
                    close(torch.sign(code.double()) * c * c / most ** 2 * full, val, 1.001 * step + near.repeat_interleave(256)[:n], "codes")
    a.check_device_status()


def test_adamw_codes_are_the_formulas_bit_by_bit():
    """Codes and scales of three steps equal those of elementary operations, each rounded to 32 bits by itself."""
    n, b1, b2 = 256 * 4000, 0.9, 0.999
    s = model([n], torch.bfloat16, torch.bfloat16, False, 8)
    a = optimizer(s, 8)
    scale = torch.tensor([0.37], device=DEV)
    code = {k: s[k][0].clone().float().view(-1, 256) for k in ("m", "v")}
    top = {"m": s["ms"][0].clone().view(-1, 1), "v": s["vs"][0].clone().view(-1, 1)}

    unit = {"m": torch.tensor(1 / 127 ** 2, device=DEV), "v": torch.tensor(1 / 255 ** 2, device=DEV)}

    def codes(size, most, first):
        t = size.amax(1, keepdim=True)
        c = torch.round(most * torch.sqrt(size / torch.where(t > 0, t, torch.ones_like(t))))
        return torch.where(size > 0, c.clamp(min=first), c), t

    for step in range(3):
        g = s["g"][0].float().view(-1, 256) * scale
        m = b1 * (code["m"] * code["m"].abs() * (top["m"] * unit["m"])) + (1.0 - b1) * g
        root = code["v"] * code["v"] * (top["v"] * unit["v"])
        v = b2 * (root * root) + (1.0 - b2) * g * g
        c, top["m"] = codes(m.abs(), 127, 0)
        code["m"] = torch.sign(m) * c
        code["v"], top["v"] = codes(torch.sqrt(v), 255, 1)
        a.egeria_adamw_step(1e-3, b1, b2, grad_scale=scale)
        assert torch.equal(s["ms"][0], top["m"].view(-1)) and torch.equal(s["vs"][0], top["v"].view(-1)), step
        assert torch.equal(s["m"][0].float().view(-1, 256), code["m"]) and torch.equal(s["v"][0].float().view(-1, 256), code["v"]), step


ADAM_SIZES = [1, 255, 256, 257, 0, 4096, 4097, 100, 2304, 16, 8192 + 300]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,gtype,master", [(torch.float32, torch.float32, False), (torch.bfloat16, torch.bfloat16, False),
                                                (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, True),
                                                (torch.float16, torch.float16, True), (torch.float16, torch.float32, False),
                                                (torch.bfloat16, torch.float32, False), (torch.float16, torch.float16, False)])
def test_adamw_types(dtype, gtype, master, bits):
    check_adamw(ADAM_SIZES, dtype, gtype, master, bits, steps=3)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 4, 8])
def test_adamw_unaligned_tensors(bits, shift):
    check_adamw(ADAM_SIZES, torch.bfloat16, torch.bfloat16, True, bits, shift=shift)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_leaves_frozen_modules_alone(bits):
    check_adamw([300, 5000, 64, 0, 9000, 12], torch.bfloat16, torch.bfloat16, False, bits, frozen=[1, 0, 1], modules=[0, 0, 1, 2, 2, -1], steps=2)


@pytest.mark.parametrize("betas,eps,wd,gs", [((0.0, 0.0), 1e-8, 0.0, None), ((0.0, 0.999), 1e-3, 0.5, 2.0), ((0.95, 0.0), 1.0, 0.0, 1.0),
                                             ((0.9, 0.9999), 0.0, 0.01, 1e-3)])
def test_adamw_settings(betas, eps, wd, gs):
    check_adamw([700, 4096], torch.float32, torch.float32, False, 32, betas=betas, eps=eps, wd=wd, gs=gs, steps=2)


def test_adamw_many_steps_and_mixed_types():
    """Bias corrections far along, and tensors of different types in one optimizer."""
    sizes, kinds = [500, 4500, 260], [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)]
    parts = [model([n], d, g, False, 32, seed=i) for i, (n, (d, g)) in enumerate(zip(sizes, kinds))]
    s = {k: [q[k][0] for q in parts] for k in ("p", "g", "m", "v")}
    steps = torch.tensor([0, 99999, 7], dtype=torch.int32, device=DEV)
    before = [t.double() for t in s["p"]]
    m, v = [0.9 * a.double() + 0.1 * g.double() for a, g in zip(s["m"], s["g"])], [0.999 * a.double() + 0.001 * g.double() ** 2 for a, g in zip(s["v"], s["g"])]
    a = ops.AdamW(s["p"], s["g"], s["m"], s["v"], steps)
    a.egeria_adamw_step(1e-2)
    assert a.egeria_adamw_launch_count() == 3
    for i, t in enumerate((1, 100000, 8)):
        change = 1e-2 * (m[i] / (1 - 0.9 ** t)) / ((v[i] / (1 - 0.999 ** t)).sqrt() + 1e-8)
        close(s["p"][i], before[i] - change, U[s["p"][i].dtype] * (before[i] - change).abs() + 2.0 ** -18 * change.abs() + 2.0 ** -23 * before[i].abs(), f"{i}")
    assert steps.tolist() == [1, 100000, 8]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_adamw_leaves_a_step_out_on_a_bad_scale(bits, bad):
    s = model([300, 5000], torch.bfloat16, torch.bfloat16, False, bits)
    a = optimizer(s, bits)
    before = [t.clone() for k in ("p", "m", "v") for t in s[k]]
    a.egeria_adamw_step(1e-2, grad_scale=torch.tensor([bad], device=DEV))
    assert all(torch.equal(x, y) for x, y in zip(before, [t for k in ("p", "m", "v") for t in s[k]]))
    assert s["steps"].tolist() == [0, 1]
    a.egeria_adamw_step(1e-2, grad_scale=torch.tensor([1.0], device=DEV))
    assert s["steps"].tolist() == [1, 2]


def test_adamw_bad_gradients_stay_where_they_are():
    """A NaN reaches its own value of 32-bit moments, its own block of 8-bit ones."""
    for bits, first, last in ((32, 700, 701), (8, 512, 768)):
        s = model([1000], torch.float32, torch.float32, False, bits)
        s["g"][0][700] = float("nan")
        a = optimizer(s, bits)
        a.egeria_adamw_step(1e-2)
        a.egeria_adamw_step(1e-2)
        bad = torch.isnan(s["p"][0])
        assert bad[first:last].all() and int(bad.sum()) == last - first


def test_adamw_zero_moments_and_gradients():
    s = model([600], torch.float32, torch.float32, False, 8)
    for k in ("m", "v", "ms", "vs"):
        s[k][0].zero_()
    s["g"][0].zero_()
    before = s["p"][0].clone()
    optimizer(s, 8).egeria_adamw_step(1e-2, eps=1e-8)
    assert torch.equal(s["p"][0], before) and not s["v"][0].any() and not s["ms"][0].any()


def test_adamw_moves_with_new_gradients_streams_and_graphs():
    s = model([5000, 300], torch.float32, torch.float32, False, 32)
    twin = {k: [t.clone() for t in s[k]] for k in ("p", "g", "m", "v")}
    a, b = optimizer(s, 32), ops.AdamW(twin["p"], twin["g"], twin["m"], twin["v"], s["steps"].clone())
    other = [rand(n, dtype=torch.float32, seed=70 + n) for n in (5000, 300)]
    a.egeria_adamw_set_grads(other)
    for x, y in zip(twin["g"], other):
        x.copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.egeria_adamw_step(1e-2, stream=side)
    side.synchronize()
    b.egeria_adamw_step(1e-2)
    assert all(torch.equal(x, y) for x, y in zip(s["p"], twin["p"]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.egeria_adamw_step(1e-2, stream=torch.cuda.current_stream())
    for _ in range(3):
        g.replay()
        b.egeria_adamw_step(1e-2)
    assert all(torch.equal(x, y) for x, y in zip(s["p"], twin["p"])) and s["steps"].tolist() == [4, 5]


def test_adamw_refusals():
    s = model([300, 20], torch.bfloat16, torch.bfloat16, False, 32)
    a = optimizer(s, 32, modules=[0, 1])
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=1e-3, beta1=1.0), dict(lr=1e-3, beta2=-0.1), dict(lr=1e-3, eps=-1.0)):
        with pytest.raises(eg.EgeriaError) as e:
            a.egeria_adamw_step(**bad)
        assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        a.egeria_adamw_step(1e-3, frozen=torch.zeros(1, dtype=torch.uint8, device=DEV))      # two modules
    with pytest.raises(ValueError):
        a.egeria_adamw_set_grads(s["g"][:1])
    with pytest.raises(ValueError):
        ops.AdamW(s["p"], s["g"], s["m"], [t.half() for t in s["v"]], s["steps"])
    with pytest.raises(ValueError):
        ops.AdamW([t.view(-1, 10)[:, :5] for t in s["p"]], s["g"], s["m"], s["v"], s["steps"])
    with pytest.raises(eg.EgeriaError):
        ops.AdamW(s["p"], [t.half() for t in s["g"]], s["m"], s["v"], s["steps"])
