"""GPU parity of the gated feed-forward blocks against the formula in 64 bits.

Tolerances are derived as in test_ops_gpu.py, element by element and before the first run: a rounding is off by U of the
value, a sum of n products by (n + 8) 2^-23 of the products' sizes, an activation by 2^-15 of its value and its slope by 2^-14
of itself and 2^-20; the hidden values, and dg and du, are rounded once as the next product's operands.
"""
import pytest
import torch

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops
from test_ops_gpu import ACTS, DEV, TINY, U, act64, close, rand
from test_ops_gpu import check_forward as check_linear

pytestmark = pytest.mark.gpu


def handle(rows, inp, hidden, out):
    return ops.Ops(ops.egeria_gated_workspace_bytes(rows, inp, hidden, out), DEV)


def weights(inp, hidden, out, dtype, seed=0, biases=True):
    w = dict(w_gate=rand(hidden, inp, dtype=dtype, seed=seed, scale=inp ** -0.5), w_up=rand(hidden, inp, dtype=dtype, seed=seed + 1, scale=inp ** -0.5),
             w_down=rand(out, hidden, dtype=dtype, seed=seed + 2, scale=hidden ** -0.5))
    b = dict(b_gate=rand(hidden, dtype=dtype, seed=seed + 3), b_up=rand(hidden, dtype=dtype, seed=seed + 4), b_down=rand(out, dtype=dtype, seed=seed + 5))
    return w, b if biases else dict(b_gate=None, b_up=None, b_down=None)


def sum_error(n):
    return (n + 8) * 2.0 ** -23


def check_forward(o, x, w, b, act, residual=None, save=True, out=None):
    base = None if residual is None else residual.double()
    got = o.egeria_gated_forward(x, **w, **b, act=act, residual=residual, save=save, out=out)
    y, g, u = got if save else (got, None, None)
    t, xd = x.dtype, x.double()

    def projection(name):
        wd, bias = w["w_" + name].double(), b["b_" + name]
        v, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
        if bias is not None:
            v, size = v + bias.double(), size + bias.double().abs()
        return v, sum_error(x.shape[1]) * size

    (gr, eg_), (ur, eu) = projection("gate"), projection("up")
    if save:
        close(g, gr, U[t] * gr.abs() + eg_ + TINY[t], "g")
        close(u, ur, U[t] * ur.abs() + eu + TINY[t], "u")
    a = act64(gr, act)[0]
    h = a * ur
    eh = 1.2 * eg_ * (ur.abs() + eu) + a.abs() * eu + (2.0 ** -15 + U[t]) * h.abs() + TINY[t]      # no activation is steeper than 1.13
    wd = w["w_down"].double()
    yr, size = h @ wd.t(), h.abs() @ wd.abs().t()
    tol = eh @ wd.abs().t() + sum_error(wd.shape[1]) * size
    for extra in (b["b_down"], base):
        if extra is not None:
            yr = yr + extra.double()
            tol = tol + 2.0 ** -23 * (yr.abs() + extra.double().abs())
    close(y, yr, U[t] * yr.abs() + tol + TINY[t], "y")
    return got


def check_backward(o, dy, x, w, g, u, act, **need):
    got = o.egeria_gated_backward(dy, x, **w, g=g, u=u, act=act, **need)
    t, (rows, out), hidden = dy.dtype, dy.shape, g.shape[1]
    dyd, gd, ud, wd = dy.double(), g.double(), u.double(), w["w_down"].double()
    value, slope = act64(gd, act)
    dh, eh = dyd @ wd, sum_error(out) * (dyd.abs() @ wd.abs())
    exact = 0.0 if act in ("none", "relu") else 1.0
    dg, du, h = dh * ud * slope, dh * value, value * ud
    eg_ = eh * (ud * slope).abs() + (exact * 2.0 ** -14 + 2.0 ** -22) * dg.abs() + exact * 2.0 ** -20 * (dh * ud).abs()
    eu = eh * value.abs() + (exact * 2.0 ** -15 + 2.0 ** -23) * du.abs()
    rg, ru, rh = (U[t] * v.abs() + TINY[t] for v in (dg, du, h))
    rh = rh + (exact * 2.0 ** -15 + 2.0 ** -23) * h.abs()
    if need.get("need_dx", True):
        a, c = w["w_gate"].double(), w["w_up"].double()
        ref, size = dg @ a + du @ c, dg.abs() @ a.abs() + du.abs() @ c.abs()
        tol = (eg_ + rg) @ a.abs() + (eu + ru) @ c.abs() + sum_error(2 * hidden) * size
        close(got["dx"], ref, U[t] * ref.abs() + tol + TINY[t], "dx")
    else:
        assert got["dx"] is None
    if need.get("need_dw", True):
        xd = x.double()
        for name, d, e in (("dw_gate", dg, eg_ + rg), ("dw_up", du, eu + ru)):
            ref = d.t() @ xd
            close(got[name], ref, U[t] * ref.abs() + e.t() @ xd.abs() + sum_error(rows) * (d.abs().t() @ xd.abs()) + TINY[t], name)
        ref = dyd.t() @ h
        close(got["dw_down"], ref, U[t] * ref.abs() + dyd.abs().t() @ rh + sum_error(rows) * (dyd.abs().t() @ h.abs()) + TINY[t], "dw_down")
    else:
        assert got["dw_gate"] is None and got["dw_up"] is None and got["dw_down"] is None
    if need.get("need_db", False):
        for name, d, e in (("db_gate", dg, eg_), ("db_up", du, eu), ("db_down", dyd, 0.0 * dyd)):
            ref = d.sum(0)
            close(got[name], ref, U[t] * ref.abs() + e.sum(0) + sum_error(rows) * d.abs().sum(0) + TINY[t], name)
    else:
        assert got["db_gate"] is None and got["db_up"] is None and got["db_down"] is None
    return got


# rows, inp, hidden, out: one token to long batches, odd sizes, tiles with one column or row left
SIZES = [(1, 64, 64, 64), (1, 1024, 2816, 1024), (2, 8, 1, 3), (3, 513, 70, 9), (4, 1000, 257, 64), (5, 100, 333, 100), (9, 64, 32, 64), (31, 1, 5, 2),
         (64, 72, 136, 40), (128, 256, 256, 256), (129, 65, 129, 257), (200, 1024, 512, 512), (257, 264, 520, 264), (300, 131, 1001, 517),
         (513, 768, 2048, 768), (1000, 24, 3000, 24)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inp,hidden,out", SIZES)
def test_forward(rows, inp, hidden, out, dtype):
    o = handle(rows, inp, hidden, out)
    s = rows + inp + hidden
    x, r = rand(rows, inp, dtype=dtype, seed=s + 9), rand(rows, out, dtype=dtype, seed=s + 8)
    w, b = weights(inp, hidden, out, dtype, s)
    check_forward(o, x, w, b, ACTS[s % 5], r)
    check_forward(o, x, w, weights(inp, hidden, out, dtype, s, False)[1], "silu", None, False)
    o.check_device_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inp,hidden,out", SIZES)
def test_backward(rows, inp, hidden, out, dtype):
    o = handle(rows, inp, hidden, out)
    s = rows + inp + hidden
    x, dy = rand(rows, inp, dtype=dtype, seed=s + 9), rand(rows, out, dtype=dtype, seed=s + 8, scale=0.25)
    g, u = rand(rows, hidden, dtype=dtype, seed=s + 7, scale=2.0), rand(rows, hidden, dtype=dtype, seed=s + 6)
    w, _ = weights(inp, hidden, out, dtype, s)
    check_backward(o, dy, x, w, g, u, ACTS[(s + 1) % 5], need_db=True)
    check_backward(o, dy, x, w, g, u, "silu")
    o.check_device_status()


@pytest.mark.parametrize("rows,inp,hidden,out", [(4096, 1024, 2816, 1024), (2048, 2048, 5632, 2048), (16384, 256, 768, 256), (1500, 1032, 4104, 520),
                                                   (16000, 128, 2816, 1000)])
def test_larger(rows, inp, hidden, out):
    """Sizes whose products go over pairs of CTAs, tiles of 512 rows and more than one round of them."""
    o = handle(rows, inp, hidden, out)
    x, dy = rand(rows, inp, seed=1), rand(rows, out, seed=2, scale=1 / 64)
    w, b = weights(inp, hidden, out, torch.bfloat16, 3)
    _, g, u = check_forward(o, x, w, b, "gelu_tanh", rand(rows, out, seed=4))
    check_backward(o, dy, x, w, g, u, "gelu_tanh", need_db=True)
    o.check_device_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inp,out", [(16384, 4096, 1024), (15900, 2700, 1001), (9000, 2624, 2048)])
def test_linear_layers_of_long_sums(rows, inp, out, dtype):
    """Where a block's second product, or a linear layer, goes over tiles of 512 rows; the give-up path there too."""
    o = ops.Ops(ops.egeria_linear_workspace_bytes(rows, inp, out), DEV)
    x, w = rand(rows, inp, dtype=dtype, seed=1), rand(out, inp, dtype=dtype, seed=2, scale=inp ** -0.5)
    r, b = rand(rows, out, dtype=dtype, seed=3), rand(out, dtype=dtype, seed=4)
    check_linear(o, x, w, b, "none", r, False)
    want = o.egeria_linear_forward(x, w)
    for kind in (1, 2):
        o.egeria_ops_debug_stall_next(kind)
        o.egeria_linear_forward(x, w)
        assert o.egeria_ops_device_status() == eg.ERR_TIMEOUT
        assert torch.equal(o.egeria_linear_forward(x, w), want)
    o.check_device_status()


@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("act", ACTS)
def test_activations(rows, act):
    """Arguments over a wide range; every slope and value, in both passes."""
    o = handle(rows, 64, 256, 64)
    x = rand(rows, 64, seed=1, scale=3.0)
    w, b = weights(64, 256, 64, torch.bfloat16, 5)
    check_forward(o, x, w, b, act)
    check_backward(o, rand(rows, 64, seed=2), x, w, rand(rows, 256, seed=3, scale=4.0), rand(rows, 256, seed=4), act, need_db=True)


@pytest.mark.parametrize("dx,dw,db", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 0, 1)])
@pytest.mark.parametrize("rows", [7, 300])
def test_backward_of_parts(rows, dx, dw, db):
    """A frozen block wants dx alone, the first that trains none: what is not wanted need not be there."""
    o = handle(rows, 72, 136, 40)
    w, _ = weights(72, 136, 40, torch.bfloat16, 1)
    full = dict(w)
    if not dx:
        w["w_gate"] = w["w_up"] = None
    x = rand(rows, 72, seed=2) if dw else None
    dy, g, u = rand(rows, 40, seed=3), rand(rows, 136, seed=4), rand(rows, 136, seed=5)
    got = check_backward(o, dy, x, w, g, u, "silu", need_dx=bool(dx), need_dw=bool(dw), need_db=bool(db))
    whole = o.egeria_gated_backward(dy, rand(rows, 72, seed=2), **full, g=g, u=u, need_db=True)
    for k, v in got.items():
        assert v is None or torch.equal(v, whole[k]), k
    o.check_device_status()


def test_nothing_wanted():
    o = handle(8, 64, 64, 64)
    w, _ = weights(64, 64, 64, torch.bfloat16)
    got = o.egeria_gated_backward(rand(8, 64), rand(8, 64), **w, g=rand(8, 64), u=rand(8, 64), need_dx=False, need_dw=False)
    assert all(v is None for v in got.values())


@pytest.mark.parametrize("shift,pitch", [(0, 72), (1, 65), (3, 80), (8, 96), (16, 64)])
@pytest.mark.parametrize("rows", [3, 140])
def test_strides_and_offsets(rows, shift, pitch):
    """Every operand a view with its own offset and row pitch; what lies between the rows stays as it was."""

    def view(seed, n, fill=0.0):
        buf = torch.full((shift + n * pitch + 64,), fill, dtype=torch.bfloat16, device=DEV)
        v = buf[shift:shift + n * pitch].view(n, pitch)[:, :64]
        v.copy_(rand(n, 64, seed=seed, scale=0.3))
        return buf, v

    o = handle(rows, 64, 64, 64)
    x, r, dy, g, u = (view(k, rows)[1] for k in range(1, 6))
    w = dict(zip(("w_gate", "w_up", "w_down"), (view(k, 64)[1] for k in (6, 7, 8))))
    buf, y = view(9, rows, 7.0)
    _, b = weights(64, 64, 64, torch.bfloat16)
    check_forward(o, x, w, b, "silu", r, out=y)
    check_backward(o, dy, x, w, g, u, "gelu", need_db=True)
    if pitch > 64:
        assert (buf[shift:shift + rows * pitch].view(rows, pitch)[:, 64:] == 7.0).all()
    assert (buf[:shift] == 7.0).all() and (buf[shift + rows * pitch:] == 7.0).all()


@pytest.mark.parametrize("rows", [2, 130])
def test_projections_that_are_halves_of_one_matrix(rows):
    """Above one another, and side by side in its rows; dw_gate and dw_up are the halves of one tensor too."""
    o = handle(rows, 64, 96, 64)
    x, g, u, dy = rand(rows, 64, seed=1), rand(rows, 96, seed=2), rand(rows, 96, seed=3), rand(rows, 64, seed=4)
    both, beside = rand(192, 64, seed=5, scale=0.125), rand(96, 128, seed=6, scale=0.125)
    _, b = weights(64, 96, 64, torch.bfloat16)
    for gate, up in ((both[:96], both[96:]), (beside[:, :64], beside[:, 64:])):
        w = dict(w_gate=gate, w_up=up, w_down=rand(64, 96, seed=7, scale=0.1))
        check_forward(o, x, w, b, "silu")
        got = check_backward(o, dy, x, w, g, u, "silu")
        assert got["dw_up"].data_ptr() == got["dw_gate"].data_ptr() + 96 * 64 * 2


@pytest.mark.parametrize("rows", [3, 200])
def test_adds_onto_the_residual_in_place(rows):
    o = handle(rows, 64, 128, 64)
    w, b = weights(64, 128, 64, torch.bfloat16)
    r = rand(rows, 64, seed=9)
    check_forward(o, rand(rows, 64, seed=1), w, b, "silu", r, out=r)


def test_no_rows():
    o = handle(16, 64, 128, 64)
    w, b = weights(64, 128, 64, torch.bfloat16)
    x, h = rand(0, 64), rand(0, 128)
    y, g, u = o.egeria_gated_forward(x, **w, **b, save=True)
    assert y.shape == (0, 64) and g.shape == u.shape == (0, 128)
    got = o.egeria_gated_backward(x, x, **w, g=h, u=h, need_db=True)
    assert got.pop("dx").shape == (0, 64)
    assert all(not v.any() for v in got.values())


@pytest.mark.parametrize("rows", [2, 130])
def test_infinities_and_nans_stay_in_their_rows(rows):
    o = handle(rows, 64, 128, 64)
    w, b = weights(64, 128, 64, torch.bfloat16)
    x, dy, g, u = rand(rows, 64, seed=1), rand(rows, 64, seed=2), rand(rows, 128, seed=3), rand(rows, 128, seed=4)
    y, dx = o.egeria_gated_forward(x, **w, **b), o.egeria_gated_backward(dy, x, **w, g=g, u=u)["dx"]
    bad, badu = x.clone(), u.clone()
    bad[1, 5], badu[1, 7] = float("inf"), float("nan")
    y2, dx2 = o.egeria_gated_forward(bad, **w, **b), o.egeria_gated_backward(dy, x, **w, g=g, u=badu)["dx"]
    keep = [r for r in range(rows) if r != 1]
    assert not torch.isfinite(y2[1]).all() and torch.isnan(dx2[1]).all()
    assert torch.equal(y2[keep], y[keep]) and torch.equal(dx2[keep], dx[keep])


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_huge_arguments_have_finite_gradients(act):
    o = handle(130, 64, 64, 64)
    w, _ = weights(64, 64, 64, torch.bfloat16)
    big = torch.tensor([1e2, 1e10, 1e13, 1e20, 1e30, 3e38], device=DEV)
    g = torch.cat([big, -big]).to(torch.bfloat16).repeat(130 * 64)[:130 * 64].view(130, 64)
    u = rand(130, 64, seed=1) * (g.float().abs() < 1e15) / 1e3       # du and h of the largest would leave the type's range
    dy = rand(130, 64, seed=2) * 1e-30
    dy[:, 1:] = 0
    got = o.egeria_gated_backward(dy.to(torch.bfloat16), rand(130, 64, seed=3), **w, g=g, u=u.to(torch.bfloat16), act=act, need_db=True)
    assert all(torch.isfinite(v).all() for v in got.values())


def test_same_bits_every_time():
    for rows, inp, hidden, out in ((48, 1024, 2816, 1024), (777, 520, 1336, 264)):
        o = handle(rows, inp, hidden, out)
        x, dy, r = rand(rows, inp, seed=1), rand(rows, out, seed=2), rand(rows, out, seed=3)
        w, b = weights(inp, hidden, out, torch.bfloat16)
        first = o.egeria_gated_forward(x, **w, **b, residual=r, save=True)
        grads = o.egeria_gated_backward(dy, x, **w, g=first[1], u=first[2], need_db=True)
        for _ in range(4):
            assert all(torch.equal(p, q) for p, q in zip(first, o.egeria_gated_forward(x, **w, **b, residual=r, save=True)))
            again = o.egeria_gated_backward(dy, x, **w, g=first[1], u=first[2], need_db=True)
            assert all(torch.equal(grads[k], again[k]) for k in grads)


@pytest.mark.parametrize("rows", [2, 300])
def test_another_stream_and_a_graph(rows):
    o = handle(rows, 128, 256, 128)
    w, b = weights(128, 256, 128, torch.bfloat16)
    x, dy = rand(rows, 128, seed=1), rand(rows, 128, seed=2)
    want, g, u = o.egeria_gated_forward(x, **w, **b, save=True)
    back = o.egeria_gated_backward(dy, x, **w, g=g, u=u, need_db=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = o.egeria_gated_forward(x, **w, **b, stream=side)
    back2 = o.egeria_gated_backward(dy, x, **w, g=g, u=u, need_db=True, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(back[k], back2[k]) for k in back)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cur = torch.cuda.current_stream()
        y, gg, uu = o.egeria_gated_forward(x, **w, **b, save=True, stream=cur)
        grads = o.egeria_gated_backward(dy, x, **w, g=gg, u=uu, need_db=True, stream=cur)
    for k in range(3):
        x.copy_(rand(rows, 128, seed=50 + k))
        graph.replay()
        seen = [t.clone() for t in (y, *grads.values())]
        yy, g, u = o.egeria_gated_forward(x, **w, **b, save=True)
        now = o.egeria_gated_backward(dy, x, **w, g=g, u=u, need_db=True)
        assert all(torch.equal(p, q) for p, q in zip(seen, (yy, *now.values())))
    o.check_device_status()


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(act):
    """The kernel's gradients along random directions against central differences of the formula in 64 bits.  With g and u kept in
    float16 the gradients are off by a few U of their size; the differences by step^2."""
    rows, inp, hidden, out = 40, 48, 72, 56
    t = torch.float16
    o = handle(rows, inp, hidden, out)
    x, c = rand(rows, inp, dtype=t, seed=1), rand(rows, out, dtype=t, seed=2)
    w, b = weights(inp, hidden, out, t, 3)
    _, g, u = o.egeria_gated_forward(x, **w, **b, act=act, save=True)
    got = o.egeria_gated_backward(c, x, **w, g=g, u=u, act=act, need_db=True)

    def loss(p):
        h = act64(p["x"] @ p["w_gate"].t() + p["b_gate"], act)[0] * (p["x"] @ p["w_up"].t() + p["b_up"])
        return float(((h @ p["w_down"].t() + p["b_down"]) * c.double()).sum())

    point = {k: v.double() for k, v in dict(x=x, **w, **b).items()}
    for k, v in point.items():
        d = got["d" + k].double()
        along = d / d.norm()             # along itself: a gradient of zero, or of another parameter, fails by far
        step = 1e-5
        up, down = dict(point), dict(point)
        up[k], down[k] = v + step * along, v - step * along
        slope = (loss(up) - loss(down)) / (2 * step)
        # eight roundings of at most U each lie between the formula and a gradient
        assert abs(slope - float(d.norm())) <= 8 * U[t] * float(d.norm()) + 1e-6, k


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rows,inp,hidden,out", [(64, 256, 512, 256), (700, 1024, 1408, 512), (4096, 1024, 2816, 1024)])
def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(kind, rows, inp, hidden, out):
    """The give-up path in each of the launches' forms (see the same test of the linear layers)."""
    o = handle(rows, inp, hidden, out)
    x, dy = rand(rows, inp, seed=1), rand(rows, out, seed=2)
    w, b = weights(inp, hidden, out, torch.bfloat16)
    want, g, u = o.egeria_gated_forward(x, **w, **b, save=True)
    grads = o.egeria_gated_backward(dy, x, **w, g=g, u=u)
    o.check_device_status()
    for call in (lambda: o.egeria_gated_forward(x, **w, **b), lambda: o.egeria_gated_backward(dy, x, **w, g=g, u=u)):
        o.egeria_ops_debug_stall_next(kind)
        call()
        assert o.egeria_ops_device_status() == eg.ERR_TIMEOUT
        assert o.egeria_ops_device_status() == eg.OK
    for _ in range(2):
        assert torch.equal(o.egeria_gated_forward(x, **w, **b), want)
        again = o.egeria_gated_backward(dy, x, **w, g=g, u=u)
        assert all(v is None or torch.equal(v, grads[k]) for k, v in again.items())
    o.check_device_status()


def test_results_say_that_they_have_no_gradient():
    o = handle(8, 64, 64, 64)
    w, b = weights(64, 64, 64, torch.bfloat16)
    x = rand(8, 64, seed=1).requires_grad_()
    for t in o.egeria_gated_forward(x, **w, **b, save=True):
        with pytest.raises(RuntimeError, match="egeria_gated_backward"):
            t.float().sum().backward()
    with torch.no_grad():
        assert not o.egeria_gated_forward(x, **w, **b).requires_grad
    out = rand(8, 64)
    product = torch.ones(8, 64, device=DEV, dtype=torch.bfloat16, requires_grad=True) * out
    o.egeria_gated_forward(x.detach(), **w, **b, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.sum().backward()


def test_refusals():
    o = handle(16, 64, 128, 64)
    w, b = weights(64, 128, 64, torch.bfloat16)
    x, g = rand(16, 64), rand(16, 128)
    for change in (dict(act="tanh"), dict(w_up=rand(127, 64)), dict(w_down=rand(64, 127)), dict(b_gate=rand(64)), dict(b_down=rand(128)),
                   dict(w_gate=rand(64, 128).t()), dict(residual=rand(16, 65)), dict(residual=rand(16, 64).half()), dict(w_up=w["w_up"].cpu()),
                   dict(out=rand(15, 64))):
        with pytest.raises(ValueError):
            o.egeria_gated_forward(**{**dict(x=x), **w, **b, **change})
    for change in (dict(g=rand(16, 127)), dict(u=rand(15, 128)), dict(x=None), dict(w_gate=None), dict(w_down=rand(63, 128)), dict(act="tanh")):
        with pytest.raises(ValueError):
            o.egeria_gated_backward(**{**dict(dy=x, x=x, g=g, u=g), **w, **change})
    f = {k: v.float() for k, v in w.items()}
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_gated_forward(x.float(), **f)
    assert e.value.status == eg.ERR_INVALID_ARG
    # y over what other blocks read, or write
    for out, own in ((x, w), (w["w_gate"][:16], w), (w["w_down"][:16, :64], w), (b["b_gate"][:64].view(1, 64).expand(16, 64)[:1], None)):
        with pytest.raises(eg.EgeriaError) as e:
            if own is None:
                o.egeria_gated_forward(x[:1], **w, **b, out=out)
            else:
                o.egeria_gated_forward(x, **own, out=out)
        assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_gated_forward(rand(4000, 64), **w)
    assert e.value.status == eg.ERR_WORKSPACE
    with pytest.raises(eg.EgeriaError) as e:
        o.egeria_gated_backward(rand(4000, 64), rand(4000, 64), **w, g=rand(4000, 128), u=rand(4000, 128))
    assert e.value.status == eg.ERR_WORKSPACE


@pytest.mark.parametrize("most,rows", [((4096, 512, 1376, 512), (1, 5, 130, 1000, 4095)), ((300, 1000, 1001, 999), (3, 299))])
def test_a_handle_takes_smaller_calls(most, rows):
    o = handle(*most)
    _, inp, hidden, out = most
    w, b = weights(inp, hidden, out, torch.bfloat16)
    for r in rows:
        x = rand(r, inp, seed=r)
        _, g, u = check_forward(o, x, w, b, "silu")
        check_backward(o, rand(r, out, seed=r + 1), x, w, g, u, "silu")
