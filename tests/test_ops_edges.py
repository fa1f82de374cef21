"""What the training operators do at the edges: memory that other streams still use, sizes below a handle's, operands that
overlap, values at the ends of their types, autograd around the calls, aliases, gradients against differences.

Tolerances are derived as in test_ops_gpu.py, before the first run.
"""
import ctypes
import math
import subprocess
import sys
import weakref
from pathlib import Path

import pytest
import torch

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops
from test_ops_gpu import DEV, TINY, U, act64, close, rand

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- memory that other work still uses

def contended(nbytes, make):
    """make()'s handle, its workspace of `nbytes` being memory that a kernel of its stream has yet to write."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        old = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(4)]
        places = {t.data_ptr() for t in old}
        torch.cuda._sleep(20_000_000)      # about 10 ms
        for k in range(4):
            old[k].fill_(255)
        del old
        h = make()
        assert h._raw.data_ptr() in places
    torch.cuda.synchronize()
    return h


def workspace_of(h, nbytes=None):
    at = -h._raw.data_ptr() % eg.WORKSPACE_ALIGN
    return h._raw[at:][:nbytes]


def test_new_handle_waits_for_the_memory_it_is_given():
    """The clearing of an Ops' tickets and AdamW's table come after whatever still writes to the block."""
    o = contended(ops.Ops(1 << 20, DEV)._raw.numel(), lambda: ops.Ops(1 << 20, DEV))
    assert not workspace_of(o, ops.OPS_WORKSPACE_MIN).any()
    p, g, m, v = ([rand(n, dtype=torch.float32, seed=n + k) for n in (700, 5000)] for k in range(4))
    steps = torch.zeros(2, dtype=torch.int32, device=DEV)
    quiet = ops.AdamW(p, g, m, v, steps)
    size = quiet._raw.numel() - eg.WORKSPACE_ALIGN
    other = contended(quiet._raw.numel(), lambda: ops.AdamW(p, g, m, v, steps))
    assert torch.equal(workspace_of(quiet, size), workspace_of(other, size))


def test_device_status_reports_once_and_clears_the_tickets():
    """A status word and tickets as a call that gave up leaves them, on a stream of its own: reported once, then a split
    product is whole."""
    side = torch.cuda.Stream()
    x, w = rand(300, 4096, seed=1), rand(192, 4096, seed=2, scale=1 / 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        o = ops.Ops(ops.egeria_linear_workspace_bytes(300, 4096, 192), DEV)
        want = o.egeria_linear_forward(x, w)
        o.check_device_status()
        words = workspace_of(o, ops.OPS_WORKSPACE_MIN).view(torch.int32)
        assert not words.any()
        for _ in range(3):
            words.fill_(1)
            words[0] = eg.ERR_TIMEOUT
            assert o.egeria_ops_device_status() == eg.ERR_TIMEOUT
            assert o.egeria_ops_device_status() == eg.OK
            assert torch.equal(o.egeria_linear_forward(x, w), want)
            assert not words.any()


def test_new_context_waits_for_the_memory_it_is_given():
    """The same for the plasticity evaluation's workspace: counters, slots and windows start from what creation wrote."""
    from paper_2201_06227_b200 import workloads as wl
    ds, b = [4096, 64 * 148], 128
    pairs = [wl.make_pair(b, d, "relu", 0.2, seed=77 + d, device=DEV) for d in ds]
    at, ar = [p[0] for p in pairs], [p[1] for p in pairs]
    quiet = eg.Context(ds, b, 5, 1e-3, device=DEV)
    want = [t.clone() for t in quiet.egeria_plasticity_evaluate(at, ar)]
    other = contended(quiet._raw.numel(), lambda: eg.Context(ds, b, 5, 1e-3, device=DEV))
    got = other.egeria_plasticity_evaluate(at, ar)
    other.check_device_status()
    assert got[0].cpu().numpy().tobytes() == want[0].cpu().numpy().tobytes()      # the slopes of a first evaluation may be NaN
    assert got[1].cpu().numpy().tobytes() == want[1].cpu().numpy().tobytes() and torch.equal(got[2], want[2])


@pytest.mark.parametrize("which", ["ops", "adamw"])
def test_a_dropped_handle_keeps_its_memory_until_its_calls_have_run(which):
    """A handle made on one stream, called on another that is the current one, and dropped with the call in flight: its
    workspace is not handed out before that call has run."""
    side = torch.cuda.Stream()
    x, w = rand(200, 512, seed=1), rand(256, 512, seed=2)
    p, g, m, v = ([rand(3000, dtype=torch.float32, seed=k)] for k in range(4))
    steps = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    h = ops.Ops(ops.egeria_linear_workspace_bytes(200, 512, 256), DEV) if which == "ops" else ops.AdamW(p, g, m, v, steps)
    place, size = h._raw.data_ptr(), h._raw.numel()
    with torch.cuda.stream(side):
        torch.cuda._sleep(600_000_000)         # about 0.3 s
        if which == "ops":
            h.egeria_linear_forward(x, w)
        else:
            h.egeria_adamw_step(1e-3)
    del h
    new = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(3)]
    busy = not side.query()
    assert busy and place not in {t.data_ptr() for t in new}
    side.synchronize()


def test_new_gradients_are_kept_for_the_streams_of_the_steps():
    """set_grads on a handle whose steps run on another stream: what it then lets go of is not handed out under a step."""
    side = torch.cuda.Stream()
    p, m, v = ([rand(3000, dtype=torch.float32, seed=k)] for k in range(3))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    first, second = [torch.ones(3000, device=DEV)], [torch.ones(3000, device=DEV)]
    a = ops.AdamW(p, first, m, v, torch.zeros(1, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a.egeria_adamw_step(1e-3)
        a.egeria_adamw_set_grads(second)
        places = {first[0].data_ptr(), second[0].data_ptr()}
        torch.cuda._sleep(600_000_000)
        a.egeria_adamw_step(1e-3)
    del a, first, second
    new = [torch.empty(3000, device=DEV) for _ in range(4)]
    busy = not side.query()
    assert busy and not places & {t.data_ptr() for t in new}
    side.synchronize()


def test_refused_gradients_leave_the_old_ones_in_force():
    """set_grads is refused on a capturing stream: the table still names the old gradients, so the handle keeps them."""
    p, g, m, v = ([rand(3000, dtype=torch.float32, seed=k, scale=0.1)] for k in range(4))
    v[0].abs_()
    a = ops.AdamW(p, g, m, v, torch.zeros(1, dtype=torch.int32, device=DEV))
    new, x = [torch.zeros(3000, device=DEV)], torch.zeros(8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        with pytest.raises(eg.EgeriaError) as e:
            a.egeria_adamw_set_grads(new)
    assert e.value.status == eg.ERR_INVALID_ARG
    want = 0.9 * m[0].double() + 0.1 * g[0].double()
    size = 0.9 * m[0].double().abs() + 0.1 * g[0].double().abs()
    kept = weakref.ref(g[0])
    del g, new
    assert kept() is not None
    a.egeria_adamw_step(1e-3)
    close(m[0], want, 8 * 2.0 ** -24 * size + 1e-37, "m")


# ----------------------------------------------------------------------------- operands that overlap

def test_linear_refuses_an_output_that_overlaps_what_it_reads():
    o = ops.Ops(ops.egeria_linear_workspace_bytes(300, 64, 64), DEV)
    for rows in (3, 300):
        x, w, r = rand(rows, 64, seed=1), rand(64, 64, seed=2), rand(rows + 1, 64, seed=3)
        for bad in (dict(out=x), dict(out=x, residual=x), dict(residual=r[:-1], out=r[1:])):
            before = {k: t.clone() for k, t in bad.items()}
            with pytest.raises(eg.EgeriaError) as e:
                o.egeria_linear_forward(x, w, **bad)
            assert e.value.status == eg.ERR_INVALID_ARG
            assert all(torch.equal(bad[k], before[k]) for k in bad)
        both = torch.cat([w, rand(rows, 64, seed=4)])
        with pytest.raises(eg.EgeriaError):
            o.egeria_linear_forward(x, both[:64], out=both[63:63 + rows])
        bias = rand(rows * 64, seed=5)
        with pytest.raises(eg.EgeriaError):
            o.egeria_linear_forward(x, w, bias=bias[-64:], out=bias.view(rows, 64))


def test_linear_takes_operands_that_share_a_buffer_without_overlapping():
    """Columns of one buffer: input and output side by side, a residual between them, and different pitches."""
    rows = 150
    o = ops.Ops(ops.egeria_linear_workspace_bytes(rows, 64, 64), DEV)
    w = rand(64, 64, seed=2, scale=0.1)
    buf = rand(rows, 192, seed=1)
    x, r, y = buf[:, :64], buf[:, 64:128], buf[:, 128:]
    want = o.egeria_linear_forward(x.clone(), w, residual=r.clone())
    assert o.egeria_linear_forward(x, w, residual=r, out=y) is not None and torch.equal(y, want)
    o.egeria_linear_forward(x, w, residual=r, out=r)
    assert torch.equal(r, want)
    # rows of 64 every 192 values, and the output in the 65th of every second one's 128 gaps (a pitch of 384)
    buf = rand(2 * rows, 192, seed=7)
    y = buf.view(rows, 384)[:, 100:164]
    x = buf[:rows, :64]
    want = o.egeria_linear_forward(x.clone(), w)
    o.egeria_linear_forward(x, w, out=y)
    assert torch.equal(y, want)
    with pytest.raises(eg.EgeriaError):
        o.egeria_linear_forward(x, w, out=buf.view(rows, 384)[:, 150:214])       # 22 columns into every second row of x


# ----------------------------------------------------------------------------- sizes

@pytest.mark.parametrize("most,rows", [((13824, 768, 768), (1, 5, 1280, 5000, 13568)), ((10496, 1024, 1024), (768, 10240)),
                                       ((41000, 256, 256), (40000, 300))])
def test_linear_handle_takes_smaller_calls(most, rows):
    """A ragged last batch on the handle of the whole one."""
    o = ops.Ops(ops.egeria_linear_workspace_bytes(*most), DEV)
    _, inp, out = most
    w = rand(out, inp, seed=2, scale=inp ** -0.5)
    for n in rows:
        x, dy = rand(n, inp, seed=n), rand(n, out, seed=n + 1)
        own = ops.Ops(ops.egeria_linear_workspace_bytes(n, inp, out), DEV)
        assert torch.equal(o.egeria_linear_forward(x, w, act="relu"), own.egeria_linear_forward(x, w, act="relu"))
        for a, b in zip(o.egeria_linear_backward(dy, x, w), own.egeria_linear_backward(dy, x, w)):
            assert torch.equal(a, b)
    o.check_device_status()


@pytest.mark.parametrize("most,least", [(1025, 1024), (257, 256), (513, 300)])
def test_norm_handle_takes_fewer_columns(most, least):
    o = ops.Ops(ops.egeria_norm_workspace_bytes(9000, most), DEV)
    x, w = rand(9000, least, seed=1), rand(least, seed=2)
    y, h, st = o.egeria_norm_forward(x, x, w_pre=w)
    got = o.egeria_norm_backward(x, x, y, x, st, w_pre=w)
    own = ops.Ops(ops.egeria_norm_workspace_bytes(9000, least), DEV).egeria_norm_backward(x, x, y, x, st, w_pre=w)
    assert all(torch.equal(got[k], own[k]) for k in ("dx", "df", "dw_pre"))


@pytest.mark.parametrize("rows", [1, 2, 4])
def test_linear_of_a_few_rows_needs_no_workspace(rows):
    x, w = rand(rows, 1024, seed=1), rand(4096, 1024, seed=2, scale=1 / 32)
    own = ops.Ops(ops.egeria_linear_workspace_bytes(rows, 1024, 4096), DEV)
    assert torch.equal(ops.Ops(device=DEV).egeria_linear_forward(x, w), own.egeria_linear_forward(x, w))


def test_linear_of_one_row_with_the_most_outputs():
    """2^31 - 1024 outputs: the column of a warp's next turn passes 31 bits."""
    n = 2 ** 31 - 1024
    x = torch.full((1, 1), 3.0, dtype=torch.bfloat16, device=DEV)
    w = torch.full((n, 1), 0.5, dtype=torch.bfloat16, device=DEV)
    w[-1] = 2.0
    y = ops.Ops(device=DEV).egeria_linear_forward(x, w)
    assert y.shape == (1, n) and float(y[0, -1]) == 6.0 and float(y[0, 0]) == 1.5
    assert all((part == 1.5).all() for part in y[0, :-1].split(2 ** 28))


# ----------------------------------------------------------------------------- values at the ends

@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("inner", [False, True])
def test_slopes_of_huge_values(act, inner):
    """Where the argument is finite, however large, so is the slope (0 or 1 exactly from 1e3 on): through dz (act) and through
    dx's epilogue (act_in)."""
    n = 64
    sizes = torch.tensor([40.0, 1e3, 1e9, 1e12, 2e13, 1e15, 1e19, 3e19, 1e25, 3e38], device=DEV)
    z = torch.cat([sizes, -sizes]).repeat(n * n)[:n * n].view(n, n).to(torch.bfloat16)
    dy = rand(n, n, seed=3)
    eye = torch.eye(n, dtype=torch.bfloat16, device=DEV)
    o = ops.Ops(ops.egeria_linear_workspace_bytes(n, n, n), DEV)
    kw = dict(z_in=z, act_in=act) if inner else dict(z=z, act=act)
    dx, _, db = o.egeria_linear_backward(dy, eye, eye, **kw)
    ref = dy.double() * act64(z.double(), act)[1]
    close(dx, ref, (U[dx.dtype] + 2.0 ** -14) * ref.abs(), "dx")
    far = z.abs() >= 1e3
    assert torch.equal(dx[far], torch.where(z > 0, dy, torch.zeros_like(dy))[far])
    if not inner:
        close(db, ref.sum(0), U[db.dtype] * ref.sum(0).abs() + (n + 8) * 2.0 ** -23 * ref.abs().sum(0), "db")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows", [4, 500])
def test_activations_alone(rows, act, dtype):
    """x times the identity is x itself: what is left is the activation's own error, 2^-15 of the value (next to the zero of
    a slope, of its two terms), and one rounding.  The approximate units take what is below 2^-126 for zero, so
    that a value below |z| 2^-126 may be one."""
    n = 64
    z = torch.linspace(-12.0, 12.0, rows * n, device=DEV).to(dtype).view(rows, n)
    eye = torch.eye(n, dtype=dtype, device=DEV)
    o = ops.Ops(ops.egeria_linear_workspace_bytes(rows, n, n), DEV)
    zd = z.double()
    ref, slope = act64(zd, act)
    floor = TINY[dtype] + zd.abs() * 2.0 ** -126
    close(o.egeria_linear_forward(z, eye, act=act), ref, (U[dtype] + 2.0 ** -15) * ref.abs() + floor, "value")
    # the slope, of p + q: through dz and through dx's epilogue
    p = torch.where(zd == 0, torch.full_like(zd, 0.5), ref / zd)
    terms = p.abs() + (slope - p).abs()
    one = torch.ones_like(z)
    tol = U[dtype] * slope.abs() + 2.0 ** -15 * terms + TINY[dtype] + (1 + zd * zd) * 2.0 ** -126
    close(o.egeria_linear_backward(one, None, eye, z=z, act=act, need_dw=False)[0], slope, tol, "slope")
    close(o.egeria_linear_backward(one, None, eye, z_in=z, act_in=act, need_dw=False)[0], slope, tol, "slope in the epilogue")


@pytest.mark.parametrize("inner", [False, True])
def test_slope_of_gelu_next_to_its_zero(inner):
    """Every f16 argument between -0.8 and -0.7: Phi(z) and z times the density cancel at -0.75.  Each is at most 0.25 there and
    off by 2^-21 of itself (eight roundings of 2^-24): 2^-22 in all, and one rounding."""
    z = torch.arange(0x3999, 0x3A67, device=DEV).to(torch.int16).view(torch.float16).neg()
    z = torch.nn.functional.pad(z, (0, -len(z) % 64), value=-0.75).view(-1, 64)
    n, one, eye = z.shape[0], torch.ones_like(z), torch.eye(64, dtype=z.dtype, device=DEV)
    o = ops.Ops(ops.egeria_linear_workspace_bytes(n, 64, 64), DEV)
    kw = dict(z_in=z, act_in="gelu") if inner else dict(z=z, act="gelu")
    slope = act64(z.double(), "gelu")[1]
    assert float(slope.abs().min()) < 2.0 ** -12
    close(o.egeria_linear_backward(one, None, eye, need_dw=False, **kw)[0], slope, U[z.dtype] * slope.abs() + 2.0 ** -22 + TINY[z.dtype], "slope")


@pytest.mark.parametrize("act,at_zero", [("relu", 0.0), ("gelu", 0.5), ("gelu_tanh", 0.5), ("silu", 0.5)])
def test_slopes_at_both_zeros(act, at_zero):
    z = torch.zeros(64, 64, dtype=torch.bfloat16, device=DEV)
    z[::2] = -0.0
    one, eye = torch.ones_like(z), torch.eye(64, dtype=z.dtype, device=DEV)
    o = ops.Ops(ops.egeria_linear_workspace_bytes(64, 64, 64), DEV)
    for kw in (dict(z_in=z, act_in=act), dict(z=z, act=act)):
        assert (o.egeria_linear_backward(one, None, eye, need_dw=False, **kw)[0] == at_zero).all()
    assert not o.egeria_linear_forward(z, eye, act=act).any()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_second_moments_below_the_normal_range(bits):
    """Without an eps to hide it: a second moment of 1e-41 has a root.  It is held to 2^-149, so v is off by three units of
    that after its products and its sum, and the root by half of what v is off relatively."""
    n = 3000
    g = rand(n, dtype=torch.float32, seed=1).sign() * 1e-19 * (1 + torch.rand(n, device=DEV))
    kinds = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
    p, m, v = rand(n, dtype=torch.float32, seed=2), *(torch.zeros(n, dtype=t, device=DEV) for t in kinds)
    scales = {} if bits == 32 else {k: [torch.zeros(-(-n // 256), device=DEV)] for k in ("m_scales", "v_scales")}
    before, gd = p.double(), g.double()
    a = ops.AdamW([p], [g], [m], [v], torch.zeros(1, dtype=torch.int32, device=DEV), **scales)
    a.egeria_adamw_step(1e-2, 0.9, 0.999, eps=0.0)
    if bits == 32:
        close(v, 0.001 * gd * gd, 3 * 2.0 ** -149 + 2.0 ** -20 * 0.001 * gd * gd, "v")
    change = 1e-2 * gd.sign()                 # m and v corrected for the first step are g and g^2
    off = 3 * 2.0 ** -149 / (0.001 * gd * gd) + 2.0 ** -19
    close(p, before - change, 1e-2 * off + 2.0 ** -22 * before.abs(), "param")


# ----------------------------------------------------------------------------- autograd around the calls

def test_results_say_that_they_have_no_gradient():
    """Where an input requires grad, going back through a call's result is an error, not a gradient that is left out."""
    o = ops.Ops(max(ops.egeria_linear_workspace_bytes(8, 64, 64), ops.egeria_norm_workspace_bytes(8, 64)), DEV)
    x, w = rand(8, 64, seed=1), rand(64, 64, seed=2)
    plain = o.egeria_linear_forward(x, w, save_z=True)
    assert not any(t.requires_grad for t in plain)
    for hot in (dict(x=x.clone().requires_grad_(), w=w), dict(x=x, w=w.clone().requires_grad_())):
        y, z = o.egeria_linear_forward(**hot, save_z=True)
        assert torch.equal(y, plain[0]) and torch.equal(z, plain[1])
        for out in (y, z):
            with pytest.raises(RuntimeError, match="egeria_linear_backward"):
                (hot["x"].float().sum() + hot["w"].float().sum() + out.float().sum()).backward()
        with torch.no_grad():
            assert not o.egeria_linear_forward(**hot).requires_grad
    h = x.clone().requires_grad_()
    y, n, st = o.egeria_norm_forward(h, x)
    for out in (y, n, st):
        with pytest.raises(RuntimeError, match="egeria_norm_backward"):
            out.float().sum().backward()
    # gradients of the gradient calls are nobody's: plain tensors, as before
    assert not any(t.requires_grad for t in o.egeria_linear_backward(x, hot["x"], hot["w"]))


def test_in_place_results_raise_the_version():
    """Autograd's check of the tensors it has saved sees that a call has written to them."""
    o = ops.Ops(ops.egeria_linear_workspace_bytes(8, 64, 64), DEV)
    x, w, out = rand(8, 64, seed=1), rand(64, 64, seed=2), rand(8, 64, seed=3)
    a = torch.ones(8, 64, device=DEV, dtype=torch.bfloat16, requires_grad=True)
    product = a * out
    o.egeria_linear_forward(x, w, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.sum().backward()
    p = torch.nn.Parameter(rand(512, dtype=torch.float32, seed=4))
    loss = (p * p).sum()
    opt = ops.AdamW([p], [torch.ones(512, device=DEV)], [torch.zeros(512, device=DEV)], [torch.zeros(512, device=DEV)],
                    torch.zeros(1, dtype=torch.int32, device=DEV))
    opt.egeria_adamw_step(1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_handle_talks_to_the_library_it_was_made_with(monkeypatch):
    o = ops.Ops(ops.egeria_linear_workspace_bytes(8, 64, 64), DEV)
    p, g, m, v = ([rand(300, dtype=torch.float32, seed=k)] for k in range(4))
    a = ops.AdamW(p, g, m, v, torch.zeros(1, dtype=torch.int32, device=DEV))

    def other():
        raise AssertionError("the library in force now may be another one")

    monkeypatch.setattr(ops, "lib", other)
    o.egeria_linear_forward(rand(8, 64), rand(64, 64))
    o.check_device_status()
    a.egeria_adamw_set_grads(g)
    a.egeria_adamw_step(1e-3)
    a.check_device_status()
    assert o.egeria_ops_launch_count() >= 1 and a.egeria_adamw_launch_count() == 1


# ----------------------------------------------------------------------------- bounded waits

@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rows,inp,out", [(300, 4096, 192), (64, 2048, 64), (2048, 1024, 4096), (4096, 768, 768)])
def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(kind, rows, inp, out):
    """The give-up path of the products' kernel: the first worker issues no loads (1) or stops after its first stage (2), for one
    launch whose waits are limited to a millisecond.  The kernel returns, the status says EGERIA_ERR_TIMEOUT once, and the
    next call is whole: split products (whose tickets the others have raised), pairs of thread blocks, single ones."""
    o = ops.Ops(ops.egeria_linear_workspace_bytes(rows, inp, out), DEV)
    x, w = rand(rows, inp, seed=1), rand(out, inp, seed=2, scale=inp ** -0.5)
    want = o.egeria_linear_forward(x, w)
    o.check_device_status()
    o.egeria_ops_debug_stall_next(kind)
    o.egeria_linear_forward(x, w)
    assert o.egeria_ops_device_status() == eg.ERR_TIMEOUT
    assert o.egeria_ops_device_status() == eg.OK
    for _ in range(2):
        assert torch.equal(o.egeria_linear_forward(x, w), want)
    o.check_device_status()


# ----------------------------------------------------------------------------- gradients against differences

def test_linear_gradients_along_themselves():
    """A step along a gradient changes the loss by the gradient's square.  The outputs' roundings are each within
    2^-11 |y|, independent and weighted by c: six deviations of their sum are the noise; the step moves z by some 0.1, so that
    its third derivative is under 2 % of the change; the gradient's own rounding is far below that."""
    rows, inp, out, t = 40, 48, 56, torch.float16
    o = ops.Ops(ops.egeria_linear_workspace_bytes(rows, inp, out), DEV)
    x, w, b, c = rand(rows, inp, dtype=t, seed=1), rand(out, inp, dtype=t, seed=2, scale=0.15), rand(out, dtype=t, seed=3), rand(rows, out, dtype=t, seed=4)

    def outputs(x, w, b):
        return o.egeria_linear_forward(x, w, bias=b, act="gelu").double()

    y, z = o.egeria_linear_forward(x, w, bias=b, act="gelu", save_z=True)
    noise = 6 * 2.0 ** -11 / math.sqrt(3) * math.sqrt(2.0) * float((c.double() * y.double()).square().sum().sqrt())
    for which, grad in enumerate(o.egeria_linear_backward(c, x, w, z=z, act="gelu")):
        args = [x, w, b]
        moved = [grad.double() @ w.double().t(), x.double() @ grad.double().t(), grad.double().view(1, -1)][which] if which < 2 else grad.double()
        step = 0.1 / float(moved.abs().max())
        up, down = list(args), list(args)
        up[which] = (args[which].double() + step * grad.double()).to(t)
        down[which] = (args[which].double() - step * grad.double()).to(t)
        slope = float((grad.double() * (up[which].double() - down[which].double())).sum())
        change = float(((outputs(*up) - outputs(*down)) * c.double()).sum())
        assert slope > 8 * noise                          # a gradient of zero, or of the other sign, is far outside
        assert abs(change - slope) <= noise + 0.02 * slope, (which, change, slope, noise)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_gradients_along_themselves(kind):
    """The same for the residual norms in 32 bits, every gradient: the outputs are off by (cols + 64) 2^-24 of their parts."""
    rows, cols, t = 24, 72, torch.float32
    o = ops.Ops(ops.egeria_norm_workspace_bytes(rows, cols), DEV)
    s = dict(x=rand(rows, cols, dtype=t, seed=1), f=rand(rows, cols, dtype=t, seed=2), gate=rand(6, cols, dtype=t, seed=3, base=0.5))
    for k in ("post", "pre"):
        s["w_" + k], s["b_" + k] = rand(cols, dtype=t, seed=4, scale=0.2, base=1.0), rand(cols, dtype=t, seed=5)
    dy, dh = rand(rows, cols, dtype=t, seed=8), rand(rows, cols, dtype=t, seed=9)

    def loss(s):
        y, h, _ = o.egeria_norm_forward(s["x"], s["f"], **{k: s[k] for k in s if k not in "xf"}, gate_rows=4, kind=kind, alpha=0.75)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    vectors = {k: s[k] for k in s if k not in "xf"}
    y, h, st = o.egeria_norm_forward(s["x"], s["f"], **vectors, gate_rows=4, kind=kind, alpha=0.75)
    noise = (cols + 64) * 2.0 ** -24 * 8 * float((dy.double().abs() * y.double().abs()).sum() + (dh.double().abs() * (1 + h.double().abs())).sum())
    got = o.egeria_norm_backward(dy, dh, y, s["f"], st, **vectors, gate_rows=4, kind=kind, alpha=0.75)
    for k in s:
        grad = got["d" + k]
        step = 0.02 / float(grad.abs().max())             # no value moves by more than 0.02 of the norm of what it is among
        up, down = (dict(s, **{k: s[k] + sign * step * grad}) for sign in (1, -1))
        slope = float((grad.double() * (up[k].double() - down[k].double())).sum())
        change = loss(up) - loss(down)
        assert slope > 8 * noise, k
        assert abs(change - slope) <= noise + 0.02 * slope, (k, change, slope, noise)


# ----------------------------------------------------------------------------- aliases

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


def _struct(name, fields):
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for t, names in fields for f in names.split()]})


NormForward = _struct("NormForward", ((_i32, "type param_type kind post pre"), (_f32, "alpha eps"), (_i64, "rows cols gate_rows"),
                                      (_vp, "x f gate w_post b_post w_pre b_pre"), (_i64, "ldx ldf"), (_vp, "y h"), (_i64, "ldy ldh"), (_vp, "stats")))
NormBackward = _struct("NormBackward", ((_i32, "type param_type kind post pre"), (_f32, "alpha"), (_i64, "rows cols gate_rows"),
                                        (_vp, "dy dh y f gate w_post b_post w_pre b_pre"), (_i64, "lddy lddh ldy ldf"), (_vp, "stats dx df"),
                                        (_i64, "lddx lddf"), (_vp, "dgate dw_post db_post dw_pre db_pre")))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols,pitch,dtype", [(700, 256, 256, torch.bfloat16), (700, 250, 256, torch.bfloat16), (333, 1001, 1003, torch.float16),
                                                   (90, 1536, 1544, torch.bfloat16), (40, 4096, 4096, torch.float32), (31, 8192, 8192, torch.float32),
                                                   (31, 8192, 8192, torch.bfloat16)])
def test_norm_writes_onto_what_it_reads(rows, cols, pitch, dtype, kind):
    """y = x, h = f; dx = dy with df = f or df = dh: the same bits as with separate outputs, at wide and narrow pitches and where
    one row or three are on their way (8192 columns of float are one)."""
    o = ops.Ops(ops.egeria_norm_workspace_bytes(rows, cols), DEV)
    L, stream = ops.lib(), torch.cuda.current_stream().cuda_stream
    t = ops.TYPES[dtype]

    def matrix(seed):
        return rand(rows, pitch, dtype=dtype, seed=seed)

    w, gate = rand(cols, dtype=dtype, seed=1, base=1.0), rand(-(-rows // 7), cols, dtype=dtype, seed=2)
    common = dict(type=t, param_type=t, kind=ops.KINDS[kind], post=1, pre=1, alpha=0.5, rows=rows, cols=cols, gate_rows=7, gate=gate.data_ptr(),
                  w_post=w.data_ptr(), w_pre=w.data_ptr())

    def forward(x, f, y, h):
        st = torch.zeros(rows, 4, device=DEV)
        a = NormForward(**common, eps=1e-5, x=x.data_ptr(), f=f.data_ptr(), y=y.data_ptr(), h=h.data_ptr(), ldx=pitch, ldf=pitch, ldy=pitch, ldh=pitch,
                        stats=st.data_ptr())
        assert L.egeria_norm_forward(o._h, _vp(stream), ctypes.byref(a)) == eg.OK
        return st

    x, f = matrix(3), matrix(4)
    y, h = x.clone(), f.clone()                   # (what lies between the rows stays what it was)
    st = forward(x, f, y, h)
    x2, f2 = x.clone(), f.clone()
    assert torch.equal(forward(x2, f2, x2, f2), st)
    assert torch.equal(x2, y) and torch.equal(f2, h)

    def backward(dy, dh, f, dx, df):
        dgate, dw_post, dw_pre = torch.zeros_like(gate), torch.zeros_like(w), torch.zeros_like(w)
        a = NormBackward(**common, dy=dy.data_ptr(), dh=dh.data_ptr(), y=y.data_ptr(), f=f.data_ptr(), lddy=pitch, lddh=pitch, ldy=pitch, ldf=pitch,
                         stats=st.data_ptr(), dx=dx.data_ptr(), df=df.data_ptr(), lddx=pitch, lddf=pitch, dgate=dgate.data_ptr(),
                         dw_post=dw_post.data_ptr(), dw_pre=dw_pre.data_ptr())
        assert L.egeria_norm_backward(o._h, _vp(stream), ctypes.byref(a)) == eg.OK
        return dgate, dw_post, dw_pre

    dy, dh = matrix(5), matrix(6)
    dx, df = dy.clone(), f.clone()
    sums = backward(dy, dh, f, dx, df)
    for onto in ("f", "dh"):
        g = dict(dy=dy.clone(), dh=dh.clone(), f=f.clone())
        again = backward(g["dy"], g["dh"], g["f"], g["dy"], g[onto])
        assert all(torch.equal(p, q) for p, q in zip(sums, again))
        assert torch.equal(g["dy"], dx) and torch.equal(g[onto][:, :cols], df[:, :cols])
    o.check_device_status()


# ----------------------------------------------------------------------------- the checked build

def test_checked_build_finds_nothing_on_the_operators():
    """A cross-section of the operators' tests on the second library, whose kernels check their indexes, in a process of its
    own: the same results, and no check fires (the tests end with a status query, which would say EGERIA_ERR_CHECK)."""
    here = Path(__file__).resolve().parent
    r = subprocess.run([sys.executable, "-m", "pytest", str(here / "test_ops_gpu.py"), "-m", "gpu", "-x", "-q", "--checked-library", "-p", "no:cacheprovider",
                        "-k", "linear_forward or linear_backward or linear_larger or norm_sizes or norm_gate_groups or adamw_types or frozen_modules"],
                       capture_output=True, text=True, cwd=str(here.parent))
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
