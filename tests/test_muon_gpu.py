"""GPU parity of the Muon step against the formula in 64 bits.

Tolerances, derived before the first run.  One step of the orthogonalisation is bounded value by value: the products' operands are
rounded by 2^-11 of themselves (X once, A once, a I + b A + c A^2 once), what X's rounding leaves by 2^-21 of X and multiplied by a
alone, a value of f16 below 2^-14 by 2^-25; with N = |X| |X|^T that gives the sums written out in `one_step`.  Over five steps the
roundings of one go into the next.  Near 1, where the singular values end, |b A + c A^2| is at most 2.81, by which X's rounding is
multiplied, while the step returns at least 0.67 of X; A's rounding moves it by 0.72 at most, its own by itself; and a step's slope is
at most 0.72 there: a step adds at most 2^-11 (2.81 + 0.72 + 0.67) / 0.67 = 3.1e-3, five of them 3.1e-3 / (1 - 0.72) = 1.1e-2 of a single
singular value, and 1.7e-2 is allowed for.  Over a matrix the roundings are independent, of root mean square 2^-11 / sqrt(12) or less:
sqrt(2) 2.81 / 0.67 / sqrt(12) 2^-11 = 8.4e-4 a step at most, 1.2e-3 for five; six times that is allowed for in the 2-norm, 7e-3.
"""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops
from test_ops_gpu import DEV, U, close

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315
MATRIX, VECTOR = 7e-3, 1.7e-2


def normal(*shape, seed=0, scale=1.0, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(4321 + seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def low_rank(rows, cols, rank, seed=0, noise=0.0):
    return normal(rows, rank, seed=seed) @ normal(rank, cols, seed=seed + 1) + noise * normal(rows, cols, seed=seed + 2)


def orthogonal64(t, steps=5, eps=1e-7):
    x = t.double().reshape(t.shape[0], -1)
    x = x / x.norm().clamp(min=eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(steps):
        a = x @ x.t()
        x = A * x + (B * a + C * a @ a) @ x
    return (x.t() if tall else x).reshape(t.shape)


def orthogonalised(grads, steps=5, **more):
    """The kernel's X of these matrices: the weights that a step with lr = scale = 1 and no momentum makes of zeros."""
    params = [torch.zeros(g.shape, device=DEV) for g in grads]
    m = ops.Muon(params, grads, [torch.zeros(g.shape, device=DEV) for g in grads], scale=1.0, ns_steps=steps)
    m.egeria_muon_step(1.0, beta=0.0, nesterov=False, **more)
    m.check_device_status()
    return [-p for p in params]


def near(got, want, tol, what=""):
    off, size = float((got.double() - want).norm()), float(want.norm())
    assert off <= tol * size, f"{what}: off by {off / size:.2e} of itself"


SHAPES = [(1, 1), (1, 700), (700, 1), (2, 3), (16, 144), (33, 47), (47, 33), (64, 64), (64, 576), (100, 100), (128, 128), (129, 257), (257, 129),
          (130, 1000), (519, 519), (333, 1332), (1332, 333), (1024, 256), (128, 768), (768, 128), (100, 767), (767, 65), (128, 769), (129, 768), (1, 768), (5, 65)]


def one_step(t):
    """(X after one step, bound of its error value by value)."""
    x = t.double() / t.double().norm()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    a, n = x @ x.t(), x.abs() @ x.abs().t()
    want = A * x + (B * a + C * a @ a) @ x
    da = (2.0 ** -10 + 2.0 ** -11 + 2.0 ** -16) * n + 2.0 ** -25
    size = -B * n + C * n @ n
    size = size + A * torch.eye(len(n), device=DEV, dtype=torch.float64)
    db = -B * da + C * (n @ da + da @ n + da @ da) + 2.0 ** -11 * (size + db_size(da)) + 2.0 ** -25
    # the product takes X's first value alone, of the second a is taken: what is left out is (b A + c A^2) times it
    tol = db @ x.abs() * (1 + 2.0 ** -10) + 2.0 ** -11 * (size + db) @ x.abs() + 2.0 ** -20 * A * x.abs() + 2.0 ** -20 * want.abs() + 2.0 ** -40
    return (want.t(), tol.t()) if tall else (want, tol)


def db_size(da):
    return 5.0 * da


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_one_step(rows, cols):
    t = normal(rows, cols, seed=rows + cols)
    want, tol = one_step(t)
    close(orthogonalised([t], steps=1)[0], want, tol, "X")


def test_one_step_of_many_matrices():
    """More tiles than thread blocks, pairs of them, every shape at once."""
    grads = [normal(r, c, seed=r + 3 * c) for r, c in SHAPES + [(1024, 1024), (2048, 512), (512, 2048), (1000, 3000), (3000, 1000), (2049, 2051)]]
    for x, t in zip(orthogonalised(grads, steps=1), grads):
        want, tol = one_step(t)
        close(x, want, tol, str(tuple(t.shape)))


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 6, 16])
def test_steps(steps):
    grads = [normal(96, 160, seed=1), normal(300, 200, seed=2), low_rank(128, 128, 8, seed=3, noise=0.1)]
    for x, t in zip(orthogonalised(grads, steps=steps), grads):
        near(x, orthogonal64(t, steps), MATRIX, f"{steps} steps of {tuple(t.shape)}")


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_five_steps(rows, cols):
    t = normal(rows, cols, seed=rows + cols)
    near(orthogonalised([t])[0], orthogonal64(t), VECTOR if min(rows, cols) < 16 else MATRIX)


@pytest.mark.parametrize("rows,cols", [(256, 256), (200, 900), (900, 200), (1024, 1024)])
def test_matrices_of_low_rank(rows, cols):
    """What lies across the null space is multiplied by a in every step and must not be a rounding."""
    kinds = [(r, e) for r in (1, 4, 16) for e in (0.0, 1e-3, 0.1)]
    grads = [low_rank(rows, cols, r, seed=r, noise=e) for r, e in kinds]
    for x, t, (rank, _) in zip(orthogonalised(grads), grads, kinds):
        near(x, orthogonal64(t), VECTOR if rank < 16 else MATRIX)


def test_larger_matrices():
    grads = [normal(1024, 1024, seed=k) for k in range(5)] + [normal(4096, 1024, seed=9), normal(1024, 4096, seed=10), normal(2048, 5632, seed=11),
                                                              low_rank(2048, 2048, 128, seed=12, noise=0.2)]
    for x, t in zip(orthogonalised(grads), grads):
        near(x, orthogonal64(t), MATRIX)


# ----------------------------------------------------------------------------- the whole step

class Model:
    """Matrices with their state, and the same in 64 bits."""

    def __init__(self, shapes, dtype=torch.float32, gtype=None, master=False, wd=0.1, scale="rms", modules=None, shift=0, seed=0):
        self.shapes, self.dtype = shapes, dtype

        def place(values, kind):
            """The values at an offset of `shift` values in a buffer of their own."""
            buf = torch.zeros(values.numel() + shift, dtype=kind, device=DEV)
            v = buf[shift:].view(values.shape)
            v.copy_(values)
            return v

        weights = [normal(*s, seed=seed + 10 * i, scale=0.05) for i, s in enumerate(shapes)]
        self.params = [place(w, dtype) for w in weights]
        self.masters = [place(w, torch.float32) for w in weights] if master else None
        self.m = [place(normal(*s, seed=seed + 10 * i + 1, scale=0.01), torch.float32) for i, s in enumerate(shapes)]
        self.grads = [place(normal(*s, seed=seed + 10 * i + 2, scale=0.02), gtype or dtype) for i, s in enumerate(shapes)]
        self.wd, self.modules = wd, modules or [-1] * len(shapes)
        self.scales = [0.2 * max(s[0], p.numel() // max(s[0], 1)) ** 0.5 for s, p in zip(shapes, self.params)]
        self.muon = ops.Muon(self.params, self.grads, self.m, masters=self.masters, weight_decay=wd, scale=scale, modules=modules)

    def held(self):
        return self.masters if self.masters is not None else self.params

    def check(self, lr=1e-2, beta=0.9, nesterov=True, grad_scale=None, frozen=None, **more):
        before = [p.double().clone() for p in self.held()]
        kept = [(p.clone(), m.clone()) for p, m in zip(self.params, self.m)]
        gs = None if grad_scale is None else torch.full((1,), grad_scale, device=DEV)
        mask = None if frozen is None else torch.tensor(frozen, dtype=torch.uint8, device=DEV)
        self.muon.egeria_muon_step(lr, beta=beta, nesterov=nesterov, grad_scale=gs, frozen=mask, **more)
        self.muon.check_device_status()
        for i, p in enumerate(self.params):
            if p.numel() == 0:
                continue
            if frozen is not None and self.modules[i] >= 0 and frozen[self.modules[i]]:
                assert torch.equal(p, kept[i][0]) and torch.equal(self.m[i], kept[i][1])
                assert torch.equal(self.held()[i].double(), before[i])
                continue
            g = self.grads[i].double() * (1.0 if grad_scale is None else grad_scale)
            old = kept[i][1].double()
            m = beta * old + (1 - beta) * g
            # a product with beta and 1 - beta as floats, and the sum: four roundings of the two terms
            close(self.m[i], m, 2.0 ** -22 * (beta * old.abs() + (1 - beta) * g.abs()) + 2.0 ** -126, "m")
            x = orthogonal64(beta * m + (1 - beta) * g if nesterov else m)
            move = lr * self.scales[i] * x
            want = before[i] * (1 - lr * self.wd) - move
            got, held = p.double(), self.held()[i].double()
            off = (held - want).norm()
            tol = VECTOR if min(x.shape[0], x.numel() // x.shape[0]) < 16 else MATRIX
            rounding = U[self.held()[i].dtype] * (want.abs() + tol * move.abs()) + 2.0 ** -23 * (before[i].abs() + move.abs())
            assert off <= tol * move.norm() + rounding.norm(), (self.shapes[i], float(off / move.norm()))
            if self.masters is not None:
                assert torch.equal(p, self.masters[i].to(self.dtype))
            assert got.shape == before[i].shape
        return self


MIXED = [(64, 64), (40, 100), (100, 40), (257, 65), (8, 3, 3, 3), (16, 16, 3, 3), (200, 136), (136, 1000)]


@pytest.mark.parametrize("dtype,gtype,master", [(torch.float32, torch.float32, False), (torch.bfloat16, torch.bfloat16, False),
                                                (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, True),
                                                (torch.float16, torch.float16, False), (torch.float16, torch.float32, True),
                                                (torch.float32, torch.float32, True)])
def test_types(dtype, gtype, master):
    model = Model(MIXED, dtype, gtype, master)
    for _ in range(3):
        model.check()


@pytest.mark.parametrize("shift", [1, 4, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_unaligned_matrices(dtype, shift):
    Model([(64, 64), (40, 96), (33, 17), (300, 264)], dtype, shift=shift, master=dtype != torch.float32).check().check(nesterov=False)


def test_matrices_side_by_side_in_one_buffer():
    """Weights and momenta of all matrices without a gap between them; a neighbour's values stay its own.  The same matrix twice is refused."""
    model = Model([(33, 17), (64, 64), (300, 264), (7, 5)])
    flat = torch.cat([t.flatten() for pair in zip(model.params, model.m) for t in pair])
    at = 0
    for i, p in enumerate(model.params):
        for column in (model.params, model.m):
            column[i] = flat[at:at + p.numel()].view(p.shape)
            at += p.numel()
    model.muon = ops.Muon(model.params, model.grads, model.m, weight_decay=model.wd)
    model.check().check()
    with pytest.raises(eg.EgeriaError):
        ops.Muon(model.params + model.params[:1], model.grads + model.grads[:1], model.m + [torch.zeros(33, 17, device=DEV)])


@pytest.mark.parametrize("lr,beta,nesterov,wd,gs", [(1e-3, 0.95, True, 0.0, None), (1e-2, 0.0, True, 0.5, 2.0), (0.0, 0.5, False, 0.0, 1.0),
                                                    (1e-2, 0.99, False, 0.1, 2.0 ** -16)])
def test_settings(lr, beta, nesterov, wd, gs):
    Model([(64, 64), (48, 200)], wd=wd).check(lr=lr, beta=beta, nesterov=nesterov, grad_scale=gs)


def test_scales():
    for scale, want in (("rms", [0.2 * 96 ** 0.5, 0.2 * 96 ** 0.5]), ("spectral", [3 ** 0.5, 1.0]), (2.5, [2.5, 2.5]), ([0.5, 0.25], [0.5, 0.25])):
        model = Model([(96, 32), (32, 96)], scale=scale)
        model.scales = want
        model.check()


def test_frozen_modules_are_left_alone():
    shapes = [(64, 64), (40, 100), (300, 264), (64, 64), (24, 24)]
    model = Model(shapes, torch.bfloat16, master=True, modules=[0, 1, 1, 2, -1])
    for frozen in ([0, 0, 0], [1, 0, 0], [1, 1, 0], [1, 1, 1], [0, 1, 0]):
        model.check(frozen=frozen)


@pytest.mark.parametrize("side", [64, 300])
def test_frozen_gradients_may_be_nan(side):
    model = Model([(side, side), (side, side)], modules=[0, 1])
    model.grads[0].fill_(float("nan"))
    model.check(frozen=[1, 0])


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_a_bad_scale_leaves_the_step_out(bad):
    model = Model([(64, 64), (300, 264)], torch.bfloat16, master=True)
    before = [t.clone() for t in (*model.params, *model.masters, *model.m)]
    model.muon.egeria_muon_step(1e-2, grad_scale=torch.full((1,), bad, device=DEV))
    model.muon.check_device_status()
    assert all(torch.equal(a, b) for a, b in zip(before, (*model.params, *model.masters, *model.m)))
    model.check()


@pytest.mark.parametrize("shapes", [[(64, 64), (100, 130), (64, 64)], [(300, 264), (130, 777), (300, 264)]])
def test_a_bad_gradient_stays_in_its_matrix(shapes):
    for bad in (float("nan"), float("inf")):
        model = Model(shapes)
        model.grads[1][3, 5] = bad
        alone = Model(shapes)
        model.muon.egeria_muon_step(1e-2)
        alone.muon.egeria_muon_step(1e-2)
        assert torch.isnan(model.params[1]).all()
        assert torch.equal(model.params[0], alone.params[0]) and torch.equal(model.params[2], alone.params[2])
        # and the workspace keeps nothing of it: put back, the matrix steps as it would have
        for mine, other in ((model.params, alone.params), (model.m, alone.m), (model.grads, alone.grads)):
            mine[1].copy_(other[1])
        model.check()


def test_zero_gradients():
    """X is 0, not 0 / 0: the weights only decay."""
    model = Model([(64, 64), (5, 7)])
    for t in (*model.grads, *model.m):
        t.zero_()
    before = [p.double() for p in model.params]
    model.muon.egeria_muon_step(1e-2)
    for p, b in zip(model.params, before):
        close(p, b * (1 - 1e-3), 2.0 ** -22 * b.abs())


@pytest.mark.parametrize("size", [1e-25, 1e-12, 1.0, 1e18, 1e30])
def test_gradients_of_any_size(size):
    t = normal(64, 200, seed=3)
    params = [torch.zeros(64, 200, device=DEV)]
    m = ops.Muon(params, [t * size], [torch.zeros(64, 200, device=DEV)], scale=1.0)
    m.egeria_muon_step(1.0, beta=0.0, nesterov=False, eps=1e-30)
    m.check_device_status()
    near(-params[0], orthogonal64(t), MATRIX)


def test_small_gradients_are_held_by_eps():
    t = normal(64, 64, seed=4, scale=1e-8)
    x = orthogonalised([t], steps=1, eps=1.0)[0]
    want = A * t.double()               # |t| < 1: X = t, whose cubes are nothing
    close(x, want, 2.0 ** -10 * want.abs() + 2.0 ** -23)


def test_empty_matrices():
    model = Model([(0, 64), (64, 64), (64, 0)])
    model.check()
    assert Model([(0, 5)]).muon.egeria_muon_launch_count() == 0
    Model([(0, 5)]).muon.egeria_muon_step(1e-2)


def test_same_bits_every_time():
    shapes = MIXED + [(1024, 1024), (512, 1536), (1536, 512), (2048, 1024), (1024, 1024)]
    first = None
    for _ in range(4):
        model = Model(shapes, torch.bfloat16, master=True)
        for _ in range(2):
            model.muon.egeria_muon_step(1e-2)
        first = first or [m.clone() for m in model.masters]
        assert all(torch.equal(a, b) for a, b in zip(first, model.masters))
        del model
        torch.cuda.empty_cache()


def test_new_gradients_streams_and_graphs():
    model, plain = Model(MIXED), Model(MIXED)
    fresh = [normal(*s, seed=90 + i) for i, s in enumerate(MIXED)]
    model.muon.egeria_muon_set_grads(fresh)
    plain.muon.egeria_muon_set_grads([f.clone() for f in fresh])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    model.muon.egeria_muon_step(1e-2, stream=side)
    side.synchronize()
    plain.muon.egeria_muon_step(1e-2)
    assert all(torch.equal(a, b) for a, b in zip(model.params, plain.params))
    graph = torch.cuda.CUDAGraph()
    mask = torch.zeros(1, dtype=torch.uint8, device=DEV)
    with torch.cuda.graph(graph):
        model.muon.egeria_muon_step(1e-2, frozen=mask, stream=torch.cuda.current_stream())
    for k in range(3):
        for f, g in zip(fresh, plain.muon._grads):
            f.copy_(normal(*f.shape, seed=200 + k))
            g.copy_(f)
        graph.replay()
        plain.muon.egeria_muon_step(1e-2)
        assert all(torch.equal(a, b) for a, b in zip(model.params, plain.params))
    model.muon.check_device_status()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(eg.EgeriaError):
            model.muon.egeria_muon_set_grads(fresh, stream=torch.cuda.current_stream())


def test_two_handles_at_once():
    """Steps of two models on two streams, whose thread blocks wait for one another within each: each is whole."""
    shapes = [(1024, 1024)] * 3 + [(512, 2048), (2048, 512)]
    models = [Model(shapes, seed=k) for k in range(2)]
    plain = [Model(shapes, seed=k) for k in range(2)]
    for m in plain:
        for _ in range(4):
            m.muon.egeria_muon_step(1e-2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in models]
    for _ in range(4):
        for m, s in zip(models, streams):
            m.muon.egeria_muon_step(1e-2, stream=s)
    torch.cuda.synchronize()
    for m, p in zip(models, plain):
        m.muon.check_device_status()
        assert all(torch.equal(a, b) for a, b in zip(m.params, p.params))


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("shapes", [[(64, 64), (100, 40)], [(300, 200), (200, 900)], [(1024, 1024)] * 20 + [(512, 2048), (64, 64)]])
def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(shapes, kind):
    model = Model(shapes)
    model.muon.egeria_muon_debug_stall_next(kind)
    model.muon.egeria_muon_step(1e-2)
    assert model.muon.egeria_muon_device_status() == eg.ERR_TIMEOUT
    assert model.muon.egeria_muon_device_status() == eg.OK
    for _ in range(2):
        model.check()


def test_parameters_get_a_new_version():
    p = torch.nn.Parameter(normal(64, 64))
    loss = (p * p).sum()
    m = ops.Muon([p], [normal(64, 64, seed=1)], [torch.zeros(64, 64, device=DEV)])
    m.egeria_muon_step(1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_refusals():
    p, g, m = normal(8, 8), normal(8, 8), torch.zeros(8, 8, device=DEV)
    for bad in (dict(params=[]), dict(params=[normal(64)]), dict(params=[p.double()]), dict(grads=[g.bfloat16()]), dict(grads=[g.t()[:4]]),
                dict(momenta=[m.half()]), dict(momenta=[m.cpu()]), dict(grads=[]), dict(scale="huge"), dict(scale=[1.0, 2.0]), dict(modules=[1, 2]),
                dict(masters=[m.half()]), dict(params=[p.t()])):
        with pytest.raises((ValueError, eg.EgeriaError)):
            ops.Muon(**{**dict(params=[p], grads=[g], momenta=[m]), **bad})
    for bad in (dict(ns_steps=0), dict(ns_steps=17), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(eg.EgeriaError):
            ops.Muon([p], [g], [m], **bad)
    o = ops.Muon([p], [g], [m], modules=[2])
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=1e-3, beta=1.0), dict(lr=1e-3, beta=-0.1), dict(lr=1e-3, eps=0.0),
                dict(lr=1e-3, eps=float("inf"))):
        with pytest.raises(eg.EgeriaError) as e:
            o.egeria_muon_step(**bad)
        assert e.value.status == eg.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        o.egeria_muon_step(1e-3, frozen=torch.zeros(2, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        o.egeria_muon_step(1e-3, grad_scale=torch.zeros(2, device=DEV))
    with pytest.raises(ValueError):
        o.egeria_muon_set_grads([normal(8, 9)])
    before = p.clone()
    o.egeria_muon_step(0.0, frozen=torch.zeros(3, dtype=torch.uint8, device=DEV))
    assert torch.equal(p, before)


def test_checked_build_finds_nothing():
    """A cross-section of these tests and the gated blocks' on the second library, whose kernels check their indexes."""
    here = Path(__file__).resolve().parent
    r = subprocess.run([sys.executable, "-m", "pytest", str(here / "test_muon_gpu.py"), str(here / "test_gated_gpu.py"), "-m", "gpu", "-x", "-q",
                        "--checked-library", "-p", "no:cacheprovider", "-k",
                        "one_step or types or frozen_modules or test_forward or test_backward or larger or strides"],
                       capture_output=True, text=True, cwd=str(here.parent))
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
