"""GPU tests of the orthogonalised (Muon) update against its formula in 64 bits.

The library states the direction to be within about 1e-3 of the exact one in the
Frobenius norm (its products' operands have 11 significant bits, some fifteen
roundings, spread by the polynomial's slopes): the bound is twice that, and half
a unit of the last bit where the result is bf16 (2^-9).  Momentum and weights are
fp32 sums of a few terms.
"""
import math

import numpy as np
import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300.muon import MuonPlan

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, UBF = 2.0 ** -24, 2.0 ** -8
TOL = 2e-3
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def _lib(gpu):
    B.load()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _matrix(r, c, g, kind="gauss", std=1e-3):
    x = torch.randn(r, c, generator=g, device=DEV, dtype=torch.float64)
    if kind == "low rank":
        k = max(1, min(4, r, c))
        a = torch.randn(r, k, generator=g, device=DEV, dtype=torch.float64)
        b = torch.randn(k, c, generator=g, device=DEV, dtype=torch.float64)
        x = a @ b + 0.1 * x
    elif kind == "rows":      # rows of very different sizes
        x *= torch.logspace(0, -3, r, device=DEV, dtype=torch.float64)[:, None]
    return x * std


def _exact(u, steps=5, abc=ABC, eps=1e-7):
    a, b, c = abc
    u = u.double()
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (x.norm() + eps)
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + b * (gram @ x) + c * (gram @ (gram @ x))
    return x.T if u.shape[0] > u.shape[1] else x


def _near(got, want, tol, what=""):
    err = float((got.double() - want).norm())
    size = float(want.norm())
    assert err <= tol * size + 1e-30, (what, err / max(size, 1e-300))


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (64, 32), (32, 10), (10, 4096),
          (127, 129), (128, 256), (257, 129), (130, 1000), (1001, 65),
          (256, 256), (384, 768)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["gauss", "low rank"])
def test_direction(dtype, kind):
    """All shapes in one plan."""
    g = _gen(1)
    u = [_matrix(r, c, g, kind).to(DT[dtype]) for r, c in SHAPES]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in SHAPES]
    plan = MuonPlan(SHAPES, grad_dtype=dtype)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y, s in zip(u, o, SHAPES):
        _near(y, _exact(x), TOL + UBF / 2, s)
    assert plan.query() == 0
    first = [y.clone() for y in o]
    plan.direction(B.make_muon_hyper())
    assert all(torch.equal(a, b) for a, b in zip(first, o))


@pytest.mark.parametrize("shape", [(512, 1024), (700, 600), (1024, 1024)])
def test_direction_of_larger_matrices(shape):
    g = _gen(2)
    u = [_matrix(*shape, g, "low rank").bfloat16() for _ in range(3)]
    o = [torch.empty_like(x) for x in u]
    plan = MuonPlan([shape] * 3, grad_dtype="bf16")
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y in zip(u, o):
        _near(y, _exact(x), TOL + UBF / 2)


@pytest.mark.parametrize("shape", [(48, 80), (200, 144), (300, 300)])
def test_direction_is_nearly_orthogonal(shape):
    """Singular values of a Gaussian matrix end in the polynomial's band."""
    u = _matrix(*shape, _gen(3)).float()
    o = torch.empty(shape, device=DEV, dtype=torch.bfloat16)
    plan = MuonPlan([shape])
    plan.bind_direction([u], [o])
    plan.direction(B.make_muon_hyper(steps=8))
    s = np.linalg.svd(o.double().cpu().numpy(), compute_uv=False)
    assert s.max() < 1.3
    assert np.median(s) > 0.6


@pytest.mark.parametrize("steps,abc", [(1, ABC), (2, (1.5, -0.5, 0.0)),
                                       (12, (2.0, -1.5, 0.5))])
def test_other_polynomials(steps, abc):
    shapes = [(40, 60), (300, 150)]
    g = _gen(4)
    u = [_matrix(*s, g).float() for s in shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    plan = MuonPlan(shapes)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper(steps=steps, coefficients=abc))
    for x, y in zip(u, o):
        _near(y, _exact(x, steps, abc), TOL + UBF / 2)


def test_rows_of_different_sizes():
    shapes = [(64, 200), (200, 64), (150, 160)]
    g = _gen(5)
    u = [_matrix(*s, g, "rows").float() for s in shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    plan = MuonPlan(shapes)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y in zip(u, o):
        _near(y, _exact(x), TOL + UBF / 2)


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("scale", ["one", "spectral", "rms"])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(grad, scale, nesterov):
    shapes = [(5, 3), (0, 4), (64, 32), (130, 40), (40, 131), (256, 300)]
    mask = [1, 1, 0, 1, 0, 1]
    g = _gen(6)
    gr = [_matrix(*s, g).to(DT[grad]) for s in shapes]
    w = [_matrix(*s, g, std=0.05).float() for s in shapes]
    m = [_matrix(*s, g, std=3e-4).float() for s in shapes]
    copy = [torch.zeros(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    wd, md = [x.double() for x in w], [x.double() for x in m]
    plan = MuonPlan(shapes, mask, grad_dtype=grad, copy_dtype="bf16")
    plan.bind(w, gr, m, copy)
    lr = torch.full((1,), 0.02, device=DEV)
    beta, lam = 0.9, 0.1
    hyper = B.make_muon_hyper(momentum=beta, weight_decay=lam, scale=scale,
                              update_scale=0.5, nesterov=nesterov)
    for it in range(2):
        plan.step(hyper, lr)
        for k, (r, c) in enumerate(shapes):
            if r == 0:
                continue
            gd = gr[k].double()
            md[k] = beta * md[k] + (1 - beta) * gd
            u = (1 - beta) * gd + beta * md[k] if nesterov else md[k]
            size = 0.5 * {"one": 1.0, "spectral": math.sqrt(max(1.0, r / c)),
                          "rms": 0.2 * math.sqrt(max(r, c))}[scale]
            eta = float(lr)
            x = _exact(u)
            wd[k] = wd[k] * (1 - eta * lam * mask[k]) - eta * size * x
            # fp32: a few roundings of the terms
            terms = beta * md[k].abs() + gd.abs()
            assert ((m[k].double() - md[k]).abs() <= 8 * U32 * terms).all()
            off = float((w[k].double() - wd[k]).norm())
            assert off <= (it + 1) * (eta * size * TOL * float(x.norm()) +
                                      4 * U32 * float(wd[k].norm())), (k, it)
            assert torch.equal(copy[k], w[k].bfloat16())
            wd[k], md[k] = w[k].double(), m[k].double()
    assert plan.query() == 0


def test_zero_and_nonfinite_gradients():
    """Nothing in, nothing out; an Inf or NaN stays in its own matrix."""
    shapes = [(64, 40), (130, 200), (33, 20), (150, 140)]
    g = _gen(7)
    u = [_matrix(*s, g).float() for s in shapes]
    u[0].zero_()
    o = [torch.full(s, 3.0, device=DEV, dtype=torch.bfloat16) for s in shapes]
    plan = MuonPlan(shapes)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    assert (o[0] == 0).all() and plan.query() == 0
    good = [y.clone() for y in o]
    u[1][3, 5] = float("nan")
    u[2][0, 0] = float("inf")
    plan.direction(B.make_muon_hyper())
    assert plan.query(clear=True) == B.LAMB_STATUS_NONFINITE
    assert torch.isnan(o[1]).any() and torch.isnan(o[2]).any()
    assert torch.equal(o[0], good[0]) and torch.equal(o[3], good[3])
    u[1][3, 5] = 0.0
    u[2][0, 0] = 0.0
    plan.direction(B.make_muon_hyper())
    assert plan.query() == 0
    for x, y in zip(u[1:], o[1:]):
        _near(y, _exact(x), TOL + UBF / 2)


def test_tiny_and_large_gradients():
    shapes = [(48, 40), (140, 200)]
    for std in (1e-12, 1e8):
        g = _gen(8)
        u = [_matrix(*s, g, std=std).float() for s in shapes]
        o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
        plan = MuonPlan(shapes)
        plan.bind_direction(u, o)
        plan.direction(B.make_muon_hyper(eps=0.0))
        for x, y in zip(u, o):
            _near(y, _exact(x, eps=0.0), TOL + UBF / 2)


def test_unaligned_tensors():
    """Matrices one after another in packed buffers."""
    shapes = [(33, 65), (70, 129), (129, 257)]
    g = _gen(9)
    n = sum(r * c for r, c in shapes)
    gbuf = torch.randn(n + 1, generator=g, device=DEV).bfloat16()
    obuf = torch.empty(n + 1, device=DEV, dtype=torch.bfloat16)
    at, u, o = 1, [], []
    for r, c in shapes:
        u.append(gbuf[at:at + r * c].view(r, c))
        o.append(obuf[at:at + r * c].view(r, c))
        at += r * c
    plan = MuonPlan(shapes, grad_dtype="bf16")
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y in zip(u, o):
        _near(y, _exact(x), TOL + UBF / 2)
    # in place
    want = [y.clone() for y in o]
    plan.bind_direction(u, u)
    plan.direction(B.make_muon_hyper())
    assert all(torch.equal(a, b) for a, b in zip(u, want))


def test_step_in_a_graph_on_another_stream():
    shapes = [(64, 96), (200, 136)]
    g = _gen(10)
    gr = [_matrix(*s, g).bfloat16() for s in shapes]
    w = [_matrix(*s, g, std=0.05).float() for s in shapes]
    m = [torch.zeros(s, device=DEV) for s in shapes]
    lr = torch.full((1,), 0.02, device=DEV)
    plan = MuonPlan(shapes, grad_dtype="bf16")
    plan.bind(w, gr, m)
    w0 = [x.clone() for x in w]
    hyper = B.make_muon_hyper()
    plan.step(hyper, lr)
    plan.step(hyper, lr)
    want = [x.clone() for x in w]
    for x, y, z in zip(w, w0, m):
        x.copy_(y)
        z.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        plan.step(hyper, lr)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(w, want))


# enough work beside a test's own matrices for the larger tiles
MANY = [(700, 600)] * 20


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["gauss", "low rank"])
def test_direction_of_many(dtype, kind):
    shapes = MANY + SHAPES + [(1024, 260), (300, 2050)]
    g = _gen(11)
    u = [_matrix(r, c, g, kind).to(DT[dtype]) for r, c in shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    plan = MuonPlan(shapes, grad_dtype=dtype)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y, s in zip(u, o, shapes):
        _near(y, _exact(x), TOL + UBF / 2, s)
    assert plan.query() == 0
    first = [y.clone() for y in o]
    plan.direction(B.make_muon_hyper())
    assert all(torch.equal(a, b) for a, b in zip(first, o))


def test_step_of_many():
    """The step, and an Inf that stays in its own matrix."""
    shapes = MANY + [(64, 32), (130, 40), (257, 129), (300, 1000)]
    g = _gen(12)
    gr = [_matrix(*s, g).bfloat16() for s in shapes]
    w = [_matrix(*s, g, std=0.05).float() for s in shapes]
    m = [_matrix(*s, g, std=3e-4).float() for s in shapes]
    copy = [torch.zeros(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    wd, md = [x.double() for x in w], [x.double() for x in m]
    plan = MuonPlan(shapes, grad_dtype="bf16", copy_dtype="bf16")
    plan.bind(w, gr, m, copy)
    lr = torch.full((1,), 0.02, device=DEV)
    beta, lam, eta = 0.9, 0.1, float(lr)
    plan.step(B.make_muon_hyper(momentum=beta, weight_decay=lam), lr)
    for k, (r, c) in enumerate(shapes):
        gd = gr[k].double()
        md[k] = beta * md[k] + (1 - beta) * gd
        x = _exact((1 - beta) * gd + beta * md[k])
        size = math.sqrt(max(1.0, r / c))
        wd[k] = wd[k] * (1 - eta * lam) - eta * size * x
        terms = beta * md[k].abs() + gd.abs()
        assert ((m[k].double() - md[k]).abs() <= 8 * U32 * terms).all()
        off = float((w[k].double() - wd[k]).norm())
        assert off <= (eta * size * TOL * float(x.norm()) +
                       4 * U32 * float(wd[k].norm())), k
        assert torch.equal(copy[k], w[k].bfloat16())
    assert plan.query() == 0
    good = [x.clone() for x in w]
    gr[3][5, 7] = float("inf")
    for x, y in zip(w, good):
        x.copy_(y)
    plan.step(B.make_muon_hyper(momentum=beta, weight_decay=lam), lr)
    assert plan.query(clear=True) == B.LAMB_STATUS_NONFINITE
    assert torch.isnan(w[3]).any()
    assert all(torch.isfinite(x).all() for k, x in enumerate(w) if k != 3)


def test_refusals():
    shapes = [(8, 8), (8, 4)]
    plan = MuonPlan(shapes, grad_dtype="bf16")
    f = [torch.zeros(s, device=DEV) for s in shapes]
    h = [x.bfloat16() for x in f]
    lr = torch.zeros(1, device=DEV)
    for call in (lambda: plan.step(B.make_muon_hyper(), lr),
                 lambda: plan.direction(B.make_muon_hyper())):
        with pytest.raises(B.LambError) as e:
            call()
        assert e.value.status == B.LAMB_ERR_NOT_BOUND
    for args in ((f, f, f), (h, h, f), (f[:1], h, f), (f, h, f, h),
                 (f, [h[0], h[0]], f), (f, [h[0].cpu(), h[1]], f),
                 (f, [h[0].t().contiguous().t(), h[1].t()], f)):
        with pytest.raises(ValueError):
            plan.bind(*args)
    plan.bind(f, h, f)
    for bad in (dict(momentum=1.0), dict(momentum=-0.1), dict(steps=0),
                dict(steps=65), dict(eps=-1.0), dict(weight_decay=-1.0),
                dict(coefficients=(17.0, 0.0, 0.0)),
                dict(update_scale=float("nan"))):
        with pytest.raises(B.LambError) as e:
            plan.step(B.make_muon_hyper(**bad), lr)
        assert e.value.status == B.LAMB_ERR_INVALID_ARG, bad
