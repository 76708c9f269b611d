"""GPU tests of the global gradient norm and clipping against the formulas in 64
bits.  Of 64 or so squares (256 of an unaligned tensor's chunk: 16,384 elements, 256
threads, 64 each) fp32 sums pass 65 roundings at most, of which the root takes half;
beyond that sums are 64-bit: 34 * 2^-24, and half a step of the result."""
import math

import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300.clip import ClipPlan

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NORM = 35 * 2.0 ** -24


def _grads(sizes, dtype, size=1.0, seed=1, shift=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        x = torch.randn(n, generator=gen, device="cuda").double()
        x *= size * math.exp(k % 5 - 2)
        buf = torch.zeros(n + 16, device="cuda", dtype=TYPES[dtype])
        buf[shift:shift + n] = x
        out.append(buf[shift:shift + n])
    return out


def _norm(grads, scale=1.0):
    return abs(scale) * math.sqrt(math.fsum(
        float(g.double().square().sum()) for g in grads))


def _check(grads, before, norm, factor, max_norm, scale=1.0):
    want = _norm(before, scale)
    assert abs(float(norm) - want) <= NORM * want
    f = scale * min(1.0, max_norm / want)
    assert abs(float(factor) - f) <= NORM * abs(f)
    f = float(factor)
    for x, g in zip(grads, before):
        exact = g.double() * f
        half = torch.finfo(x.dtype).eps / 2
        # (below the smallest normal number steps do not shrink any more)
        err = (x.double() - exact).abs()
        assert (err <= half * exact.abs() + 2.0 ** -149).all()


SIZES = [[1], [0, 3, 0], [8, 7, 9, 1], [16384], [16385, 16383, 5],
         [64 * 32, 32, 320, 10], [100000, 0, 1, 70001, 33] * 3, [3000001]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("o_type", [None, "f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_clip(gpu, sizes, g_type, o_type, shift):
    before = _grads(sizes, g_type, shift=shift)
    whole = _norm(before)
    scale = torch.full((), -0.5, device="cuda")
    for s, max_norm in ((None, 0.25 * whole), (scale, 0.125 * whole),
                        (None, 2 * whole), (scale, 2 * whole), (scale, math.inf),
                        (None, 0.0)):
        grads = _grads(sizes, g_type, shift=shift)
        plan = ClipPlan(sizes, grad_dtype=g_type, out_dtype=o_type)
        out = grads
        if o_type:
            out = _grads(sizes, o_type, seed=2, shift=0)
        plan.bind(grads, out if o_type else None)
        factor = torch.zeros(1, device="cuda")
        norm = plan.clip(max_norm, scale=s, factor=factor)
        _check(out, before, norm, factor, max_norm, -0.5 if s is not None else 1.)
        if o_type or (s is None and max_norm > whole):
            assert all(torch.equal(a, b) for a, b in zip(grads, before))
        assert plan.query() == 0


def test_clip_out_may_be_the_gradients(gpu):
    before = _grads([5000, 3], "f32")
    grads = [g.clone() for g in before]
    plan = ClipPlan([5000, 3], out_dtype="f32")
    plan.bind(grads, grads)
    factor = torch.zeros(1, device="cuda")
    _check(grads, before, plan.clip(0.5, factor=factor), factor, 0.5)


@pytest.mark.parametrize("size", [1e-40, 1e-30, 1e-19, 1e19, 1e30, 1e36])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_of_tiny_and_huge_gradients(gpu, size, shift):
    sizes = [40000, 17, 300]
    grads = _grads(sizes, "f32", size, shift=shift)
    before = [g.clone() for g in grads]
    plan = ClipPlan(sizes)
    plan.bind(grads)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    whole = _norm(before)
    plan.clip(whole / 3, norm=norm, factor=factor)
    # (a norm of subnormal size has steps of 2^-149)
    assert abs(float(norm) - whole) <= NORM * whole + 2.0 ** -149
    assert abs(float(factor) * 3 - 1) <= 2 * NORM
    assert plan.query() == 0


def test_one_large_gradient_among_zeros(gpu):
    sizes = [100000]
    grads = [torch.zeros(100000, device="cuda")]
    plan = ClipPlan(sizes)
    plan.bind(grads)
    assert float(plan.clip(1.0)) == 0 and plan.query() == 0
    grads[0][77777] = -3e25
    grads[0][5] = 1e-30
    assert float(plan.clip(2.0)) == float(torch.tensor(3e25))
    assert abs(float(grads[0][77777]) + 2) < 1e-6


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_gradients_that_are_not_finite_are_not_clipped(gpu, bad):
    sizes = [70000, 9]
    grads = _grads(sizes, "bf16")
    grads[1][4] = bad
    before = [g.clone() for g in grads]
    plan = ClipPlan(sizes, grad_dtype="bf16")
    plan.bind(grads)
    factor = torch.zeros((), device="cuda")
    norm = plan.clip(1e-3, factor=factor)
    assert not math.isfinite(float(norm)) and float(factor) == 1
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16))
               for a, b in zip(grads, before))
    assert plan.query(clear=True) == B.LAMB_STATUS_GRAD_NONFINITE
    grads[1][4] = 0
    assert math.isfinite(float(plan.clip(1e9)))
    assert plan.query() == 0


def test_clip_repeats_its_bits_in_a_graph_and_after_another_binding(gpu):
    sizes = [123457, 64, 9999, 1]
    first = _grads(sizes, "f32")
    out = _grads(sizes, "bf16", seed=2)
    plan = ClipPlan(sizes, out_dtype="bf16")
    plan.bind(first, out)
    norm = plan.clip(0.7)
    kept = [t.clone() for t in out] + [norm.clone()]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        plan.clip(0.7, norm=norm)
    for _ in range(3):
        for t in out:
            t.zero_()
        norm.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, out + [norm]))
    # the graph takes what the plan is bound to when it runs
    second = [2 * g for g in first]
    plan.bind(second, out)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(norm) / float(kept[-1]) - 2) < 1e-6


def test_clip_calls_refuse(gpu):
    plan = ClipPlan([4, 2])
    with pytest.raises(B.LambError) as e:
        plan.clip(1.0)
    assert e.value.status == B.LAMB_ERR_NOT_BOUND
    good = [torch.ones(4, device="cuda"), torch.ones(2, device="cuda")]
    for call in (
            lambda: plan.bind(good[:1]), lambda: plan.bind(good, good),
            lambda: plan.bind([good[0], good[0]]),
            lambda: plan.bind([good[0].bfloat16(), good[1]]),
            lambda: plan.bind([g.cpu() for g in good]),
            lambda: plan.bind([torch.ones(8, device="cuda")[::2], good[1]]),
            lambda: ClipPlan([4], out_dtype="bf16").bind(good[:1])):
        with pytest.raises(ValueError):
            call()
    plan.bind(good)
    for call in (lambda: plan.clip(1.0, scale=torch.ones(2, device="cuda")),
                 lambda: plan.clip(1.0, norm=torch.ones(1)),
                 lambda: plan.clip(1.0, factor=torch.ones(1, device="cuda").half())):
        with pytest.raises(ValueError):
            call()
    for bad in (-1.0, math.nan):
        with pytest.raises(B.LambError) as e:
            plan.clip(bad)
        assert e.value.status == B.LAMB_ERR_INVALID_ARG
    assert abs(float(plan.clip(1.0)) - math.sqrt(6)) < 1e-6


def test_clip_refuses_tensors_that_overlap(gpu):
    """A gradient given twice would be multiplied twice."""
    whole = torch.ones(100, device="cuda")
    a, b, c = whole[:40], whole[39:79], whole[40:80]
    plan = ClipPlan([40, 40])
    for bad in ([a, a], [a, b], [b, c]):
        with pytest.raises(B.LambError) as e:
            plan.bind(bad)
        assert e.value.status == B.LAMB_ERR_INVALID_ARG
    plan.bind([a, c])
    assert abs(float(plan.clip(math.inf)) - math.sqrt(80)) < 1e-5
    other = torch.ones(80, device="cuda")
    plan = ClipPlan([40, 40], out_dtype="f32")
    for out in ([other[:40], other[39:79]], [c, a], [a, a], [c, other[:40]]):
        with pytest.raises(B.LambError):
            plan.bind([a, c], out)
    # read twice, written apart; and each into itself
    plan.bind([a, a], [other[:40], other[40:]])
    assert abs(float(plan.clip(math.inf)) - math.sqrt(80)) < 1e-5
    plan.bind([a, c], [a, c])
    half = ClipPlan([40], out_dtype="bf16")
    with pytest.raises(B.LambError):
        half.bind([a], [a.view(torch.bfloat16)[:40]])


@pytest.mark.parametrize("g_type,o_type", [("f32", None), ("f32", "bf16"),
                                           ("bf16", None), ("bf16", "f32")])
@pytest.mark.parametrize("shift", [4, 8])
def test_clip_tensors_on_16_and_32_bytes(gpu, g_type, o_type, shift):
    """fp32 tensors that start on 16 bytes but not on 32, and ones that do."""
    sizes = [20000, 16384, 31, 8]
    before = _grads(sizes, g_type, shift=shift)
    grads = [g.clone() for g in before] if o_type else before
    before = [g.clone() for g in before]
    out = _grads(sizes, o_type, shift=shift, seed=3) if o_type else None
    plan = ClipPlan(sizes, grad_dtype=g_type, out_dtype=o_type)
    plan.bind(grads, out)
    factor = torch.zeros(1, device="cuda")
    norm = plan.clip(0.5, factor=factor)
    _check(out or grads, before, norm, factor, 0.5)


@pytest.mark.parametrize("sizes", [[16384 * 1003 + 77], [16385, 3, 40000] * 350])
@pytest.mark.parametrize("g_type,o_type", [("f32", None), ("bf16", "f32")])
@pytest.mark.parametrize("shift", [0, 1])
def test_clip_of_more_chunks_than_ctas(gpu, sizes, g_type, o_type, shift):
    """A thousand pieces of 16,384 elements and more: several for each CTA."""
    grads = _grads(sizes, g_type, shift=shift)
    before = [g.clone() for g in grads]
    plan = ClipPlan(sizes, grad_dtype=g_type, out_dtype=o_type)
    out = _grads(sizes, o_type, seed=2, shift=shift) if o_type else grads
    plan.bind(grads, out if o_type else None)
    factor = torch.zeros(1, device="cuda")
    norm = plan.clip(0.5, factor=factor)
    _check(out, before, norm, factor, 0.5)
    assert plan.query() == 0


@pytest.mark.parametrize("g_type,o_type", [("f32", "f32"), ("f32", "bf16"),
                                           ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("g_shift,o_shift", [(4, 0), (0, 4), (4, 4), (4, 8), (8, 0)])
def test_clip_where_one_of_both_is_off_its_boundary(gpu, g_type, o_type, g_shift,
                                                    o_shift):
    """A gradient and its result that start at different places: eight elements of
    either may lie across a boundary while the other's do not."""
    sizes = [20000, 16384, 31, 8]
    grads = _grads(sizes, g_type, shift=g_shift)
    before = [g.clone() for g in grads]
    out = _grads(sizes, o_type, shift=o_shift, seed=3)
    for ts, t, shift in ((grads, g_type, g_shift), (out, o_type, o_shift)):
        wide = 8 * TYPES[t].itemsize
        assert all((x.data_ptr() % wide == 0) == (shift % 8 == 0) for x in ts)
    plan = ClipPlan(sizes, grad_dtype=g_type, out_dtype=o_type)
    plan.bind(grads, out)
    factor = torch.zeros(1, device="cuda")
    norm = plan.clip(0.5, factor=factor)
    _check(out, before, norm, factor, 0.5)


@pytest.mark.parametrize("o_type", [None, "f32", "bf16"])
@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-30])
def test_clip_by_a_factor_below_the_normal_numbers(gpu, o_type, g_type, shift,
                                                   max_norm):
    """The factor is 2^-131 to 2^-231.  A result passes the norm's error and the
    roundings of the factor's two parts, of a product and of the result's type."""
    sizes = [100000, 31, 16384]
    grads = _grads(sizes, g_type, 2e37, shift=shift)
    before = [g.clone() for g in grads]
    plan = ClipPlan(sizes, grad_dtype=g_type, out_dtype=o_type)
    out = _grads(sizes, o_type, seed=2, shift=shift) if o_type else grads
    plan.bind(grads, out if o_type else None)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    plan.clip(max_norm, norm=norm, factor=factor)
    f = max_norm / _norm(before)
    assert 0 < f < 2.0 ** -129
    assert abs(float(factor) - f) <= 2.0 ** -149
    for x, g in zip(out, before):
        exact = g.double() * f
        half = torch.finfo(x.dtype).eps / 2
        err = (x.double() - exact).abs()
        least = 2.0 ** -149 if x.dtype == torch.float32 else 2.0 ** -133
        assert (err <= (NORM + 3 * 2.0 ** -24 + half) * exact.abs() + least).all()
    assert plan.query() == 0
