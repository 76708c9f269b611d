"""GPU tests of the root-mean-square norm and its gradient against the formulas in 64
bits.

A sum of n fp32 terms passes at most 64 roundings on its way here (32 columns a
thread, five exchanges between lanes, sixteen warps; the walk over wide rows 82 at
20,999 columns), each of half a step, 2^-24; r takes half of the sum's relative error,
and three more roundings, and its approximation's 2^-22.  `ROUNDS` bounds all of that
in units of 2^-24."""
import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300.norm import NormPlan

pytestmark = pytest.mark.gpu

F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
ROUNDS = 64 * 2.0 ** -24
EPS = 1e-6


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _rows(n, d, dtype, seed, pad=0, shift=0):
    """Rows of different sizes with a few large columns, `pad` more elements from row
    to row, and the first one `shift` elements behind an aligned address."""
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((n, d), generator=gen, device="cuda")
    x *= torch.exp(torch.randn((n, 1), generator=gen, device="cuda"))
    x[:, ::97] *= 20
    buf = torch.full((n * (d + pad) + shift + 8,), float("nan"), device="cuda",
                     dtype=dtype)
    view = buf[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
    view.copy_(x)
    return view


def _weight(d, dtype, seed=5):
    gen = torch.Generator("cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(dtype)


def _formula(h, w):
    h = h.double()
    r = (h.square().mean(1, keepdim=True) + EPS).rsqrt()
    return h * r * (1.0 if w is None else w.double()), r


def _close(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4])


SHAPES = [  # rows, columns, elements between rows, shift: all layouts of a row
    (1, 1, 0, 0), (5, 1, 2, 0), (3, 8, 0, 0), (70, 7, 0, 0), (33, 40, 0, 0),
    (129, 31, 1, 1), (17, 256, 0, 0), (9, 257, 0, 0), (10, 512, 8, 0),
    (6, 520, 0, 3), (1, 1024, 0, 0), (515, 1024, 0, 0), (4, 1000, 24, 0),
    (5, 1023, 0, 0), (3, 1032, 0, 0), (2, 1600, 0, 4), (700, 2048, 0, 0),
    (3, 5000, 0, 0), (2, 8192, 0, 0), (2, 8191, 0, 0), (1, 8200, 0, 0),
    (2, 16384, 0, 0), (1, 16383, 0, 0), (3, 20999, 0, 0)]


@pytest.mark.parametrize("n,d,pad,shift", SHAPES)
@pytest.mark.parametrize("x_type,h_type", [(BF16, BF16), (BF16, F32),
                                           (F32, BF16), (F32, F32)])
def test_norm(gpu, n, d, pad, shift, x_type, h_type):
    x = _rows(n, d, x_type, 1, pad, shift)
    res = _rows(n, d, h_type, 2, pad, shift)
    sum_ = (x.float() + res.float()).to(h_type)
    with NormPlanOf(d, n) as plan:
        for w in (None, _weight(d, BF16), _weight(d, F32)):
            for out_type in (F32, BF16):
                total = _rows(n, d, h_type, 3, pad, shift)
                out = _rows(n, d, out_type, 4, pad, shift)
                got = plan.norm(x, w, residual=res, total=total, out=out)
                assert got[0] is out and got[1] is total
                assert torch.equal(total, sum_)
                want, _ = _formula(sum_, w)
                rounding = _half(out_type) if out_type == BF16 else 0
                _close(out, want, (ROUNDS + rounding) * want.abs())
                # and without a residual, allocated
                y = plan.norm(x, w, dtype=out_type)
                want, _ = _formula(x, w)
                _close(y, want, (ROUNDS + rounding) * want.abs())


class NormPlanOf:
    def __init__(self, d, n):
        self.plan = NormPlan(d, n, eps=EPS)

    def __enter__(self):
        return self.plan

    def __exit__(self, *_):
        torch.cuda.synchronize()
        self.plan.destroy()


@pytest.mark.parametrize("n,d,pad,shift", SHAPES)
@pytest.mark.parametrize("block", [0, 32, 128])
def test_norm_8bit(gpu, n, d, pad, shift, block):
    for x_type, h_type in ((BF16, F32), (F32, BF16)):
        x = _rows(n, d, x_type, 1, pad, shift)
        res = _rows(n, d, h_type, 2, pad, shift)
        w = _weight(d, BF16)
        with NormPlanOf(d, n) as plan:
            out, scales, total = plan.norm_8bit(x, w, residual=res, block=block)
            wide = torch.zeros((n, d + pad), device="cuda", dtype=F8)
            kept = wide[:, :d]
            assert plan.norm_8bit(x, w, block=block, out=kept)[0] is kept
        assert torch.equal(total, (x.float() + res.float()).to(h_type))
        assert not wide[:, d:].view(torch.uint8).any()
        want, _ = _formula(total, w)
        width = block or d
        blocks = -(-d // width)
        padded = torch.nn.functional.pad(want.abs(), (0, blocks * width - d))
        s = padded.view(n, blocks, width).amax(2).clamp(min=2.0 ** -100) / 448
        _close(scales, s, (ROUNDS + 2.0 ** -24) * s)
        s = scales.double().repeat_interleave(width, 1)[:, :d]
        # half a step of 8 bits, of its normal numbers or of its smallest ones
        _close(out.double() * s, want, (2.0 ** -4 + 2 * ROUNDS) * want.abs() +
               2.0 ** -10 * s)


def test_norm_in_place_and_rows_left_alone(gpu):
    n, d = 6, 1024
    x, res = _rows(n, d, BF16, 1), _rows(n, d, BF16, 2)
    sum_ = (x.float() + res.float()).bfloat16()
    with NormPlanOf(d, 8) as plan:
        want = plan.norm(x, residual=res)[0].clone()
        big = torch.full((8, d), 7.0, device="cuda", dtype=BF16)
        big[:n] = x
        out, total = plan.norm(big[:n], residual=res, total=res, out=big[:n])
        assert torch.equal(out, want) and torch.equal(total, sum_)
        assert (big[n:] == 7).all()
        assert plan.norm(x[:0]).shape == (0, d)


def test_norm_of_zeros_large_values_and_nan(gpu):
    d = 1024
    x = torch.zeros((5, d), device="cuda")
    x[1] = 3e20                       # squares overflow: r = 0
    x[2, 7] = float("nan")
    x[3] = 1e-25                      # squares vanish beside eps
    x[4, 3], x[4, 40] = 1e4, 1e-4
    with NormPlanOf(d, 5) as plan:
        y = plan.norm(x)
        q, s = plan.norm_8bit(x, block=32)
    assert (y[0] == 0).all() and (y[1] == 0).all()
    assert y[2].isnan().all()
    assert torch.allclose(y[3], x[3] * 1e3, rtol=1e-5)
    least = torch.tensor(2.0 ** -100 / 448, dtype=F32)
    assert (s[0].cpu() == least).all() and (q[0].float() == 0).all()
    assert s[2].isnan().all() and q[2].float().isnan().all()
    assert float(s[4, 0]) > 1e4 * float(s[4, 1]) > 0
    assert float(q[4, 3].float()) == 448 and float(q[4, 40].float()) == 448


def _grads(h, dy, w, dh_in):
    """dh, dw from the formula, and the sizes that their roundings go by."""
    _, r = _formula(h, None)
    h, dy = h.double(), dy.double()
    g = dy * (1.0 if w is None else w.double())
    c = (g * h).mean(1, keepdim=True) * r * r
    size = r * (g.abs() + (g * h).abs().mean(1, keepdim=True) * r * r * h.abs())
    dh = r * (g - c * h)
    if dh_in is not None:
        dh = dh + dh_in.double()
        size = size + dh_in.double().abs()
    return dh, size, (dy * h * r).sum(0), (dy * h * r).abs().sum(0)


@pytest.mark.parametrize("n,d,pad,shift", SHAPES)
@pytest.mark.parametrize("g_type,h_type", [(BF16, BF16), (BF16, F32),
                                           (F32, BF16), (F32, F32)])
def test_norm_grad(gpu, n, d, pad, shift, g_type, h_type):
    """A weight's gradient passes up to 200 additions: rows of a thread, up to 128
    groups of a CTA, parts of 32 warps, warps."""
    h = _rows(n, d, h_type, 1, pad, shift)
    dy = _rows(n, d, g_type, 2, pad, shift)
    dh_in = _rows(n, d, h_type, 3, pad, shift)
    with NormPlanOf(d, n) as plan:
        for w, w_type, arrives, add in ((None, F32, None, False),
                                        (_weight(d, BF16), BF16, dh_in, True),
                                        (_weight(d, F32), F32, dh_in, True),
                                        (_weight(d, BF16), BF16, None, False)):
            dw = _weight(d, w_type, 9)
            dw0 = dw.double() if add else torch.zeros(d, device="cuda").double()
            dh = _rows(n, d, h_type, 4, pad, shift)
            assert plan.norm_grad(dy, h, w, dh, dw, grad_in=arrives,
                                  accumulate=add) is dh
            want, size, ww, wsize = _grads(h, dy, w, arrives)
            rounding = _half(h_type) if h_type == BF16 else 0
            _close(dh, want, 2 * ROUNDS * size + rounding * want.abs())
            ww, wsize = ww + dw0, wsize + dw0.abs()
            rounding = _half(w_type) if w_type == BF16 else 0
            _close(dw, ww, 256 * 2.0 ** -24 * wsize + rounding * ww.abs())
        # no weight's gradient, and results over an input
        for over in ("grad_in", "grad_out", "total"):
            if over == "grad_out" and g_type != h_type:
                continue
            ts = dict(grad_in=dh_in.clone(), grad_out=dy.clone(),
                      total=h.clone())
            want, size, _, _ = _grads(h, dy, None, dh_in)
            plan.norm_grad(ts["grad_out"], ts["total"], None, ts[over],
                           grad_in=ts["grad_in"])
            rounding = _half(h_type) if h_type == BF16 else 0
            _close(ts[over], want, 2 * ROUNDS * size + rounding * want.abs())


def test_norm_grad_many_rows_and_differences(gpu):
    n, d = 20000, 256
    h, dy = _rows(n, d, F32, 1), _rows(n, d, F32, 2)
    w = _weight(d, F32)
    dh, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    with NormPlanOf(d, n) as plan:
        plan.norm_grad(dy, h, w, dh, dw)
    _, _, ww, wsize = _grads(h, dy, w, None)
    # (a thread's rows: 20,000 in 456 CTAs of four, 11)
    _close(dw, ww, 256 * 2.0 ** -24 * wsize)
    # along a direction, by differences of the formula: central, error of the order
    # of step^2, and of 2^-52 / step
    gen = torch.Generator("cuda").manual_seed(3)
    for k in range(3):
        u = torch.randn(h.shape, generator=gen, device="cuda").double() * h.abs()
        v = torch.randn(d, generator=gen, device="cuda").double()
        step = 1e-5
        ends = [(_formula(h.double() + s * step * u, w.double() + s * step * v)[0]
                 * dy.double()).sum() for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        along = (dh.double() * u).sum() + (dw.double() * v).sum()
        size = (dh.double() * u).abs().sum() + (dw.double() * v).abs().sum()
        assert abs(float(slope - along)) < 1e-6 * float(size)


def test_norm_grad_without_rows(gpu):
    d = 100
    none = torch.empty((0, d), device="cuda")
    dw = torch.ones(d, device="cuda")
    with NormPlanOf(d, 4) as plan:
        plan.norm_grad(none, none, None, none, dw, accumulate=True)
        assert (dw == 1).all()
        plan.norm_grad(none, none, None, none, dw)
        assert (dw == 0).all()


def test_norm_repeats_its_bits_in_a_graph_on_another_stream(gpu):
    n, d = 3000, 768
    x, res = _rows(n, d, BF16, 1), _rows(n, d, F32, 2)
    dy, w = _rows(n, d, BF16, 3), _weight(d, BF16)
    plan = NormPlan(d, n)
    out, total = torch.empty_like(x), torch.empty_like(res)
    dh, dw = torch.empty_like(res), torch.empty(d, device="cuda")

    def run():
        plan.norm(x, w, residual=res, total=total, out=out)
        plan.norm_grad(dy, total, w, dh, dw, grad_in=res)
    run()
    torch.cuda.synchronize()
    first = [t.clone() for t in (out, total, dh, dw)]
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run()
    for _ in range(3):
        for t in (out, total, dh, dw):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b)
                   for a, b in zip(first, (out, total, dh, dw)))
    with torch.cuda.stream(stream):
        y, _ = plan.norm(x, w, residual=res)
    z, _ = plan.norm(x, w, residual=res, stream=stream.cuda_stream)
    stream.synchronize()
    assert torch.equal(y, plan.norm(x, w, residual=res, dtype=BF16)[0])
    assert torch.equal(z, y)


def test_norm_rows_beyond_32_bits(gpu):
    """Offsets in elements that pass 2^31: a row stride of 2^30."""
    d, stride = 64, 2 ** 30
    buf = torch.zeros(2 * stride + d, device="cuda", dtype=BF16)
    x = buf.as_strided((3, d), (stride, 1))
    x.copy_(_rows(3, d, BF16, 1))
    plan = NormPlan(d, 3, eps=EPS)
    want = plan.norm(x.contiguous())
    dense, far = x.clone(), torch.empty((3, d), device="cuda", dtype=BF16)
    assert torch.equal(plan.norm(x), want)
    plan.norm_grad(dense, dense, None, far)
    plan.norm_grad(dense, x, None, x)
    assert torch.equal(x, far)


def test_norm_calls_refuse(gpu):
    plan = NormPlan(16, 4)
    x = torch.zeros((4, 16), device="cuda", dtype=BF16)
    for call in (
            lambda: plan.norm(x[:, :8]), lambda: plan.norm(x.cpu()),
            lambda: plan.norm(x.half()), lambda: plan.norm(x[0]),
            lambda: plan.norm(x, torch.ones(15, device="cuda")),
            lambda: plan.norm(x, torch.ones(16, device="cuda").double()),
            lambda: plan.norm(x, total=x), lambda: plan.norm(x.t()),
            lambda: plan.norm(x, residual=x, total=x.float()),
            lambda: plan.norm(x, out=torch.zeros((4, 16), device="cuda",
                                                 dtype=F8)),
            lambda: plan.norm_8bit(x, block=64),
            lambda: plan.norm_8bit(x, out=x),
            lambda: plan.norm_8bit(x, scales=torch.zeros(4, device="cuda")),
            lambda: plan.norm_grad(x, x, None, x.float()),
            lambda: plan.norm_grad(x[:3], x, None, x),
            lambda: plan.norm_grad(x, x, None, x, x[0].double())):
        with pytest.raises(ValueError):
            call()
    many = torch.zeros((5, 16), device="cuda", dtype=BF16)
    for call in (lambda: plan.norm(many),
                 lambda: plan.norm_grad(many, many, None, many)):
        with pytest.raises(B.LambError) as e:
            call()
        assert e.value.status == B.LAMB_ERR_INVALID_ARG
    torch.cuda.synchronize()


@pytest.mark.parametrize("widths", [(8192, 4096, 2048, 1024, 520),
                                    (520, 1024, 2048, 4096, 8192)])
@pytest.mark.parametrize("g_type,h_type", [(BF16, BF16), (BF16, F32),
                                           (F32, BF16), (F32, F32)])
def test_norm_grad_of_plans_that_live_together(gpu, widths, g_type, h_type):
    """Plans of other widths that are made later leave a plan's launches as they are."""
    n = 5
    plans = [NormPlan(d, n, eps=EPS) for d in widths]
    for d, plan in zip(widths, plans):
        h, dy = _rows(n, d, h_type, 1), _rows(n, d, g_type, 2)
        w, dw = _weight(d, BF16), torch.empty(d, device="cuda")
        dh = torch.empty_like(h)
        plan.norm_grad(dy, h, w, dh, dw)
        want, size, ww, wsize = _grads(h, dy, w, None)
        rounding = _half(h_type) if h_type == BF16 else 0
        _close(dh, want, 2 * ROUNDS * size + rounding * want.abs())
        _close(dw, ww, 256 * 2.0 ** -24 * wsize)
    torch.cuda.synchronize()
    for plan in plans:
        plan.destroy()


@pytest.mark.parametrize("n,d,shift", [(1300, 8200, 0), (700, 20999, 0),
                                       (1000, 5001, 0), (640, 2048, 1),
                                       (9000, 257, 0), (30000, 31, 3)])
@pytest.mark.parametrize("g_type,h_type", [(BF16, BF16), (F32, F32)])
def test_norm_grad_of_more_rows_than_ctas(gpu, n, d, shift, g_type, h_type):
    """Walked rows and rows taken column by column, several of them for each CTA: as
    many additions as in test_norm_grad."""
    h = _rows(n, d, h_type, 1, shift=shift)
    dy = _rows(n, d, g_type, 2, shift=shift)
    dh_in = _rows(n, d, h_type, 3, shift=shift)
    w, dw = _weight(d, BF16), _weight(d, F32, 9)
    dw0, dh = dw.double(), torch.empty_like(h)
    with NormPlanOf(d, n) as plan:
        plan.norm_grad(dy, h, w, dh, dw, grad_in=dh_in, accumulate=True)
        want, size, ww, wsize = _grads(h, dy, w, dh_in)
        rounding = _half(h_type) if h_type == BF16 else 0
        _close(dh, want, 2 * ROUNDS * size + rounding * want.abs())
        _close(dw, ww + dw0, 256 * 2.0 ** -24 * (wsize + dw0.abs()))


LAYOUTS = [(1024, 0), (1024, 1), (2048, 0), (2048, 1), (64, 0), (64, 1), (8200, 0)]


@pytest.mark.parametrize("d,shift", LAYOUTS)
def test_norm_grad_of_tiny_rows(gpu, d, shift):
    """grad_out h is below the normal numbers of 32 bits, grad_out h r is not."""
    n, eps = 6, 1e-20
    h = _rows(n, d, F32, 1, shift=shift)
    dy = _rows(n, d, F32, 2, shift=shift)
    h *= 1e-15
    dy *= 1e-28
    plan = NormPlan(d, n, eps=eps)
    dh, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    plan.norm_grad(dy, h, None, dh, dw)
    x, g = h.double(), dy.double()
    r = (x.square().mean(1, keepdim=True) + eps).rsqrt()
    terms = g * x * r
    _close(dw, terms.sum(0), 256 * 2.0 ** -24 * terms.abs().sum(0))
    # (each of the row's products is off by half of 2^-149, too)
    c = (g * x).mean(1, keepdim=True) * r * r
    size = r * (g.abs() + (g * x).abs().mean(1, keepdim=True) * r * r * x.abs())
    _close(dh, r * (g - c * x), 2 * ROUNDS * size + 2.0 ** -148 * r ** 3 * x.abs())


@pytest.mark.parametrize("d,shift", LAYOUTS)
def test_norm_grad_of_rows_whose_squares_overflow(gpu, d, shift):
    """Such rows have r = 0: nothing goes through them, whatever grad_out h is."""
    n = 4
    h, dy = _rows(n, d, F32, 1, shift=shift), _rows(n, d, F32, 2, shift=shift)
    dh_in, w = _rows(n, d, F32, 3, shift=shift), _weight(d, F32)
    h[1] = 3e20 * (1 + torch.rand(d, device="cuda"))
    dy[1] = 1e19 * (1 + torch.rand(d, device="cuda"))
    h[2] = -2e19
    plan = NormPlan(d, n, eps=EPS)
    dh, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    y = plan.norm(h, w)
    plan.norm_grad(dy, h, w, dh, dw, grad_in=dh_in)
    assert (y[1:3] == 0).all() and torch.equal(dh[1:3], dh_in[1:3])
    rows = [0, 3]
    want, size, ww, wsize = _grads(h[rows], dy[rows], w, dh_in[rows])
    _close(dh[rows], want, 2 * ROUNDS * size)
    _close(dw, ww, 256 * 2.0 ** -24 * wsize)
