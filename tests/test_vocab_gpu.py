"""GPU tests of the word table's lookup, its gradient and the vocabulary head
against their formulas in 64 bits.

Tolerances come from the formats: a sum of n terms in fp32 is within (n + 2)
2^-24 of the sum of the terms' sizes (products: 2^-23 a term, the tensor cores
truncate), a result in bf16 within 2^-8 of itself.  The head's bounds follow its
steps: logits, softmax, the logits' gradient in bf16, two products.
"""
import math

import numpy as np
import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300.vocab import VocabPlan

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, UBF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, g, std=1.0, dtype=torch.float32, pad=0, shift=0):
    """Rows of `shape[1]` inside rows of shape[1] + pad, `shift` elements on."""
    r, c = shape
    buf = torch.randn(r * (c + pad) + shift, generator=g, device=DEV)
    x = (buf * std).to(dtype)[shift:].view(r, c + pad)
    return x[:, :c]


def _ids(n, vocab, g, skew, absent=0.1):
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    ids = (u ** skew * vocab).long().clamp(max=vocab - 1)
    gone = torch.rand(n, generator=g, device=DEV) < absent
    return torch.where(gone, -1, ids)


def _close(got, want, bound):
    got, bound = got.double(), bound + 1e-300
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (
        f"{int(bad.sum())} of {bad.numel()} outside the bound, worst "
        f"{float(((got - want).abs() / bound).nan_to_num(9e9).max()):.3g} x")


@pytest.fixture(scope="module", autouse=True)
def _lib(gpu):
    B.load()


# ---------------------------------------------------------------------------
# lookup
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width,pad,shift", [
    (1, 1, 1, 0, 0), (7, 50, 64, 0, 0), (33, 1000, 129, 3, 1),
    (513, 30522, 768, 8, 0), (100, 77, 100, 0, 2)])
def test_lookup(table, out, n, vocab, width, pad, shift):
    g = _gen(n)
    tab = _randn((vocab, width), g, 0.02, DT[table], pad, shift)
    ids = _ids(n, vocab, g, 2.0)
    dst = _randn((n, width), g, 1.0, DT[out], pad, shift)
    plan = VocabPlan(vocab, width, n)
    scale = math.sqrt(width)
    got = plan.embed(tab, ids, scale=scale, out=dst)
    want = torch.where((ids >= 0)[:, None],
                       tab[ids.clamp(min=0)].double() * scale, 0.0)
    _close(got, want, want.abs() * (4 * U32 + (UBF if out == "bf16" else 0)))
    assert plan.query() == 0
    if out == table and shift == 0:
        new = plan.embed(tab, ids, scale=scale)
        assert new.dtype == DT[table] and torch.equal(new, got)
    plan.destroy()


def test_lookup_of_nothing_and_of_bad_ids():
    plan = VocabPlan(10, 16, 8)
    tab = torch.ones(10, 16, device=DEV)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    assert plan.embed(tab, none).shape == (0, 16)
    ids = torch.tensor([3, 10, -1, 2 ** 40, -2 ** 40, 9], device=DEV)
    got = plan.embed(tab, ids)
    assert got.sum(1).tolist() == [16.0, 0.0, 0.0, 0.0, 0.0, 16.0]
    assert plan.query(clear=True) == B.LAMB_STATUS_BAD_INDEX
    assert plan.query() == 0


# ---------------------------------------------------------------------------
# the lookup's gradient
# ---------------------------------------------------------------------------
def _grad_case(n, vocab, width, skew, grad, table, add, pad=0, shift=0,
               ids=None, seed=0):
    g = _gen(seed + n)
    if ids is None:
        ids = _ids(n, vocab, g, skew)
    dy = _randn((n, width), g, 1.0, DT[grad], pad, shift)
    dst = _randn((vocab, width), g, 1.0, DT[table], pad, shift)
    before = dst.double()
    scale = 0.75
    rows = torch.where((ids >= 0)[:, None], dy.double() * scale, 0.0)
    at = ids.clamp(min=0)
    want = torch.zeros(vocab, width, device=DEV, dtype=torch.float64)
    size = want.clone().index_add_(0, at, rows.abs())
    want.index_add_(0, at, rows)
    count = torch.zeros(vocab, device=DEV, dtype=torch.float64).index_add_(
        0, at, (ids >= 0).double())
    if add:
        want += before
        size += before.abs()
    bound = (count[:, None] + 3) * U32 * size
    if table == "bf16":
        bound = bound + UBF * want.abs()
    plan = VocabPlan(vocab, width, max(n, 1))
    got = plan.embed_grad(dy, ids, dst, scale=scale, accumulate=add)
    _close(got, want, bound)
    if add:      # rows without a token keep their bits
        still = count == 0
        assert torch.equal(got[still].double(), before[still])
    assert plan.query() == 0
    plan.destroy()
    return got


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,vocab,width,skew,pad,shift", [
    (1, 30522, 64, 1, 0, 0), (129, 3, 33, 1, 2, 1), (4095, 999, 100, 6, 4, 0),
    (4096, 256, 64, 1, 0, 0), (9001, 70000, 72, 8, 0, 1)])
def test_lookup_gradient(grad, table, add, n, vocab, width, skew, pad, shift):
    _grad_case(n, vocab, width, skew, grad, table, add, pad, shift)


@pytest.mark.parametrize("n", [127, 128, 129, 256, 257, 4097, 20000])
@pytest.mark.parametrize("where", ["one word", "absent", "runs"])
def test_lookup_gradient_of_long_rows(n, where):
    """One word for all tokens, no word at all, and words with runs of 100 to
    400 tokens that start anywhere in a chunk."""
    if where == "one word":
        ids = torch.full((n,), 4, device=DEV)
    elif where == "absent":
        ids = torch.full((n,), -1, device=DEV)
    else:
        rng = np.random.default_rng(n)
        words = np.repeat(np.arange(400), rng.integers(100, 400, 400))[:n]
        ids = torch.from_numpy(rng.permutation(words)).to(DEV)
    _grad_case(n, 400, 36, 1, "bf16", "f32", False, ids=ids)


def test_lookup_gradient_repeats_its_bits():
    args = (30000, 5000, 96, 6, "f32", "f32", False)
    assert torch.equal(_grad_case(*args), _grad_case(*args))


def test_lookup_gradient_of_nothing():
    plan = VocabPlan(10, 16, 8)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    dy = torch.zeros(0, 16, device=DEV)
    g = torch.ones(10, 16, device=DEV)
    plan.embed_grad(dy, none, g, accumulate=True)
    assert g.sum() == 160
    plan.embed_grad(dy, none, g)
    assert g.abs().sum() == 0


def test_lookup_gradient_against_differences():
    """d/dE of sum(out * r), for a few entries, by differences of the lookup."""
    g = _gen(3)
    plan = VocabPlan(12, 8, 20)
    tab = _randn((12, 8), g)
    ids = _ids(20, 12, g, 1.0)
    r = _randn((20, 8), g)
    grad = plan.embed_grad(r, ids, torch.empty_like(tab), scale=0.5)
    for v, d in ((0, 0), (3, 7), (11, 2), (5, 5)):
        f = []
        for h in (0.5, -0.5):
            t = tab.clone()
            t[v, d] += h
            f.append((plan.embed(t, ids, scale=0.5).double() * r).sum())
        assert abs(float(f[0] - f[1]) - float(grad[v, d])) < 1e-4


# ---------------------------------------------------------------------------
# the head
# ---------------------------------------------------------------------------
def _head_inputs(n, vocab, width, g, ignored, lean=8.0, pad=0, shift=0,
                 std=0.05):
    w = _randn((vocab, width), g, std, torch.bfloat16, pad, shift)
    y = (torch.rand(n, generator=g, device=DEV) * vocab).long().clamp(
        max=vocab - 1)
    rows = w[y].float()
    rows = rows / rows.square().sum(1, keepdim=True).sqrt().clamp(min=1e-6)
    k = torch.rand((n, 1), generator=g, device=DEV) * lean
    h = _randn((n, width), g, 1.0, torch.bfloat16, pad, shift)
    h.copy_(h.float() + k * rows)
    gone = torch.rand(n, generator=g, device=DEV) < ignored
    return h, w, torch.where(gone, -100, y)


def _head_reference(h, w, y, scale=1.0):
    """Loss, token losses and gradients with bounds of each."""
    keep = (y >= 0)
    hd = torch.where(keep[:, None], h.double(), 0.0)
    wd = w.double()
    logits = hd @ wd.T
    width = h.shape[1]
    # a logit's error; a softmax entry's relative error
    e_logit = (width + 2) * 2 * U32 * float((hd.abs() @ wd.abs().T).max())
    logp = torch.log_softmax(logits, 1)
    e_p = 2 * e_logit + 2.0 ** -20
    at = y.clamp(min=0)[:, None]
    token = torch.where(keep, -torch.gather(logp, 1, at)[:, 0], 0.0)
    n = max(1, int(keep.sum()))
    e_token = 2 * e_logit + 2.0 ** -19 + 2 * U32 * float(logits.abs().max())
    p = logp.exp()
    coef = torch.where(keep, scale / n, 0.0)[:, None]
    dl = p.clone()
    dl.scatter_add_(1, at, -torch.ones_like(at, dtype=torch.float64))
    dl = dl * coef
    e_dl = (e_p * p * coef.abs() + (2.0 ** -8 + 4 * U32) * dl.abs())
    vocab = w.shape[0]
    dh, dw = dl @ wd, dl.T @ hd
    dh_err = e_dl @ wd.abs() + (vocab + 2) * 2 * U32 * (dl.abs() @ wd.abs())
    dw_err = e_dl.T @ hd.abs() + \
        (len(y) + 2) * 2 * U32 * (dl.abs().T @ hd.abs())
    return dict(token=token, e_token=e_token, loss=token.sum() / n,
                dh=dh, dw=dw, dh_err=dh_err, dw_err=dw_err)


def _head_case(n, vocab, width, ignored=0.1, pad=0, shift=0, grad="bf16",
               add=False, scale=None, lean=8.0, seed=0, max_tokens=None):
    g = _gen(seed + 7 * n + width)
    h, w, y = _head_inputs(n, vocab, width, g, ignored, lean, pad, shift)
    ref = _head_reference(h, w, y, 1.0 if scale is None else scale)
    plan = VocabPlan(vocab, width, max_tokens or n)
    token = torch.full((n,), 7.0, device=DEV)
    loss = plan.loss(h, w, y, token_loss=token)
    _close(token, ref["token"], ref["token"] * 2 ** -20 + ref["e_token"])
    _close(loss[0], ref["loss"], ref["loss"] * 2 ** -20 + ref["e_token"])
    # the gradients
    dh = _randn((n, width), g, 1.0, torch.bfloat16, pad, shift)
    dw = _randn((vocab, width), g, 0.01, DT[grad], pad, shift)
    before = dw.double()
    token2 = torch.full((n,), 7.0, device=DEV)
    s = None if scale is None else torch.full((1,), scale, device=DEV)
    loss2 = plan.loss_grad(h, w, y, dh, dw, scale=s, accumulate=add,
                           token_loss=token2)
    assert torch.equal(loss, loss2) and torch.equal(token, token2)
    assert plan.query() == 0
    _close(dh, ref["dh"], ref["dh_err"] + UBF * ref["dh"].abs())
    want = ref["dw"] + before if add else ref["dw"]
    bound = ref["dw_err"] + 4 * U32 * before.abs()
    if grad == "bf16":
        bound = bound + UBF * want.abs()
    _close(dw, want, bound)
    assert (dh[y < 0] == 0).all()
    # the same bits again
    dh3, dw3 = torch.empty_like(dh), torch.empty_like(dw)
    dw3.copy_(before)
    plan.loss_grad(h, w, y, dh3, dw3, scale=s, accumulate=add)
    assert torch.equal(dh, dh3) and torch.equal(dw, dw3)
    plan.destroy()


@pytest.mark.parametrize("n,vocab,width", [
    (1, 1, 8), (1, 30522, 64), (5, 255, 8), (127, 256, 64), (128, 257, 72),
    (129, 1000, 136), (300, 5003, 256), (1000, 2100, 520)])
def test_head(n, vocab, width):
    _head_case(n, vocab, width)


@pytest.mark.parametrize("n,vocab,width,pad,shift", [
    (50, 300, 1, 0, 0), (130, 700, 63, 0, 0), (65, 513, 129, 3, 1),
    (200, 400, 64, 8, 0), (200, 400, 64, 1, 0), (70, 400, 64, 0, 1)])
def test_head_of_odd_widths_and_strides(n, vocab, width, pad, shift):
    _head_case(n, vocab, width, pad=pad, shift=shift)


@pytest.mark.parametrize("grad,add,scale", [
    ("f32", False, None), ("f32", True, 0.5), ("bf16", True, 1024.0)])
def test_head_gradient_forms(grad, add, scale):
    _head_case(333, 1500, 200, grad=grad, add=add, scale=scale)
    _head_case(64, 300, 36, pad=1, grad=grad, add=add, scale=scale)


@pytest.mark.parametrize("ignored", [0.5, 0.97, 1.0])
def test_head_with_few_labels(ignored):
    _head_case(400, 600, 64, ignored=ignored, max_tokens=500)


def test_head_of_many_tokens():
    """Rows counted in runs: labels far apart, and none in most runs."""
    g = _gen(11)
    n, vocab, width = 40000, 40, 16
    h, w, y = _head_inputs(n, vocab, width, g, 0.0)
    y[5000:31000] = -1
    y[20000] = 7
    y[39990:] = -3
    ref = _head_reference(h, w, y)
    plan = VocabPlan(vocab, width, n)
    token = torch.full((n,), 7.0, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = plan.loss_grad(h, w, y, dh, dw, token_loss=token)
    _close(token, ref["token"], ref["token"] * 2 ** -20 + ref["e_token"])
    _close(loss[0], ref["loss"], ref["loss"] * 2 ** -20 + ref["e_token"])
    _close(dh, ref["dh"], ref["dh_err"] + UBF * ref["dh"].abs())
    _close(dw, ref["dw"], ref["dw_err"] + UBF * ref["dw"].abs())


def test_head_in_several_pieces():
    """More logits than the workspace holds."""
    _head_case(4500, 30001, 64, ignored=0.0)


def test_head_of_sure_rows():
    """Labels with a probability of nearly one, and of nearly zero."""
    _head_case(200, 900, 256, lean=60.0)


def test_absent_rows_may_hold_anything():
    g = _gen(5)
    h, w, y = _head_inputs(200, 500, 64, g, 0.3)
    plan = VocabPlan(500, 64, 200)

    def go(hidden):
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        loss = plan.loss_grad(hidden, w, y, dh, dw)
        return loss, dh, dw
    a = go(h)
    bad = h.clone()
    bad[y < 0] = float("nan")
    bad[(y < 0).nonzero()[0, 0]] = float("inf")
    for x, z in zip(a, go(bad)):
        assert torch.equal(x, z)
    # a row with a label keeps its Inf and NaN to itself where the formula does
    bad = h.clone()
    row = int((y >= 0).nonzero()[3, 0])
    bad[row, 0] = float("nan")
    loss, dh, dw = go(bad)
    assert torch.isnan(loss).all() and torch.isnan(dh[row]).all()
    others = torch.arange(200, device=DEV) != row
    assert torch.equal(dh[others], a[1][others])
    # and the next call is not touched by what that one left
    for x, z in zip(a, go(h)):
        assert torch.equal(x, z)


def test_masked_words_have_no_share():
    """Logits of the type's lowest values and of -inf."""
    g = _gen(6)
    h, w, y = _head_inputs(40, 300, 64, g, 0.0)
    h[:, 0] = 1.0
    w[:, 0] = 0.0
    plan = VocabPlan(300, 64, 40)
    y = y % 200
    want = plan.loss(h, w[:300], y).clone()
    ref = _head_reference(h, w[:200], y)
    for low in (-float("inf"), torch.finfo(torch.bfloat16).min):
        masked = w.clone()
        masked[200:] = 0.0
        masked[200:, 0] = low
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        loss = plan.loss_grad(h, masked, y, dh, dw)
        _close(loss[0], ref["loss"], ref["loss"] * 2 ** -20 + ref["e_token"])
        assert float(loss) < float(want)
        assert (dw[200:] == 0).all()


def test_head_bad_labels_and_no_tokens():
    plan = VocabPlan(30, 16, 8)
    g = _gen(8)
    h, w, _ = _head_inputs(4, 30, 16, g, 0.0)
    y = torch.tensor([3, 30, -5, 2 ** 40], device=DEV)
    token = torch.empty(4, device=DEV)
    loss = plan.loss(h, w, y, token_loss=token)
    assert plan.query(clear=True) == B.LAMB_STATUS_BAD_INDEX
    assert token[1:].tolist() == [0, 0, 0] and float(loss) == float(token[0])
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    dw = torch.ones(30, 16, device=DEV, dtype=torch.bfloat16)
    loss = plan.loss_grad(h[:0], w, none, h[:0].clone(), dw, accumulate=True)
    assert float(loss) == 0 and float(dw.sum()) == 480
    loss = plan.loss_grad(h[:0], w, none, h[:0].clone(), dw)
    assert float(loss) == 0 and float(dw.abs().sum()) == 0


def test_head_gradient_against_differences():
    """Along a random direction of h and of W, by differences of the loss."""
    g = _gen(9)
    h, w, y = _head_inputs(60, 90, 32, g, 0.2, lean=3.0, std=0.3)
    plan = VocabPlan(90, 32, 60)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    plan.loss_grad(h, w, y, dh, dw)

    def loss64(hd, wd):
        z = hd @ wd.T
        return torch.nn.functional.cross_entropy(z, y, ignore_index=-100)
    rh = torch.randn(h.shape, generator=g, device=DEV, dtype=torch.float64)
    rw = torch.randn(w.shape, generator=g, device=DEV, dtype=torch.float64)
    e = 1e-5
    for got, a, b in ((dh, rh, 0 * rw), (dw, 0 * rh, rw)):
        diff = (loss64(h.double() + e * a, w.double() + e * b) -
                loss64(h.double() - e * a, w.double() - e * b)) / (2 * e)
        r = a if a.shape == got.shape and a.abs().sum() else b
        along = (got.double() * r).sum()
        # each entry is within 2^-7 of itself or of its terms (some 2^-8 each)
        assert abs(float(along - diff)) <= 2 ** -7 * float(
            (got.double() * r).norm()) * 4


def test_head_in_a_graph_and_on_another_stream():
    g = _gen(10)
    h, w, y = _head_inputs(300, 700, 64, g, 0.1)
    plan = VocabPlan(700, 64, 300)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = torch.empty(1, device=DEV)
    plan.loss_grad(h, w, y, dh, dw, loss=loss)
    want = [x.clone() for x in (loss, dh, dw)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        plan.loss_grad(h, w, y, dh, dw, loss=loss)
        plan.embed_grad(dh, y, dw, accumulate=True)
    for x in (loss, dh, dw):
        x.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(dh, want[1])
    tied = plan.embed_grad(want[1], y, want[2].clone(), accumulate=True)
    assert torch.equal(dw, tied)


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def test_tensors_are_checked():
    plan = VocabPlan(30, 16, 8)
    f = dict(device=DEV)
    tab = torch.zeros(30, 16, **f)
    bf = tab.bfloat16()
    ids = torch.zeros(4, dtype=torch.int64, **f)
    rows = torch.zeros(4, 16, **f)
    bad = [
        lambda: plan.embed(tab.double(), ids),
        lambda: plan.embed(tab[:29], ids),
        lambda: plan.embed(tab.t().contiguous().t(), ids),
        lambda: plan.embed(tab, ids.int()),
        lambda: plan.embed(tab, ids[None]),
        lambda: plan.embed(tab.cpu(), ids),
        lambda: plan.embed(tab, ids.cpu()),
        lambda: plan.embed(tab, ids, out=rows[:3]),
        lambda: plan.embed_grad(rows[:3], ids, tab),
        lambda: plan.embed_grad(rows.half(), ids, tab),
        lambda: plan.loss(rows, bf, ids),
        lambda: plan.loss(rows.bfloat16(), tab, ids),
        lambda: plan.loss_grad(rows.bfloat16(), bf, ids, rows, bf),
        lambda: plan.loss(rows.bfloat16(), bf, ids,
                          token_loss=torch.zeros(3, **f)),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    many = torch.zeros(9, dtype=torch.int64, **f)
    with pytest.raises(B.LambError) as e:
        plan.embed(tab, many)
    assert e.value.status == B.LAMB_ERR_INVALID_ARG and "max_tokens" in str(e)
    assert plan.query() == 0
