"""GPU tests of the language-model operators where two plans, two streams, a
refused call or extreme values meet.  Bounds as in the operators' other tests.
"""
import math

import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300.muon import MuonPlan
from paper_1904_00962_gb300.state import DeviceState, LambPlan
from paper_1904_00962_gb300.vocab import VocabPlan
from test_muon_gpu import TOL, _exact, _matrix, _near
from test_vocab_gpu import (DEV, U32, UBF, _close, _gen, _head_reference,
                            _randn)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib(gpu):
    B.load()


# ---------------------------------------------------------------------------
# plans beside one another
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_later_muon_plan_leaves_an_earlier_one_its_shared_memory(dtype):
    """The small matrices' kernel takes as much of it as the plan's largest
    needs: plans of less, or without such a matrix, come after one of more."""
    g = _gen(20)
    shapes = [(64, 128), (256, 300)]
    u = [_matrix(*s, g).to(dtype) for s in shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    kind = "f32" if dtype == torch.float32 else "bf16"
    plan = MuonPlan(shapes, grad_dtype=kind)
    plan.bind_direction(u, o)
    later = [MuonPlan([(256, 256)]), MuonPlan([(4, 4)], grad_dtype="bf16")]
    plan.direction(B.make_muon_hyper())
    for x, y in zip(u, o):
        _near(y, _exact(x), TOL + UBF / 2)
    w = [_matrix(*s, g, std=0.05).float() for s in shapes]
    m = [torch.zeros(s, device=DEV) for s in shapes]
    plan.bind(w, u, m)
    before = [x.double() for x in w]
    lr = torch.full((1,), 0.02, device=DEV)
    plan.step(B.make_muon_hyper(weight_decay=0.0, scale="one"), lr)
    for x, y, z in zip(w, before, u):
        moved = (y - x.double()) / 0.02
        want = _exact(z.double() * 0.0975)  # (1 - b) (1 + b) g, b = 0.95
        # the weights' own fp32 digits beside the direction's error
        off = float((moved - want).norm())
        assert off <= TOL * float(want.norm()) + \
            4 * U32 / 0.02 * float(y.norm())
    assert plan.query() == 0 and all(p.query() == 0 for p in later)


def test_every_small_matrix_fits_shared_memory():
    """The sides at which such a matrix needs most."""
    shapes = [(64, 128), (25, 819), (819, 25), (1, 20480), (5, 4096), (3, 6826),
              (64, 64), (2, 10239)]
    g = _gen(21)
    u = [_matrix(*s, g).float() for s in shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    plan = MuonPlan(shapes)
    plan.bind_direction(u, o)
    plan.direction(B.make_muon_hyper())
    for x, y, s in zip(u, o, shapes):
        _near(y, _exact(x), TOL + UBF / 2, s)


@pytest.mark.parametrize("how", ["stream", "handle", "default"])
def test_results_belong_to_the_stream_that_writes_them(how):
    """Memory of a result that is dropped goes on in its stream's order: the
    current stream does not get it."""
    g = _gen(30)
    vocab, width, n = 500, 1000, 1700
    tab = _randn((vocab, width), g)
    ids = torch.randint(vocab, (n,), generator=g, device=DEV)
    h, w = tab[:40].bfloat16(), tab.bfloat16()
    plan = VocabPlan(vocab, width, n)
    s = torch.cuda.Stream()
    given = {"stream": s, "handle": s.cuda_stream, "default": 0}[how]
    current = torch.cuda.Stream() if how == "default" else \
        torch.cuda.current_stream()
    want = plan.loss(h, w, ids[:40]).clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(current):
        for call, value, like in (
                (lambda: plan.embed(tab, ids, stream=given), tab[ids], (n, width)),
                (lambda: plan.loss(h, w, ids[:40], stream=given), want, (1,)),
                (lambda: plan.loss_grad(h, w, ids[:40], torch.empty_like(h),
                                        torch.empty_like(w), stream=given),
                 want, (1,))):
            torch.cuda.synchronize()
            got = call()
            torch.cuda.synchronize()
            assert torch.equal(got, value)
            at = got.data_ptr()
            del got
            new = [torch.empty(like, device=DEV) for _ in range(8)]
            assert at not in [x.data_ptr() for x in new]


# ---------------------------------------------------------------------------
# the head where labels are nearly sure
# ---------------------------------------------------------------------------
def _sure_rows(n, vocab, width, word, g):
    """Hidden rows whose label is `word`, its probability between a quarter and
    1 - 1e-6.  Column 0 of W is that word's alone and no hidden row has it, so
    grad_hidden[:, 0] is the label's entry of the logits' gradient itself."""
    w = _randn((vocab, width), g, 0.05, torch.bfloat16)
    w[:, 0] = 0.0
    way = w[word].float() / w[word].float().norm()
    w[word, 0] = 1.0
    h = _randn((n, width), g)
    top = torch.linspace(8.0, 27.0, n, device=DEV)[:, None]
    at = (w[word].float() * way).sum()
    h = h - (h @ way)[:, None] * way + top / at * way
    h[:, 0] = 0.0
    return h.bfloat16(), w


@pytest.mark.parametrize("n,vocab,width,word", [
    (77, 701, 128, 300), (300, 5003, 96, 4999), (1, 300, 64, 0)])
def test_sure_labels_keep_their_digits(n, vocab, width, word):
    """The token losses and the label's entries of the gradient, each against
    itself.  With R the sum of exp(l_v - l_y) over the other words both are
    functions of R, whose relative error is that of two logits (a product's sum
    of `width` terms is within 2^-23 of the sum of their sizes for each), of
    base-2 exponents formed in fp32, and of a sum of `vocab` terms."""
    g = _gen(vocab)
    h, w = _sure_rows(n, vocab, width, word, g)
    y = torch.full((n,), word, device=DEV)
    logits = h.double() @ w.double().T
    others = logits.clone()
    others[:, word] = -math.inf
    r = torch.exp(torch.logsumexp(others, 1) - logits[:, word])
    want = torch.log1p(r)
    entry = -r / (1.0 + r) / n
    e_logit = (width + 2) * 2 * U32 * (h.double().abs() @
                                       w.double().abs().T).amax(1)
    rel = 2 * e_logit + 8 * U32 * logits.abs().amax(1) + 2.0 ** -20 + \
        (vocab + 2) * U32
    if n > 1:      # what the inputs are for
        assert float(r.min()) < 2e-6 and float(r.max()) > 1e-2
        assert float(rel.max()) < 2e-3

    plan = VocabPlan(vocab, width, n)
    token = torch.empty(n, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    plan.loss_grad(h, w, y, dh, dw, token_loss=token)
    _close(token, want, want * (rel + 2.0 ** -21))
    # one bf16 term: rounded as the logits' gradient, once more on its way out
    e_entry = entry.abs() * (rel + UBF)
    _close(dh[:, 0], entry, e_entry)
    dw_want = entry @ h.double()
    _close(dw[word], dw_want, e_entry @ h.double().abs() +
           (n + 2) * 2 * U32 * (entry.abs() @ h.double().abs()) +
           UBF * dw_want.abs())
    assert plan.query() == 0


# ---------------------------------------------------------------------------
# masks of the lowest values
# ---------------------------------------------------------------------------
LOWS = [-1e4, -1e10, -1e30, float(torch.finfo(torch.bfloat16).min)]


@pytest.mark.parametrize("low", LOWS)
@pytest.mark.parametrize("n", [40, 200])
def test_tiles_of_masked_words(n, low):
    """Words from 200 on are masked by a low value in W's first column, which
    every hidden row has as one: whole tiles hold nothing else.  The others'
    loss and gradients are those of a vocabulary without them."""
    g = _gen(n)
    vocab, width, real = 900, 64, 200
    h = _randn((n, width), g, 1.0, torch.bfloat16)
    w = _randn((vocab, width), g, 0.1, torch.bfloat16)
    h[:, 0] = 1.0
    w[:, 0] = 0.0
    y = torch.arange(n, device=DEV) % real
    y[3] = -1
    ref = _head_reference(h, w[:real], y)
    w[real:] = 0.0
    w[real:, 0] = low
    plan = VocabPlan(vocab, width, n)
    token = torch.empty(n, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = plan.loss_grad(h, w, y, dh, dw, token_loss=token)
    _close(token, ref["token"], ref["token"] * 2 ** -20 + ref["e_token"])
    _close(loss[0], ref["loss"], ref["loss"] * 2 ** -20 + ref["e_token"])
    _close(dh, ref["dh"], ref["dh_err"] + UBF * ref["dh"].abs())
    _close(dw[:real], ref["dw"], ref["dw_err"] + UBF * ref["dw"].abs())
    assert (dw[real:] == 0).all()


@pytest.mark.parametrize("low", LOWS + [1e10, 1e30])
@pytest.mark.parametrize("n,vocab", [(5, 300), (150, 700)])
def test_rows_whose_mask_leaves_nothing(n, vocab, low):
    """Every word has the same logit, however low or high: the loss is ln V and
    the softmax 1 / V."""
    g = _gen(vocab)
    width = 64
    h = _randn((n, width), g, 1.0, torch.bfloat16)
    w = torch.zeros(vocab, width, device=DEV, dtype=torch.bfloat16)
    h[:, 0] = 1.0
    w[:, 0] = low
    y = torch.arange(n, device=DEV) * 7 % vocab
    dl = torch.full((n, vocab), 1.0 / vocab, device=DEV, dtype=torch.float64)
    dl[torch.arange(n, device=DEV), y] -= 1.0
    dl /= n
    want = dl.T @ h.double()
    plan = VocabPlan(vocab, width, n)
    token = torch.empty(n, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = plan.loss_grad(h, w, y, dh, dw, token_loss=token)
    ln_v = torch.full((n,), math.log(vocab), device=DEV, dtype=torch.float64)
    _close(token, ln_v, ln_v * 2.0 ** -18)      # sums of V equal terms: exact
    _close(loss[0], ln_v[0], ln_v[0] * 2.0 ** -18)
    # the logits' gradient in bf16 (2^-9, the exponentials 2^-20), n terms
    size = dl.abs().T @ h.double().abs()
    _close(dw, want, (2.0 ** -9 + 2.0 ** -18 + (n + 2) * 2 * U32) * size +
           UBF * want.abs())
    assert (dh[:, 1:] == 0).all()               # W is zero there


def test_an_infinite_logit_of_the_label_is_not_a_loss_of_zero():
    """inf - inf: the formula has no value, and neither have the results."""
    h = torch.ones(1, 16, device=DEV, dtype=torch.bfloat16)
    w = torch.zeros(300, 16, device=DEV, dtype=torch.bfloat16)
    w[7, 3] = math.inf
    plan = VocabPlan(300, 16, 1)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = plan.loss_grad(h, w, torch.tensor([7], device=DEV), dh, dw)
    assert torch.isnan(loss).all() and torch.isnan(dw[7]).all()


# ---------------------------------------------------------------------------
# after a refused call
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("refused", ["memory", "device", "another's device"])
def test_a_failed_plan_is_not_the_next_call_s_error(refused):
    """A plan of 2 TB is refused by the allocation, one on a device that is not
    there by the runtime: the error belongs to that call alone."""
    words = VocabPlan(10, 16, 8)
    muon = MuonPlan([(8, 8), (80, 70)])
    state = DeviceState([100])
    lamb = LambPlan(state)
    tab = torch.ones(10, 16, device=DEV)
    odd = torch.ones(10, 17, device=DEV, dtype=torch.bfloat16)[:, :16]
    ids = torch.arange(8, device=DEV)
    u = [torch.ones(s, device=DEV) for s in muon.shapes]
    o = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in muon.shapes]
    muon.bind_direction(u, o)
    one = torch.ones(1, device=DEV)
    step = torch.ones(1, dtype=torch.int64, device=DEV)
    fail = {"memory": lambda: VocabPlan(2 ** 30, 2 ** 10, 64),
            "device": lambda: MuonPlan([(8, 8)], device="cuda:99"),
            "another's device": lambda: B.lamb_plan_create([8], device=99)}
    calls = [lambda: words.embed(tab, ids),
             lambda: words.embed_grad(tab[:0], ids[:0], tab.clone()),
             lambda: words.embed_grad(tab[:8], ids, tab.clone()),
             lambda: words.loss(odd[:8], odd, ids),
             lambda: words.loss_grad(odd[:0], odd, ids[:0], odd[:0],
                                     odd.clone()),
             lambda: muon.direction(B.make_muon_hyper())]
    if refused != "another's device":
        calls.append(lambda: lamb.lamb_step(B.make_hyper(), step, one))
    for call in calls:
        with pytest.raises(B.LambError) as e:
            fail[refused]()
        assert e.value.status in (B.LAMB_ERR_OOM, B.LAMB_ERR_CUDA,
                                  B.LAMB_ERR_INVALID_ARG)
        call()
    torch.cuda.synchronize()
    assert words.query() == 0 and muon.query() == 0 and lamb.query() == 0


# ---------------------------------------------------------------------------
# what lies beside a result
# ---------------------------------------------------------------------------
def _framed(rows, width, pad, shift, dtype):
    """A [rows, width] view of rows of width + pad, and whether all beside it
    in its buffer is still as it was."""
    buf = torch.full((rows * (width + pad) + shift + 64,), 7.0, device=DEV,
                     dtype=dtype)
    mine = torch.zeros_like(buf, dtype=torch.bool)
    at = slice(shift, shift + rows * (width + pad))
    mine[at].view(rows, width + pad)[:, :width] = True
    view = buf[at].view(rows, width + pad)[:, :width]
    return view, lambda: bool((buf[~mine] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("width,pad,shift", [
    (1, 7, 0), (37, 3, 8), (44, 4, 0), (63, 1, 0), (64, 8, 0), (100, 28, 8),
    (257, 7, 0), (30, 2, 1)])
def test_columns_beside_a_result_are_left_alone(dtype, add, width, pad, shift):
    """Columns between the width and the row stride belong to others."""
    g = _gen(width)
    n, vocab = 150, 700
    plan = VocabPlan(vocab, width, n)
    tab = _randn((vocab, width), g, 0.1, torch.bfloat16)
    h = _randn((n, width), g, 1.0, torch.bfloat16)
    y = torch.randint(vocab, (n,), generator=g, device=DEV)
    y[::5] = -1
    out, out_ok = _framed(n, width, pad, shift, dtype)
    plan.embed(tab, y, out=out)
    assert out_ok()
    for rows in (n, 60):                       # pairs of CTAs, single ones
        dw, dw_ok = _framed(vocab, width, pad, shift, dtype)
        dh, dh_ok = _framed(rows, width, pad, shift, torch.bfloat16)
        token, token_ok = _framed(1, rows, 0, shift, torch.float32)
        dw.zero_()
        plan.loss_grad(h[:rows], tab, y[:rows], dh, dw, accumulate=add,
                       token_loss=token[0])
        assert dw_ok() and dh_ok() and token_ok()
        plan.embed_grad(dh, y[:rows], dw, accumulate=add)
        assert dw_ok()
    assert plan.query() == 0
