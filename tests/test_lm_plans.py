"""CPU tests of the Python plans of the language-model operators: what they
allocate where, what they keep, and what they take.  The C entry points are
stand-ins; no kernel runs."""
import contextlib
import types

import pytest
import torch

from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300 import muon as muon_mod
from paper_1904_00962_gb300 import vocab as vocab_mod
from paper_1904_00962_gb300.muon import MuonPlan
from paper_1904_00962_gb300.vocab import VocabPlan


def _words(monkeypatch, vocab=10, width=16, calls=None):
    """A vocabulary plan on the CPU's tensors whose C calls are recorded."""
    monkeypatch.setattr(B, "lamb_vocab_create", lambda *a: 0)
    for name in ("embed", "embed_grad", "loss", "loss_grad"):
        monkeypatch.setattr(
            B, "lamb_vocab_" + name,
            lambda *a, name=name: None if calls is None
            else calls.append((name, a)))
    plan = VocabPlan(vocab, width, 8)
    plan.device, plan._index = torch.device("cpu"), -1
    return plan


@pytest.mark.parametrize("raw,handle", [(False, 77), (True, 77), (True, 0)])
def test_results_are_allocated_for_the_stream_that_writes_them(monkeypatch,
                                                               raw, handle):
    """A tensor that the plan makes belongs to the given stream: the allocator
    may hand its memory on in that stream's order only."""
    calls, current, made = [], [None], []
    plan = _words(monkeypatch, calls=calls)
    stream = types.SimpleNamespace(cuda_stream=handle)

    @contextlib.contextmanager
    def on(s):
        before, current[0] = current[0], s.cuda_stream
        yield
        current[0] = before

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(
        torch.cuda, "ExternalStream",
        lambda s, device=None: types.SimpleNamespace(cuda_stream=s))
    monkeypatch.setattr(
        torch.cuda, "default_stream",
        lambda device=None: types.SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(
        torch, "empty",
        lambda *a, **k: made.append(current[0]) or empty(*a, **k))
    table, ids = torch.zeros(10, 16), torch.zeros(4, dtype=torch.int64)
    rows = torch.zeros(4, 16, dtype=torch.bfloat16)
    given = handle if raw else stream
    plan.embed(table, ids, stream=given)
    plan.loss(rows, table.bfloat16(), ids, stream=given)
    plan.loss_grad(rows, table.bfloat16(), ids, rows.clone(),
                   table.bfloat16(), stream=given)
    assert made == [handle] * 3
    assert [name for name, _ in calls] == ["embed", "loss", "loss_grad"]
    assert all(args[-1] == handle for _, args in calls)
    assert current == [None]
    # without a stream: PyTorch's current one, for both
    made.clear()
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5,
                        raising=False)
    plan.embed(table, ids)
    assert made == [None] and calls[-1][1][-1] == 5


class _OnGpu:
    """What a plan asks of a tensor."""
    is_cuda = True

    def __init__(self, shape, dtype):
        self.shape, self.dtype = shape, dtype

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 256


def _muon(monkeypatch, shapes, **kw):
    monkeypatch.setattr(B, "lamb_muon_create", lambda *a: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5,
                        raising=False)
    return MuonPlan(shapes, **kw)


def _all_bound(plan):
    return [t for ts in plan._bound.values() for t in ts]


def test_a_refused_binding_keeps_the_earlier_tensors(monkeypatch):
    """The device's table still holds their addresses."""
    shapes = [(4, 4), (4, 2)]
    plan = _muon(monkeypatch, shapes)
    bound, fail = [], []

    def c_bind(*args, stream):
        if fail:
            raise B.LambError(B.LAMB_ERR_CUDA, "copy failed")
        bound.append(args)
    monkeypatch.setattr(B, "lamb_muon_bind", c_bind)
    monkeypatch.setattr(B, "lamb_muon_bind_direction", c_bind)
    f32, bf16 = torch.float32, torch.bfloat16

    def tensors(dtype=f32):
        return [_OnGpu(s, dtype) for s in shapes]
    first = w, g, m = tensors(), tensors(), tensors()
    plan.bind(*first)
    u, o = tensors(), tensors(bf16)
    plan.bind_direction(u, o)
    held = w + g + m + u + o
    assert set(map(id, _all_bound(plan))) == set(map(id, held))
    for bad in ((tensors(), tensors(bf16), m), (tensors(), g[:1], m),
                (tensors(), tensors(), tensors(bf16))):
        with pytest.raises(ValueError):
            plan.bind(*bad)
    with pytest.raises(ValueError):
        plan.bind_direction(tensors(), tensors())
    fail.append(True)
    with pytest.raises(B.LambError):
        plan.bind(tensors(), tensors(), tensors())
    with pytest.raises(B.LambError):
        plan.bind_direction(tensors(), tensors(bf16))
    assert len(bound) == 2
    assert set(map(id, _all_bound(plan))) >= set(map(id, held))
    # and a binding that succeeds replaces them
    fail.clear()
    new = tensors(), tensors(), tensors()
    plan.bind(*new)
    assert set(map(id, _all_bound(plan))) == \
        set(map(id, sum(new, []) + u + o))


def test_cuda_is_the_current_device(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(B, "lamb_vocab_create",
                        lambda *a: made.append(a[-1]) or 0)
    monkeypatch.setattr(B, "lamb_muon_create",
                        lambda *a: made.append(a[-1]) or 0)
    plans = [VocabPlan(10, 16, 8, device="cuda"),
             MuonPlan([(4, 4)], device=torch.device("cuda")),
             VocabPlan(10, 16, 8, device="cuda:1"), MuonPlan([(4, 4)])]
    assert made == [3, 3, 1, 0]
    assert [p.device.index for p in plans] == [3, 3, 1, 0]


def test_one_element_has_no_dimension_or_one(monkeypatch):
    """The scale and the loss of one element, as a loss or a gradient scaler
    has them."""
    calls = []
    plan = _words(monkeypatch, calls=calls)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5,
                        raising=False)
    rows = torch.zeros(4, 16, dtype=torch.bfloat16)
    weight, y = torch.zeros(10, 16, dtype=torch.bfloat16), torch.arange(4)
    for scale, loss in ((torch.ones(()), torch.zeros(())),
                        (torch.ones(1), torch.zeros(1))):
        assert plan.loss(rows, weight, y, loss=loss) is loss
        assert calls[-1][1][-2] == loss.data_ptr()
        plan.loss_grad(rows, weight, y, rows.clone(), weight.clone(),
                       scale=scale, loss=loss)
        assert calls[-1][1][7] == scale.data_ptr()
    n = len(calls)
    for scale in (torch.ones(2), torch.ones((), dtype=torch.float64),
                  torch.ones(1, 1)):
        with pytest.raises(ValueError):
            plan.loss_grad(rows, weight, y, rows.clone(), weight.clone(),
                           scale=scale)
    assert len(calls) == n
