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
