"""Trains a small language model with a tied word table, on synthetic text.

    python examples/tied_language_model.py [--steps 60]

One step, as a training loop around this library makes it:
  lookup    rows of the table's bf16 copy, scaled          (VocabPlan.embed)
  layer     x + tanh(x W1) W2, forward and backward        (plain PyTorch)
  head      cross entropy against the same table, with the gradients of the
            hidden rows and of the table                   (VocabPlan.loss_grad)
  lookup's gradient, added to the head's                   (VocabPlan.embed_grad)
  update    LAMB on the table and the bias                 (LambPlan.lamb_step),
            orthogonalised momentum on W1 and W2           (MuonPlan.step)
The text is a Markov chain: each word has one likely successor, and a tenth of
the positions are padding, so the loss falls from ln(vocab) towards the chain's
entropy.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1904_00962_gb300 import binding as B  # noqa: E402
from paper_1904_00962_gb300.muon import MuonPlan  # noqa: E402
from paper_1904_00962_gb300.state import DeviceState, LambPlan  # noqa: E402
from paper_1904_00962_gb300.vocab import VocabPlan  # noqa: E402


class TiedModel:
    def __init__(self, vocab=500, width=64, inner=256, tokens=1024, seed=0,
                 device="cuda:0"):
        self.vocab, self.width = vocab, width
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.gen, self.device = gen, device
        self.words = VocabPlan(vocab, width, max_tokens=tokens, device=device)
        # table and bias: LAMB's tensors, fp32 with a bf16 copy and gradients
        self.state = DeviceState([vocab * width, width], grad_dtype="bf16",
                                 copy_dtype="bf16", device=device)
        self.table = self.state.view("copy", 0).view(vocab, width)
        self.table_grad = self.state.view("g", 0).view(vocab, width)
        self.bias = self.state.view("w", 1)
        self.bias_grad = self.state.view("g", 1)
        w = self.state.view("w", 0)
        w.copy_(torch.randn(w.shape, generator=gen, device=device) * 0.05)
        self.table.copy_(w.view(vocab, width))
        self.lamb = LambPlan(self.state, [1, 0])
        # W1, W2: Muon's matrices
        shapes = [(width, inner), (inner, width)]
        self.w = [torch.randn(s, generator=gen, device=device) / math.sqrt(s[0])
                  for s in shapes]
        self.m = [torch.zeros_like(x) for x in self.w]
        self.g = [torch.zeros_like(x, dtype=torch.bfloat16) for x in self.w]
        self.copy = [x.bfloat16() for x in self.w]
        self.muon = MuonPlan(shapes, grad_dtype="bf16", copy_dtype="bf16",
                             device=device)
        self.muon.bind(self.w, self.g, self.m, self.copy)
        self.step_count = torch.ones(1, dtype=torch.int64, device=device)
        self.lr = torch.full((1,), 0.02, device=device)
        self.muon_lr = torch.full((1,), 0.02, device=device)
        self.hyper = B.make_hyper(weight_decay=0.01, increment_step=True)
        self.muon_hyper = B.make_muon_hyper(scale="rms")
        self.scale = math.sqrt(width)

    def step(self, ids, labels):
        """One update; the loss (a device tensor) before it."""
        x = self.words.embed(self.table, ids, scale=self.scale)
        a = torch.tanh(x @ self.copy[0])
        h = x + a @ self.copy[1] + self.bias.bfloat16()
        dh = torch.empty_like(h)
        loss = self.words.loss_grad(h, self.table, labels, dh, self.table_grad)
        self.bias_grad.copy_(dh.float().sum(0))
        self.g[1].copy_(a.T @ dh)
        dz = (dh @ self.copy[1].T) * (1 - a * a)
        self.g[0].copy_(x.T @ dz)
        dx = dh + dz @ self.copy[0].T
        self.words.embed_grad(dx, ids, self.table_grad, scale=self.scale,
                              accumulate=True)
        self.lamb.lamb_step(self.hyper, self.step_count, self.lr)
        self.muon.step(self.muon_hyper, self.muon_lr)
        return loss

    def batch(self, tokens):
        """Words and their successors: nine of ten times the word's usual one;
        a tenth of the positions are padding."""
        g, d = self.gen, self.device
        ids = torch.randint(self.vocab, (tokens,), generator=g, device=d)
        usual = (ids * 7 + 3) % self.vocab
        other = torch.randint(self.vocab, (tokens,), generator=g, device=d)
        pick = torch.rand(tokens, generator=g, device=d)
        labels = torch.where(pick < 0.9, usual, other)
        pad = torch.rand(tokens, generator=g, device=d) < 0.1
        return torch.where(pad, -1, ids), torch.where(pad, -1, labels)


def train(steps=60, tokens=1024, seed=0, log=None, **model):
    """The losses of `steps` updates."""
    m = TiedModel(tokens=tokens, seed=seed, **model)
    losses = []
    for k in range(steps):
        losses.append(m.step(*m.batch(tokens)).clone())
        if log and k % 10 == 9:
            log(f"step {k + 1:4d}  loss {float(losses[-1]):.4f}")
    assert m.words.query() == 0 and m.lamb.query() == 0 and m.muon.query() == 0
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=1024)
    args = ap.parse_args()
    train(args.steps, args.tokens, log=print)
