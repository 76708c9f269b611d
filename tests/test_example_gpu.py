"""GPU test of the tied language model's example: the operators and both
optimizers together, whose loss has to fall."""
import importlib.util
import math
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location(
        "tied_language_model",
        os.path.join(ROOT, "examples", "tied_language_model.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_tied_language_model_learns(gpu):
    losses = _example().train(steps=80)
    assert all(math.isfinite(x) for x in losses)
    # blind guessing is ln(500) = 6.2, the chain's entropy about 1
    assert losses[0] > 5.5
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0]


def test_tied_language_model_repeats_its_bits(gpu):
    mod = _example()
    assert mod.train(steps=6) == mod.train(steps=6)
