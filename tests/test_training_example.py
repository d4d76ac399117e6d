"""The example that runs SignMuon, AdamW with clipping and layer norm together."""
import importlib.util
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("state_bits", [32, 8])
def test_the_example_learns(state_bits):
    """From a uniform guess (ln 64) at least half of the way to the chain's entropy, without a step that is not finite."""
    spec = importlib.util.spec_from_file_location("train_language_model", os.path.join(ROOT, "examples", "train_language_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, entropy = example.train(steps=150, workers=3, state_bits=state_bits, vocabulary=64, context=16, width=64)
    assert all(math.isfinite(x) for x in losses) and abs(losses[0] - math.log(64)) < 1.0
    assert sum(losses[-10:]) / 10 < 0.5 * (math.log(64) + entropy)


@pytest.mark.gpu
@pytest.mark.parametrize("width", [256, 768])
def test_the_example_steps_at_widths_of_ordinary_models(width):
    """The first layer norm has no residual and the others have one, step after step."""
    spec = importlib.util.spec_from_file_location("train_language_model", os.path.join(ROOT, "examples", "train_language_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, _ = example.train(steps=4, workers=2, vocabulary=64, context=16, batch=4, width=width)
    assert len(losses) == 4 and all(math.isfinite(x) for x in losses)
