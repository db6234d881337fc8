"""The example that puts the language-model calls and the search together runs, and does what it says: neighbours help the
untrained model, and training towards them and towards the text helps the model alone."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_runs_and_learns():
    spec = importlib.util.spec_from_file_location("neighbour_lm", os.path.join(ROOT, "examples", "neighbour_lm.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(vocab=500, train=40_000, test=1_000, steps=30)
    assert got["before"]["model"] > 300                                       # 500 tokens, nothing learnt
    assert got["before"]["mixture"] < 0.5 * got["before"]["model"]            # the neighbours know
    assert got["distilled"]["model"] < 0.8 * got["before"]["model"]
    assert got["trained"]["model"] < got["distilled"]["model"]
