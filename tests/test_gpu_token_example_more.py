"""The token model of examples/: reading without targets."""
import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_reading_without_targets_gives_no_log_probabilities_of_them():
    spec = importlib.util.spec_from_file_location("token_model", os.path.join(ROOT, "examples", "token_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = example.TokenModel(100, 64, 2)
    tokens, positions = example.text(100, 30), torch.arange(30, device="cuda")
    logp, entropy, ids, alternatives = model.read(tokens, positions, top=2)
    assert logp is None
    given, e, i, a = model.read(tokens, positions, targets=ids[0], top=2)
    assert torch.equal(e, entropy) and torch.equal(i, ids) and torch.equal(a, alternatives)
    assert torch.equal(given, alternatives[0])          # the likeliest token's own
