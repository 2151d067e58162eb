"""The example of a quantised inference with its proofs runs, and answers the same twice."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example_runs_and_repeats(capsys):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "quantised_inference.py")
    spec = importlib.util.spec_from_file_location("quantised_inference", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    answers, reports = mod.main()
    assert answers.shape == (3, 6) and int(answers.min()) >= 0 and int(answers.max()) < mod.VOCAB
    for i, r in enumerate(reports):
        assert torch.equal(r["top_ids"][:, 0].long(), answers[:, i]) and (r["rank"] == 0).all()
        assert torch.equal(r["top"][:, 0], r["target"]) and torch.isfinite(r["entropy"]).all()
    again, _ = mod.main()
    assert torch.equal(again, answers)
    assert "proof of" in capsys.readouterr().out
