"""The example runs the training-side operators and the attribution path together."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_policy_example_learns_and_finds_its_own_answers():
    path = os.path.join(ROOT, "examples", "attribute_policy_step.py")
    spec = importlib.util.spec_from_file_location("attribute_policy_step", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    out = mod.main()
    assert out["policy"][-1] < out["policy"][0] and np.isfinite(out["policy"]).all()
    assert abs(out["preference"][0] - np.log(2)) < 1e-5        # the reference is the policy itself
    assert out["preference"][-1] < 0.8 * out["preference"][0]
    # an answer's own gradient is its nearest row, at a cosine of 1 within fp16
    assert out["index"][:, 0].tolist() == list(range(mod.B))
    assert np.abs(out["scores"][:, 0].numpy() - 1).max() < 1e-3
