"""The example of the operators around the actor step runs as it stands and learns."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_warm_start_and_grpo():
    spec = importlib.util.spec_from_file_location("warm_start_and_grpo", os.path.join(ROOT, "examples", "warm_start_and_grpo.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, report = example.main(["--warm-steps", "30", "--grpo-steps", "2"])
    # 256 tokens, so log 256 = 5.5 at best without learning anything
    assert losses[0] > 4.0 and losses[-1] < 0.5 * losses[0], losses
    for r in report:
        assert all(np.isfinite(v) for v in r.values()), r
        # the policy that made the rollouts is the one that is updated: ratios are one up to bf16 rounding of two forward passes
        assert abs(r["ratio"] - 1.0) < 0.05, r
        assert 0.0 < r["entropy"] < np.log(256) and 0.0 <= r["among_four"] <= 1.0
