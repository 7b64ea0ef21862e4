"""The example of a policy update runs end to end: the sampled trees' rewarded tokens become likelier, and the
distillation loss falls with every step."""
import importlib.util
import os

import pytest

from conftest import ROOT
from test_gpu_parity import _built  # noqa: F401

pytestmark = pytest.mark.gpu


def test_policy_step_example():
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    even, kl = mod.main(steps=6)
    assert len(even) == 6 and all(0 <= x <= 1 for x in even)
    assert even[-1] > even[0] + 0.02
    assert all(b < a for a, b in zip(kl, kl[1:]))
