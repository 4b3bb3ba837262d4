"""The example that trains two replicas, from norm and step to repair, restore
and 8-bit moments, does what its text says."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_replica_training():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("replica_training", os.path.join(ROOT, "examples", "replica_training.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    steps = 12
    seen = mod.main(steps)
    flagged = seen["flagged"]
    # nothing differs but in the step after the flip, and there few chunks do: the second moment's, and where the
    # update has reached them the master's and the parameter's
    assert [i for i, n in enumerate(flagged) if n] == [steps // 2 - 1]
    assert 1 <= flagged[steps // 2 - 1] <= 3
    assert seen["differing_after_repair"] == 0 and seen["restored_bad"] == 0 and seen["form8_differs"] == 0
    loss = seen["losses"]
    assert all(b < a for a, b in zip(loss, loss[1:])), loss
