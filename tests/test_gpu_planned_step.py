"""The example of a training step at planned addresses: same losses, norms and weights to the last bit as with buffers of their own, in a
pool as large as the plan says."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("more", [dict(layers=2, hidden=256, heads=4, kv_heads=2, head_dim=64, vocabulary=1000, tokens=333, sequences=4),
                                  dict(layers=1, hidden=512, heads=4, kv_heads=4, head_dim=128, vocabulary=5003, tokens=512, sequences=1)], ids=["grouped", "one"])
def test_planned_step(more):
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    spec = importlib.util.spec_from_file_location("planned_step", os.path.join(ROOT, "examples", "planned_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    c = example.config(**more)
    r = example.run(c, steps=4)
    assert int(c.status.item()) == 0
    assert r["losses"][0] == r["losses"][1] and r["norms"][0] == r["norms"][1] and r["same"]
    assert r["losses"][0][-1] < r["losses"][0][0]
    assert r["bound"] <= r["extent"] <= 1.05 * r["bound"] and r["extent"] < r["sum"]
