"""The example of a training step says so when a batch is wrong: a target beyond the vocabulary, boundaries that descend."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("what,status", [("targets", "BAD_TOKEN"), ("bounds", "BAD_BOUNDS")])
def test_wrong_batches(what, status):
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    spec = importlib.util.spec_from_file_location("planned_step", os.path.join(ROOT, "examples", "planned_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    c = example.config(layers=1, hidden=256, heads=4, kv_heads=2, head_dim=64, vocabulary=1000, tokens=333, sequences=4)
    batch = example.make_batch(c)
    if what == "targets":
        batch["targets"][7] = 1000
    else:
        batch["bounds"][1] = 334
    with pytest.raises(S.StallocError, match=status):
        example.run(c, steps=1, batch=batch)
