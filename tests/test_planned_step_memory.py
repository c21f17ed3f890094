"""The example's Memory at planned addresses: a workspace that turns out larger than its place in the plan is an error, not a tensor from elsewhere.  No GPU is needed."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("planned_step", os.path.join(ROOT, "examples", "planned_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_workspaces_are_where_the_plan_says(example):
    import torch
    import paper_2507_16274_amd as S
    memory = example.Memory(torch.empty(2048, dtype=torch.uint8), [512, 1024])
    memory.sizes = [512, 512]

    def operator(need, *, workspace_cache):
        return {"workspace": S._workspace(need, "cpu", workspace_cache)}

    out = memory.call(operator, 500)
    assert out["workspace"].data_ptr() == memory.pool.data_ptr() + 512
    with pytest.raises(MemoryError):
        memory.call(operator, 600)
