"""How the binding calls an operator with a workspace at hand: one call, whatever it returns; the workspace's size is only asked for where that can be the reason of a refusal.
(An operator that works in place and is called twice differentiates its own result.)  No GPU is needed: the library is a stand-in."""
import ctypes

import pytest


@pytest.fixture
def S(monkeypatch):
    import paper_2507_16274_amd as S
    monkeypatch.setattr(S, "_stream", lambda stream: None)
    return S


class Library:
    """A call that needs `need` bytes and returns `rc` where it has them."""

    def __init__(self, rc, need):
        self.rc, self.need, self.worked = rc, need, 0

    def __call__(self, workspace, nbytes, stream):
        size = ctypes.cast(nbytes, ctypes.POINTER(ctypes.c_size_t))[0]
        if workspace is None:
            ctypes.cast(nbytes, ctypes.POINTER(ctypes.c_size_t))[0] = self.need
            return 0
        if size < self.need:
            return 1
        if self.rc != 1:
            self.worked += 1
        rc, self.rc = self.rc, 0
        return rc


def _call(S, fn, cache):
    import torch
    return S._call(fn, "operator", (), torch.empty(1), None, cache, {})


@pytest.mark.parametrize("rc", [5, 9])
def test_an_error_is_raised_and_nothing_is_repeated(S, rc):
    import torch
    fn = Library(rc, 512)
    with pytest.raises(S.StallocError, match=S.STATUS[rc]):
        _call(S, fn, {"ws": torch.empty(512, dtype=torch.uint8)})
    assert fn.worked == 1


def test_a_refusal_that_the_workspace_is_not_the_reason_of(S):
    import torch
    fn, ws = Library(1, 512), torch.empty(512, dtype=torch.uint8)
    with pytest.raises(S.StallocError, match="STALLOC_ERR_INVALID_ARG"):
        _call(S, fn, {"ws": ws})
    assert fn.worked == 0


def test_workspaces_grow_and_stay(S):
    import torch
    cache = {"ws": torch.empty(256, dtype=torch.uint8)}
    fn = Library(0, 1000)
    out = _call(S, fn, cache)
    assert fn.worked == 1 and out["workspace"] is cache["ws"] and cache["ws"].numel() >= 1000
    kept = cache["ws"]
    assert _call(S, fn, cache)["workspace"] is kept and fn.worked == 2
    assert _call(S, fn, None)["workspace"].numel() >= 1000 and fn.worked == 3
