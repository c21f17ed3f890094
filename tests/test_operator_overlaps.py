"""Norms whose output takes the place of an input: refused where the input's rows are not as far apart as the output's, since rows that are still to be read would be written.
No GPU is needed."""
import ctypes

import pytest

INVALID = 1


@pytest.fixture(scope="module")
def S():
    import paper_2507_16274_amd as S
    return S


@pytest.mark.parametrize("x,residual,total,x_stride,residual_stride", [(512, 1024, 512, 108, 100), (512, 1024, 1024, 100, 108), (512, 1024, 512, 0, 100),
                                                                       (512, 1024, 1024, 100, 0), (512, None, 512, 108, 0)])
def test_forward(S, x, residual, total, x_stride, residual_stride):
    assert S.lib.stalloc_rms_norm(1, 4, 100, x, x_stride, residual, residual_stride, 256, 1e-6, total, 2048, None, None, 256, None) == INVALID


@pytest.mark.parametrize("stride", [0, 99, 108, 200])
def test_backward(S, stride):
    have = ctypes.c_size_t(1 << 40)
    assert S.lib.stalloc_rms_norm_backward(1, 4, 100, 512, stride, 256, 256, 256, None, 512, 256, 256, ctypes.byref(have), None) == INVALID
