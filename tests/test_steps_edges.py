"""The client's other steps at the edges of what their calls take: tensors that are refused, the ends of a norm's range,
and the choice of the next token among many rows."""
import ctypes

import numpy as np
import pytest

import steps_plain as plain
from test_attention import Fake
from test_steps import _dev, _host, pv  # noqa: F401


# ---------------------------------------------------------------- rows to write that lie on one another

@pytest.mark.parametrize("token", [0, 1, 7, -1, -7])
def test_overlapping_rows_to_write_are_refused(pv, token):
    """Rows closer than they are long would be written by several threads at once.  (A single row has no other.)"""
    R = pv.pvmvmd_rows(data_dev=64, token=8, scale=1.0, type=pv.PVMVMD_F32)
    good = pv.pvmvmd_rows_out(data_dev=64, token=8, scale=1.0, limit=127, type=pv.PVMVMD_F32)
    r, g = ctypes.byref(R), ctypes.byref(good)
    for kind in (pv.PVMVMD_F32, pv.PVMVMD_FIELD):
        bad = ctypes.byref(pv.pvmvmd_rows_out(data_dev=64, token=token, scale=1.0, limit=127, type=kind))
        assert pv._lib.pvmvmd_block_norm(2, 8, r, None, None, 1.0, r, 1.0, g, None, bad, None) == pv.PVMVMD_E_ARG
        assert pv._lib.pvmvmd_glu(2, 8, r, 3, r, bad, None) == pv.PVMVMD_E_ARG
    bad = ctypes.byref(pv.pvmvmd_rows_out(data_dev=64, token=token, scale=1.0, limit=127, type=pv.PVMVMD_F32))
    assert pv._lib.pvmvmd_block_norm(2, 8, r, None, None, 1.0, r, 1.0, bad, None, g, None) == pv.PVMVMD_E_ARG


@pytest.mark.parametrize("stride", [0, 5, 15])
def test_binding_refuses_overlapping_rows_to_write(pv, stride):
    import torch
    x = Fake((3, 16), torch.float32, address=64)
    bad, good = Fake((3, 16), torch.float32, (stride, 1), 64), Fake((3, 16), torch.float32, address=64)
    for call in (lambda: pv.pvmvmd_block_norm(x, x, residual_out=bad, stream=0),
                 lambda: pv.pvmvmd_block_norm(x, x, residual_out=good, out=bad, stream=0),
                 lambda: pv.pvmvmd_glu(x, out=bad, stream=0)):
        with pytest.raises(ValueError, match="on one another"):
            call()


@pytest.mark.gpu
def test_one_row_to_write_of_any_stride(pv):
    import torch
    x = torch.randn(1, 40, device="cuda")
    for stride in (0, 3):
        out = torch.empty(40, device="cuda").as_strided((1, 40), (stride, 1))
        pv.pvmvmd_glu(x, act="relu", out=out)
        assert torch.equal(out, x.clamp(min=0))
