"""Calls around the blocks' halves on no rows at all."""
import pytest
import torch

from test_gpu_row_norm import c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm(c2r, dtype):  # noqa: F811
    x = torch.randn(4, 64, device="cuda").to(dtype)[:0]
    for kw in (dict(), dict(bits8=True), dict(bits8=True, dense=False)):
        for residual in (None, x):
            y, total, y8, scale = c2r.add_rms_norm(x, residual, **kw)
            assert (y is None) == (kw.get("dense") is False) and (y is None or y.shape == (0, 64))
            assert (total is None) == (residual is None) and (total is None or total.shape == (0, 64))
            assert not kw or (y8.shape == (0, 64) and scale.shape == (0,))
