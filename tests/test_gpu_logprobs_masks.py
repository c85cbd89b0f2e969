"""Log probabilities of rows whose mask is a finite number and leaves fewer tokens than are asked for: the places behind them are masked
tokens, the lowest indices first.  Tolerances are those of tests/test_gpu_logprobs.py."""
import pytest
import torch

from test_gpu_logprobs import _check, c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(1, 40000), (3, 5003), (1100, 5003)])
@pytest.mark.parametrize("keep", [0, 1, 10])
@pytest.mark.parametrize("mask", ["lowest", -1e9, -30000.0])
def test_fewer_than_are_asked_for(c2r, dtype, T, V, keep, mask):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(keep + V)
    row = torch.randn((3, V), generator=g, device="cuda").to(dtype)
    gone = torch.rand((3, V), generator=g, device="cuda").argsort(1) >= keep
    row = row.masked_fill(gone, torch.finfo(dtype).min if mask == "lowest" else mask)
    l = row[torch.arange(T, device="cuda") % 3].contiguous()
    _check(c2r, l, n_top=20)                 # (1100 rows: a block to a whole row)
    _check(c2r, l[:3], n_top=1, given=1)
