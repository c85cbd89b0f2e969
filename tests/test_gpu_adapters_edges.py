"""Adapters on the GPU at the edges of their types, against the definition in 64 bits; tolerances are those of tests/test_gpu_adapters.py."""
import numpy as np
import pytest
import torch

from test_gpu_adapters import Case, c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 20, 300])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_product_above_the_largest_of_bf16(c2r, T, sign):  # noqa: F811
    """A x = (2 - 2^-9) 2^127, a number in 32 bits that bf16 would round to an infinity; B takes it back to some 2^8."""
    c = Case("bf16", T, 8, 16, 8, 1, [0] * T, scaled=False)
    c.x.zero_(), c.A.zero_()
    c.x[:, :2] = 2.0 ** 64
    c.A[0, 3, 0], c.A[0, 3, 1] = sign * (2 - 2.0 ** -7) * 2.0 ** 63, sign * 1.5 * 2.0 ** 55
    c.B.fill_(2.0 ** -120)
    c.values = c.x.double().cpu().numpy()
    h = float(c.values[0, :2] @ c.A[0, 3, :2].double().cpu().numpy())
    assert h == sign * (2 - 2.0 ** -9) * 2.0 ** 127
    out = c.run(c2r)
    assert torch.isfinite(out).all()
    c.check(out)


def test_infinite_products_stay_infinite(c2r):  # noqa: F811
    c = Case("bf16", 3, 8, 16, 8, 1, [0] * 3, scaled=False)
    c.x.zero_(), c.A.zero_()
    c.x[0, 0], c.x[1, 0], c.x[2, 0] = float("inf"), float("-inf"), 1.0
    c.A[0, 0, 0] = 1.0
    c.B.fill_(0.5)
    out, h = c.run(c2r).double().cpu().numpy(), np.array([np.inf, -np.inf, 1.0])
    # (the other ranks' rows of A are 0: they give 0 times an infinity, which is no number)
    assert np.isnan(out[:2]).all()
    c.A.fill_(1.0)
    out = c.run(c2r).double().cpu().numpy()
    assert (out[:2] == h[:2, None]).all() and np.isfinite(out[2]).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_every_row_that_is_not_finite(c2r, kind, what):  # noqa: F811
    """A row with a NaN or an infinity, or of an adapter with a NaN in every rank, has no finite result; the others keep theirs."""
    c = Case(kind, 80, 512, 256, 32, 4, [i % 4 for i in range(80)], seed=9)
    ref = c.run(c2r)
    if kind == "e4m3":
        c.x_scale[7], c.x_scale[41] = float(what), float(what)
    else:
        c.x[7, 3], c.x[41, 100] = float(what), -float(what)
    c.A[3, :, 5] = float("nan")
    out = c.run(c2r)
    bad = torch.tensor([i in (7, 41) or i % 4 == 3 for i in range(80)])
    assert torch.equal(out[~bad], ref[~bad])
    assert not torch.isfinite(out[bad]).any()
