"""Calls large enough to pass by the caches, sampled rows against the definitions in 64 bits (oracle/serving.py); tolerances are those of
the operators' own tests."""
import numpy as np
import pytest
import torch

from oracle import serving as osv
from test_gpu_adapters import B8, U, _np, _random_ids
from test_gpu_logprobs import _check, c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "e4m3": torch.bfloat16, "f32": torch.float32}


# 32 MB of results or more; 16 rows to a tile below 48 rows for each adapter and for those without
@pytest.mark.parametrize("kind,T,d_out,r,n", [
    ("bf16", 2100, 8200, 64, 5), ("bf16", 2100, 8200, 64, 60), ("bf16", 4100, 4104, 128, 3), ("bf16", 4100, 4104, 128, 200), ("bf16", 2100, 8200, 24, 60),
    ("e4m3", 2100, 8200, 64, 5), ("e4m3", 4100, 4104, 128, 200), ("f32", 2100, 4104, 16, 5), ("f32", 2100, 4104, 16, 60), ("f32", 1030, 8200, 64, 4),
    ("f32", 1030, 8200, 64, 60), ("f32", 1030, 8200, 128, 4), ("f32", 1030, 8200, 128, 60)])
def test_adapters(c2r, kind, T, d_out, r, n):  # noqa: F811
    d_in, dt = 264, DT[kind]
    assert T * d_out * dt.itemsize >= 32 << 20 and (T >= 48 * (n + 1)) == (n < 10)
    g = torch.Generator(device="cuda").manual_seed(T + r + n)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, x_scale = rnd(T, d_in), None
    if kind == "e4m3":
        x_scale = x.abs().amax(1) / 448
        x = (x / x_scale[:, None]).to(torch.float8_e4m3fn)
    else:
        x = x.to(dt)
    A, B, y = (rnd(n, r, d_in) * d_in ** -0.5).to(dt), rnd(n, d_out, r).to(dt), rnd(T, d_out).to(dt)
    scale = torch.rand(n, generator=g, device="cuda") * 2 - 1
    ids = _random_ids(T, T, n)
    out = c2r.adapters(x, torch.from_numpy(ids).int().cuda(), A, B, y, scale, x_scale)
    rows = np.unique(np.r_[0:20, T // 2:T // 2 + 20, T - 20:T])
    values = _np(x[rows].float()) * (1 if x_scale is None else _np(x_scale[rows])[:, None])
    ref, size = osv.adapters(values, ids[rows], _np(A), _np(B), _np(y[rows]), _np(scale))
    tol = (d_in + r + 8) * U * size + U * np.abs(ref)
    if kind != "f32":
        tol = tol + 2.0 ** -16 * size + B8 * np.abs(ref)
    err = np.abs(_np(out[rows]) - ref)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())
    none = torch.from_numpy(ids < 0).cuda()
    assert torch.equal(out[none], y[none])
    y_there = y.clone()
    assert torch.equal(c2r.adapters(x, torch.from_numpy(ids).int().cuda(), A, B, y_there, scale, x_scale, out=y_there), out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,n", [(40003, 20), (160000, 1), (160001, 64)])
def test_logprobs(c2r, dtype, V, n):  # noqa: F811
    T = (128 << 20) // (V * dtype.itemsize) + 3
    g = torch.Generator(device="cuda").manual_seed(V + n)
    l = torch.empty((T, V), dtype=dtype, device="cuda").normal_(generator=g).mul_(2.5)
    tokens = torch.randint(0, V, (T, 2), generator=g, dtype=torch.int32, device="cuda")
    lp, ent, top, top_lp = c2r.token_logprobs(l, tokens, n)
    for rows in (slice(0, 2), slice(T // 2, T // 2 + 3), slice(T - 2, T)):
        # a call of these rows alone against the definition, then the large one against that: the same tokens, and sums of V / 256 + 64 terms
        # in another order on either side, 2 (4 * 30 + V / 256 + 64) u
        few = l[rows].clone()
        _check(c2r, few, n_top=n)
        ref = c2r.token_logprobs(few, tokens[rows].contiguous(), n)
        assert torch.equal(top[rows], ref[2])
        for a, b in ((lp[rows], ref[0]), (ent[rows], ref[1]), (top_lp[rows], ref[3])):
            assert ((a - b).abs() <= 2 * (4 * 30 + V / 256 + 64) * U * (1 + 2 * 12)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(2050, 8200), (600, 32768), (4200, 4096), (70000, 256)])
def test_norm(c2r, dtype, T, d):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(T + d)
    x, res = (torch.randn((T, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    w = 1 + 0.2 * torch.randn(d, generator=g, device="cuda")
    assert T * d * dtype.itemsize >= 32 << 20
    y, s, y8, c = c2r.add_rms_norm(x, res, w, bits8=True)
    assert torch.equal(s, x + res)                              # one rounding of a sum either way
    for i in (0, 1, T // 2, T - 2, T - 1):
        ref = osv.rms_norm(_np(s[i:i + 1]), _np(w), 1e-6)[0]
        size = np.abs(ref)
        # d squares added up: (d + 8) u of their sum, half of it in its root; four more roundings
        tol = ((d + 8) / 2 + 8) * U * size
        assert (np.abs(_np(y[i]) - ref) <= tol + (B8 if dtype is torch.bfloat16 else U) * size + 1e-37).all()
        most = size.max() / 448
        assert abs(float(c[i]) - most) <= ((d + 8) / 2 + 12) * U * most
        # (e4m3: half a step is 2^-4 of a value, and 2^-10 below the least normal number, 2^-6)
        back = _np(y8[i].float()) * float(c[i])
        assert (np.abs(back - ref) <= 2.0 ** -4 * size + 2.0 ** -10 * most + 4 * ((d + 8) / 2 + 16) * U * size).all()
