"""Low-rank adapters on the GPU against the definition in 64 bits (oracle/serving.py).

Tolerances, derived before the first run.  u = 2^-24, size = |c| sum |B| sum |A| |x|.  A x: d_in products and additions in 32 bits,
scaled once or twice; B h: rank of them; y added once: (d_in + rank + 8) u size + u |out|.  bf16: h goes to the second product in two
pieces, 2^-16 size, and the result is rounded, 2^-8 |out|."""
import numpy as np
import pytest
import torch

from oracle import serving as osv

pytestmark = pytest.mark.gpu

U, B8 = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "e4m3": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _np(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, kind, T, d_in, d_out, r, n, ids, seed=0, pad=0, scaled=True):
        g = torch.Generator().manual_seed(seed)
        dt = DT[kind]
        rnd = lambda *s, dtype=dt: torch.randn(*s, generator=g).to(dtype).cuda()
        x = torch.randn(T, d_in + pad, generator=g)
        self.kind, self.d_in, self.r, self.x_scale = kind, d_in, r, None
        if kind == "e4m3":
            self.x_scale = (x.abs().amax(1) / 448).cuda() if T else torch.empty(0, device="cuda")
            self.x = (x.cuda() / self.x_scale[:, None]).to(torch.float8_e4m3fn)[:, :d_in]
            self.values = _np(self.x.float()) * _np(self.x_scale)[:, None]
        else:
            self.x = x.to(dt).cuda()[:, :d_in]
            self.values = _np(self.x)
        self.A, self.B, self.y = rnd(n, r, d_in) * d_in ** -0.5, rnd(n, d_out, r), rnd(T, d_out + pad)[:, :d_out]
        self.scale = (torch.rand(n, generator=g) * 2 - 1).cuda() if scaled else None
        self.ids = torch.tensor(ids, dtype=torch.int32, device="cuda")

    def run(self, c2r, **kw):
        return c2r.adapters(self.x, self.ids, self.A, self.B, self.y, self.scale, self.x_scale, **kw)

    def check(self, out):
        ids = self.ids.cpu().numpy()
        ref, size = osv.adapters(self.values, ids, _np(self.A), _np(self.B), _np(self.y), None if self.scale is None else _np(self.scale))
        tol = (self.d_in + self.r + 8) * U * size + U * np.abs(ref)
        if self.kind != "f32":
            tol = tol + 2.0 ** -16 * size + B8 * np.abs(ref)
        err = np.abs(_np(out) - ref)
        assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())
        none = ~((ids >= 0) & (ids < len(self.A)))
        assert torch.equal(out[torch.from_numpy(none)], self.y[torch.from_numpy(none)])


def _random_ids(seed, T, n, none=0.2):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, n, T)
    ids[rng.random(T) < none] = -1
    return ids


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("T,d_in,d_out,r,n", [
    (1, 8, 8, 8, 1), (1, 2048, 520, 16, 8), (2, 64, 256, 24, 3), (17, 136, 264, 8, 2), (33, 520, 1000, 64, 5), (16, 1032, 248, 128, 1),
    (64, 72, 776, 40, 64), (131, 4096, 320, 64, 20), (100, 600, 512, 96, 1), (300, 256, 512, 16, 5), (700, 200, 264, 32, 3),
    (520, 1024, 72, 48, 4), (257, 96, 128, 120, 1)])
def test_random_rows(c2r, kind, T, d_in, d_out, r, n):
    c = Case(kind, T, d_in, d_out, r, n, _random_ids(T, T, n), seed=T + r, pad=16)
    keep = c.y.clone()
    out = c.run(c2r)
    assert torch.equal(c.y, keep)
    c.check(out)
    # in the place of y, the same bits
    got = c.run(c2r, out=c.y)
    assert got is c.y and torch.equal(got, out)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("runs", [[0] * 200, [1] * 63 + [0], [2] * 64 + [-1] * 65 + [2] * 64 + [0], [-1] * 130, [5] * 3 + [-7, 99, 3] * 40,
                                  list(range(150)) * 2])
def test_runs_and_rows_without(c2r, kind, runs):
    """Requests' rows side by side, adapters that no row has, ids outside the range, all rows without."""
    c = Case(kind, len(runs), 264, 312, 16, 150, runs, seed=len(runs), scaled=False)
    c.check(c.run(c2r))


def test_many_adapters_of_one_row(c2r):
    c = Case("bf16", 1024, 64, 64, 8, 1024, np.random.default_rng(3).permutation(1024), seed=5)
    c.check(c.run(c2r))


@pytest.mark.parametrize("T,n", [(257, 255), (257, 256), (1000, 3), (2048, 7), (2049, 7), (9000, 2), (17000, 5), (5000, 1000)])
@pytest.mark.parametrize("each", [1, 150])
def test_many_rows(c2r, T, n, each):
    """Either way in which rows find their places: all rows once, requests of a row or of many, some rows without."""
    rng = np.random.default_rng(T + n)
    ids = np.repeat(rng.integers(-1, n, -(-T // each)), each)[:T]
    c = Case("bf16", T, 64, 32, 8, n, ids, seed=T)
    c.check(c.run(c2r))
    keep = c.y.clone()
    out = c.run(c2r)
    c.y = keep.clone()
    assert torch.equal(c.run(c2r, out=c.y), out)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_row_alone_and_among_others(c2r, kind):
    """What a row gets is within the tolerance whatever rows stand beside it, NaN and infinities in others and in other adapters included."""
    c = Case(kind, 80, 512, 256, 32, 4, [i % 4 for i in range(80)], seed=9)
    ref = c.run(c2r)
    c.check(ref)
    if kind == "bf16":
        c.x[7, 3], c.x[40, 100] = float("nan"), float("inf")
    else:
        c.x_scale[7], c.x_scale[40] = float("nan"), float("inf")
    c.A[3] = float("nan")
    out = c.run(c2r)
    bad = torch.tensor([i in (7, 40) or i % 4 == 3 for i in range(80)])
    assert torch.equal(out[~bad], ref[~bad])
    assert not torch.isfinite(out[bad]).any(1).all()


def test_zero_rows_and_none(c2r):
    c = Case("bf16", 0, 64, 64, 8, 2, [])
    assert c.run(c2r).shape == (0, 64)


def test_rows_around_the_output_stay(c2r):
    c = Case("bf16", 21, 128, 200, 16, 3, _random_ids(1, 21, 3))
    whole = torch.full((23, 216), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[1:-1, :200]
    c.run(c2r, out=out)
    c.check(out)
    assert (whole[0] == 7).all() and (whole[-1] == 7).all() and (whole[:, 200:] == 7).all()


def test_the_same_bits_every_time_two_streams_and_a_graph(c2r):
    c = Case("bf16", 400, 1024, 512, 16, 6, _random_ids(2, 400, 6))
    ref = c.run(c2r)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(12):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(c.run(c2r))
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    g, out = torch.cuda.CUDAGraph(), torch.empty_like(ref)
    ws = torch.empty(c2r.workspace_bytes(c2r.STAGE_ADAPTERS, 400, 1024, 6, 16, 0, c2r.BF16), dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(g):
        c.run(c2r, out=out, ws=ws)
    for k in range(3):
        c.ids.copy_(torch.from_numpy(_random_ids(10 + k, 400, 6)))
        ws.fill_(255)                                       # (what an earlier call left there says nothing)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.run(c2r))
        c.check(out)
