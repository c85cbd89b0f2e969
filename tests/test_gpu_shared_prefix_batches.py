"""Decoding behind shared prefixes: what a sequence gets does not hang on how many others there are, nor on how they share out over runs.

Tolerances, derived before the first run.  The 32-bit terms of tests/test_gpu_shared_prefix.py: (2 (D + 4) spread + 2 n + 64) u size.  bf16:
weights go to the matrix pipe in two pieces, each rounded by half a step at most, 2^-8 of 2^-8: 2^-16 size in the numerator and as much in the
denominator, and the result is rounded once, 2^-8 |out| (1 + 2^-8 for the distance between what is rounded and the definition)."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_shared_prefix import B8, U, Batch, c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


def check(b, out, scale=None, window=0, sinks=0, rows=None):
    scale = b.D ** -0.5 if scale is None else scale
    q, got = b.q.double().cpu().numpy(), out.double().cpu().numpy()
    for i in range(len(b.lens)) if rows is None else rows:
        k, v = b.keys[i]
        ref, size, spread = oa.attention(q[i:i + 1], k, v, b.lens[i] - 1, scale, window, sinks)
        tol = (2 * (b.D + 4) * spread + 2 * len(k) + 64) * U * size + 1e-37
        if b.dtype == "bf16":
            tol = tol + 2 * B8 * B8 * size + B8 * (1 + B8) * np.abs(ref)
        err = np.abs(got[i] - ref[0])
        assert (err <= tol[0]).all(), (i, float((err / tol[0]).max()))


@pytest.mark.parametrize("D,H,Hkv,page", [(128, 2, 2, 16), (128, 7, 1, 24), (64, 4, 2, 64), (64, 1, 1, 1)])
@pytest.mark.parametrize("n", [2, 16, 17, 40, 130])
def test_weights_of_a_prefix_keep_both_pieces(c2r, D, H, Hkv, page, n):  # noqa: F811
    b = Batch(c2r, "bf16", D, H, Hkv, page, [n], [900], [1 + 7 * i % 50 for i in range(n)], seed=n + D)
    rows = sorted({0, 1, n // 2, n - 1})
    check(b, b.run(max_shared_len=900, max_own_len=50), rows=rows)
    check(b, b.run(window=400, sinks=5), window=400, sinks=5, rows=rows)
    check(b, b.run(scale=-0.1), scale=-0.1, rows=rows)
    check(b, b.run(scale=0.0), scale=0.0, rows=rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sizes,before,after", [
    ([128] + [1] * 8, 0, 0),            # one long run among single sequences: the mean is below 16 rows of a key head
    ([2], 70, 30),                      # a run of two beside a hundred sequences of no run: the mean is far above
    ([1, 60, 0, 1, 1], 3, 9),
    ([40] + [1] * 70, 1, 1),            # more runs than a wave has lanes
])
def test_skewed_runs(c2r, dtype, D, sizes, before, after):  # noqa: F811
    n = before + sum(sizes) + after
    prefix = [700 if s > 1 else 30 + i for i, s in enumerate(sizes)]
    b = Batch(c2r, dtype, D, 2, 2, 16, sizes, prefix, [1 + 11 * i % 60 for i in range(n)], before=before, after=after, seed=n)
    first = int(b.start[0])
    rows = sorted({0, first, first + 1, first + sum(sizes) // 2, first + sum(sizes) - 1, n - 1})
    check(b, b.run(max_shared_len=700, max_own_len=60), rows=rows)
    check(b, b.run(window=100, sinks=9), window=100, sinks=9, rows=rows)
