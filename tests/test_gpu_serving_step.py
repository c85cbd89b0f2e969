"""The operators around the blocks' halves together, as the example's decoder stack runs them for many requests at once."""
import pytest
import torch

from oracle import serving as osv
from paper_2504_01337_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _merged(block, k):
    """Both projections with adapter k added to their weights (k < 0: as they are)."""
    if k < 0:
        return block.w_qkv, block.w_o
    (Aq, Bq), (Ao, Bo), c = block.adapters
    return block.w_qkv + c[k] * (Bq[k] @ Aq[k]), block.w_o + c[k] * (Bo[k] @ Ao[k])


@pytest.mark.parametrize("window,sinks,n", [(0, 0, 3), (30, 2, 3), (0, 0, 40)])
def test_requests_with_adapters_behind_a_common_prompt(window, sinks, n):
    """Sequences that share a prompt and have adapters of their own, all in one batch, against each alone: the whole prompt as its own rows
    and its adapter merged into the weights.  fp32: sums of 256 to 512 terms in another order, 2^-24 * 512 = 3e-5 of a value in each of two
    blocks' two sums, as in the test of prompts and single tokens; 2^-11 is 16 times that."""
    from paper_2504_01337_amd.examples.decoder_block import Decoder, DecoderBlock
    w = wl.WORKLOADS["C1"]
    blocks = [DecoderBlock(w, 4, 2, 64, window, sinks, seed=i) for i in range(2)]
    for i, b in enumerate(blocks):
        b.add_adapters(3, 8, 0.3, seed=i)
    gen = torch.Generator().manual_seed(n)
    common, fresh, steps = torch.randn(70, w.d, generator=gen).cuda(), [1 + i % 3 for i in range(n)], 3
    rows = [torch.randn(f + steps, w.d, generator=gen).cuda() for f in fresh]
    ids = [(i % 4) - 1 for i in range(n)]
    dec = Decoder(blocks, n, 100, page_size=16, adapter=torch.tensor(ids, dtype=torch.int32).cuda(), vocab=501)
    first = dec.share(common)
    got = list(dec.prompt(torch.cat([r[:f] for r, f in zip(rows, fresh)]), fresh).split(fresh))
    for s in range(steps):
        y = dec.step(torch.stack([r[f + s] for r, f in zip(rows, fresh)]))
        got = [torch.cat([g, y[b:b + 1]]) for b, g in enumerate(got)]
    plain = [(b.w_qkv, b.w_o) for b in blocks]
    for k in sorted(set(ids)):
        mine = [b for b in range(n) if ids[b] == k][:2]
        # the common prompt has no adapter: its rows first, then the rest with the merged weights
        alone = Decoder(blocks, len(mine), 100, page_size=16)
        x = alone.prompt(common.repeat(len(mine), 1), [70] * len(mine))
        assert (x[:70] - first).abs().max() <= 2.0 ** -11 * first.abs().max()
        for b in blocks:
            b.w_qkv, b.w_o = _merged(b, k)
        ref = alone.prompt(torch.cat([rows[b] for b in mine]), [len(rows[b]) for b in mine]).split([len(rows[b]) for b in mine])
        for b, p in zip(blocks, plain):
            b.w_qkv, b.w_o = p
        for b, r in zip(mine, ref):
            assert (got[b] - r).abs().max() <= 2.0 ** -11 * r.abs().max(), (b, k)
    # what is answered, scored: 2^-11 of a row's norm, 16 = sqrt(256), at most moves a logit by 2^-11 * 16 * |row of the head| = 2^-7
    last = torch.cat([g[-1:] for g in got])
    tokens = torch.randint(0, 501, (n, 2), generator=gen, dtype=torch.int32).cuda()
    lp, ent, top, top_lp = dec.logprobs(last, tokens, 4)
    h = osv.rms_norm(last.double().cpu().numpy(), None, 1e-6)
    logits = h @ dec.head.double().cpu().numpy().T
    for b in range(n):
        ref, H, _, _ = osv.logprobs(logits[b])
        # products of 256 terms and the norm's (256 / 2 + 8) roundings: 2^-24 * 400 * sum |h| |head| < 2^-24 * 400 * 16 * 1.4 < 2^-10
        assert abs(ref[tokens[b].cpu().numpy()] - lp[b].double().cpu().numpy()).max() <= 2.0 ** -10
        assert abs(H - float(ent[b])) <= 2.0 ** -8
        assert abs(ref[top[b].cpu().numpy()] - top_lp[b].double().cpu().numpy()).max() <= 2.0 ** -10
        assert float(top_lp[b, 0]) >= ref.max() - 2.0 ** -10
    # the pages are everyone's own again
    dec.reset()
    again = dec.prompt(torch.cat([common, rows[0][:fresh[0]]]), [70 + fresh[0]] + [0] * (n - 1))
    if ids[0] < 0:
        assert (again[70:] - got[0][:fresh[0]]).abs().max() <= 2.0 ** -11 * again.abs().max()


def test_rows_in_8_bits_from_the_norm_to_the_adapters():
    """The norm's rows in e4m3 are what the adapters take: the definition on the values that they stand for, in the tolerance of
    tests/test_gpu_adapters.py."""
    import numpy as np
    from paper_2504_01337_amd import c2r
    g = torch.Generator().manual_seed(1)
    T, d, d_out, r, n = 90, 520, 264, 24, 3
    x, res = (torch.randn(T, d, generator=g).bfloat16().cuda() for _ in range(2))
    A, B = (torch.randn(n, r, d, generator=g) * d ** -0.5).bfloat16().cuda(), torch.randn(n, d_out, r, generator=g).bfloat16().cuda()
    y, ids = torch.randn(T, d_out, generator=g).bfloat16().cuda(), torch.randint(-1, n, (T,), generator=g, dtype=torch.int32).cuda()
    _, _, y8, scale = c2r.add_rms_norm(x, res, dense=False, bits8=True)
    out = c2r.adapters(y8, ids, A, B, y, x_scale=scale).double().cpu().numpy()
    f = lambda t: t.double().cpu().numpy()
    ref, size = osv.adapters(f(y8.float()) * f(scale)[:, None], ids.cpu().numpy(), f(A), f(B), f(y))
    assert (np.abs(out - ref) <= ((d + r + 8) * 2.0 ** -24 + 2.0 ** -16) * size + (2.0 ** -24 + 2.0 ** -8) * np.abs(ref)).all()


def test_the_example_runs():
    import sys
    from paper_2504_01337_amd.examples import decoder_block
    argv, sys.argv = sys.argv, ["decoder_block", "--adapters", "2", "--common", "50", "--vocab", "300", "--prompts", "20", "3", "--steps", "2"]
    try:
        decoder_block.main()
    finally:
        sys.argv = argv
