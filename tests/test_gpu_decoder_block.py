"""The operators together, as the example's decoder stack runs them: prompts, then a token at a time."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2504_01337_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_prompts_then_tokens(window, sinks):
    """What a token gives does not depend on whether it came in a prompt, in its second part or alone.  fp32: each block's rows
    differ by roundings of sums over 512 terms at most, 2^-24 * 512 = 3e-5 of a value, two blocks of two sums each; 2^-11 = 16 times
    that is far below what a token that saw a wrong row would differ by."""
    from paper_2504_01337_amd.examples.decoder_block import Decoder, DecoderBlock
    w = wl.WORKLOADS["C1"]
    blocks = [DecoderBlock(w, 4, 2, 64, window, sinks, seed=i) for i in range(2)]
    lengths = [90, 1, 33]
    x = torch.randn(sum(lengths), w.d, generator=torch.Generator().manual_seed(3)).cuda()
    at = np.concatenate([[0], np.cumsum(lengths)])
    whole = Decoder(blocks, 3, 100).prompt(x, lengths)

    dec = Decoder(blocks, 3, 100, page_size=16)
    parts = [[50, 0, 20], [20, 1, 0]]
    got = [[], [], []]
    seen = [0, 0, 0]

    def rows(take):
        return torch.cat([x[at[b] + seen[b]:at[b] + seen[b] + n] for b, n in enumerate(take)])
    for take in parts:
        y = dec.prompt(rows(take), take).split(take)
        for b in range(3):
            got[b].append(y[b])
            seen[b] += take[b]
    for _ in range(13):                          # single tokens; the second sequence has ended, its rows count for nothing
        xs = torch.stack([x[min(at[b] + seen[b], at[b + 1] - 1)] for b in range(3)])
        y = dec.step(xs)
        for b in (0, 2):
            got[b].append(y[b:b + 1])
            seen[b] += 1
    for b in range(3):
        g = torch.cat(got[b])
        ref = whole[at[b]:at[b] + len(g)]
        assert len(g) == (83, 1, 33)[b]
        assert (g - ref).abs().max() <= 2.0 ** -11 * ref.abs().max(), b


def test_block_attention_against_the_definition():
    """One block with its experts' part taken off: rows against 64 bits, from the projection on."""
    from paper_2504_01337_amd.examples.decoder_block import Decoder, DecoderBlock, rms_norm
    w = wl.WORKLOADS["C1"]
    H, Hkv, D, lengths = 4, 2, 64, [70, 5]
    block = DecoderBlock(w, H, Hkv, D, 20, 2)
    x = torch.randn(sum(lengths), w.d, generator=torch.Generator().manual_seed(4)).cuda()
    T = len(x)
    y = Decoder([block], 2, 80).prompt(x, lengths)
    with_attention = y - block.moe[T].y
    qkv = torch.nn.functional.linear(rms_norm(x), block.w_qkv).view(T, H + 2 * Hkv, D).double().cpu().numpy()
    pos = np.concatenate([np.arange(n) for n in lengths])
    f, wq, wk = (t.cpu().numpy() for t in (block.inv_freq, block.q_weight, block.k_weight))
    q, _ = oa.norm_rope(qkv[:, :H], wq, 1e-6, f, pos, False)
    k, _ = oa.norm_rope(qkv[:, H:H + Hkv], wk, 1e-6, f, pos, False)
    v, out, at = qkv[:, H + Hkv:], [], 0
    for n in lengths:
        s = slice(at, at + n)
        out.append(oa.attention(q[s], k[s], v[s], 0, D ** -0.5, 20, 2)[0])
        at += n
    ref = x.double().cpu().numpy() + np.concatenate(out).reshape(T, H * D) @ block.w_o.double().cpu().numpy().T
    # fp32 sums of 256 terms in the output product (2^-24 * 256), and as much again for each of rows, scores and weights
    assert np.abs(with_attention.double().cpu().numpy() - ref).max() <= 4 * 2.0 ** -16 * np.abs(ref).max()
