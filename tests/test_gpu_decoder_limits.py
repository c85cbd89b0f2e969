"""What the example's decoder stack refuses, and what it keeps."""
import pytest
import torch

from paper_2504_01337_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2504_01337_amd.examples.decoder_block import DecoderBlock
    return DecoderBlock(wl.WORKLOADS["C1"], 4, 2, 64)


def test_rows_past_the_caches_are_refused(block):
    """A page of 16 slots holds more than max_len rows: the limit is max_len, and what was refused has changed nothing."""
    from paper_2504_01337_amd.examples.decoder_block import Decoder
    d = block.w.d
    dec = Decoder([block], 2, 20, page_size=16)
    x = torch.randn(41, d, generator=torch.Generator().manual_seed(1)).cuda()
    for bad in ([21, 3], [3, 21], [3], [3, -1]):
        with pytest.raises(ValueError):
            dec.prompt(x[:sum(bad)], bad)
    assert not dec.kv_len.any()
    dec.prompt(x[:19], [18, 1])
    with pytest.raises(ValueError):
        dec.prompt(x[:3], [3, 0])
    dec.step(x[:2])
    dec.step(x[:2])
    keys = dec.caches[0].k.clone()
    with pytest.raises(ValueError):
        dec.step(x[:2])
    assert dec.kv_len.tolist() == [20, 3] and torch.equal(dec.caches[0].k.nan_to_num(), keys.nan_to_num())
    dec.reset()
    dec.prompt(x[:40], [20, 20])
    assert dec.kv_len.tolist() == [20, 20]


def test_layers_of_few_row_counts_are_kept(block):
    """Prompts of many lengths between the steps: the steps' layer stays, and rows come out as from a layer made for them."""
    from paper_2504_01337_amd.examples.decoder_block import Decoder
    d = block.w.d
    x = torch.randn(40, d, generator=torch.Generator().manual_seed(2)).cuda()
    dec = Decoder([block], 2, 400, page_size=16)
    steps = None
    for n in range(3, 20):
        dec.prompt(x[:n], [n - 1, 1])
        dec.step(x[:2])
        assert steps is None or block.moe[2] is steps
        steps = block.moe[2]
        assert len(block.moe) <= 4 and n in block.moe
    dec.reset()
    first = dec.prompt(x[:3], [2, 1]).clone()
    for n in range(20, 30):
        dec.prompt(x[:n], [n, 0])
    dec.reset()
    assert torch.equal(dec.prompt(x[:3], [2, 1]), first)
