"""What the example's decoder stack refuses leaves it as it was (no GPU: refused before any work)."""
import pytest
import torch

from paper_2504_01337_amd.examples.decoder_block import Decoder


def _decoder(max_len, batch):
    dec = Decoder.__new__(Decoder)
    dec.blocks, dec.caches, dec.max_len, dec.shared = [], [], max_len, None
    dec.lengths, dec.adapter = [0] * batch, torch.zeros(batch, dtype=torch.int32)
    return dec


def test_a_common_beginning_that_is_too_long():
    dec = _decoder(10, 3)
    adapter = dec.adapter
    with pytest.raises(ValueError):
        dec.share(torch.zeros(11, 8))
    assert dec.adapter is adapter and dec.shared is None and dec.lengths == [0, 0, 0]


def test_a_common_beginning_after_the_first_rows():
    dec = _decoder(10, 2)
    dec.lengths, adapter = [0, 1], dec.adapter
    with pytest.raises(ValueError):
        dec.share(torch.zeros(4, 8))
    assert dec.adapter is adapter and dec.shared is None and dec.lengths == [0, 1]
