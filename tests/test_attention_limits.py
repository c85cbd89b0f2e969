"""What the attention entry points refuse beside test_attention_oracle.py's cases (no GPU: rejected on the host, nothing is enqueued)."""
import pytest

from test_attention_oracle import _cache, _prefill, _rope


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def test_rows_that_share_a_place_are_not_written(c2r):
    """An append to a cache whose pages, slots or heads overlap: which row stays would be left to chance."""
    for kw in (dict(slot_stride=0), dict(slot_stride=64), dict(head_stride=0), dict(head_stride=120), dict(page_stride=0), dict(page_stride=64)):
        assert _rope(c2r, _cache(**kw)) == c2r.ERR_INVALID_ARG, kw
    # a stride that takes no step may be anything; nothing to do is fine
    for kw in (dict(page_size=1, slot_stride=0), dict(kv_heads=1, head_stride=0), dict(n_pages=1, page_stride=0)):
        assert _rope(c2r, _cache(**kw), T=0) == c2r.OK, kw


def test_prompts_past_the_stated_size(c2r):
    """T * heads from 2^31 on, and a batch whose blocks pass a grid."""
    assert _prefill(c2r, _cache(), T=1 << 29, max_q=1 << 29) == c2r.ERR_UNSUPPORTED
    assert _prefill(c2r, _cache(batch=1 << 24), T=1 << 24, max_q=1) == c2r.ERR_UNSUPPORTED
