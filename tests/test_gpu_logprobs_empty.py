"""Log probabilities of no rows, and of no tokens: empty results of the shapes that are asked for."""
import pytest
import torch

from test_gpu_logprobs import c2r  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(0,), (0, 1), (0, 4), (0, 0)])
def test_no_rows(c2r, dtype, shape):  # noqa: F811
    logits, tokens = torch.empty((0, 5000), dtype=dtype, device="cuda"), torch.empty(shape, dtype=torch.int32, device="cuda")
    lp, ent, top, top_lp = c2r.token_logprobs(logits, tokens, 3)
    assert lp.shape == shape and lp.dtype is torch.float32 and ent.shape == (0,) and top.shape == top_lp.shape == (0, 3)
    if shape != (0, 0):                    # given tokens alone
        lp, ent, top, top_lp = c2r.token_logprobs(logits, tokens, entropy=False)
        assert lp.shape == shape and ent is None and top is None and top_lp is None
    _, ent, _, _ = c2r.token_logprobs(logits)         # the entropy alone
    assert ent.shape == (0,)
    into = (torch.empty(shape, device="cuda"), torch.empty(0, device="cuda"), None, None)
    assert c2r.token_logprobs(logits, tokens, out=into)[0] is into[0]


def test_no_tokens(c2r):  # noqa: F811
    logits = torch.randn(3, 100, device="cuda")
    lp, ent, _, _ = c2r.token_logprobs(logits, torch.empty((3, 0), dtype=torch.int32, device="cuda"))
    assert lp.shape == (3, 0) and torch.equal(ent, c2r.token_logprobs(logits)[1])
    assert c2r.token_logprobs(logits)[0] is None
