"""Calls of no rows, whose arrays have no address (no GPU: nothing is enqueued)."""
from test_serving_limits import _logprobs, _norm, c2r  # noqa: F401 (the fixture)


def test_logprobs(c2r):  # noqa: F811
    none = dict(T=0, l=None, tokens=None, lp=None, ent=None, top=None, top_lp=None, ws=None, bytes=0)
    for kw in (dict(), dict(given=0), dict(n=0), dict(given=0, n=0)):
        assert _logprobs(c2r, **none, **kw) == c2r.OK, kw
    assert _logprobs(c2r, given=0, n=0, ent=None) == c2r.ERR_INVALID_ARG


def test_norm(c2r):  # noqa: F811
    none = dict(T=0, x=None, sum=None, y=None, y8=None, scale=None)
    for kw in (dict(), dict(r=None), dict(r=None, w=None)):
        assert _norm(c2r, **{**none, **kw}) == c2r.OK, kw
    assert _norm(c2r, **{**none, "T": 1, "x": 0x100000}) == c2r.ERR_INVALID_ARG
