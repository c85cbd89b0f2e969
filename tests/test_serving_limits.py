"""What the calls around the blocks' halves refuse (no GPU: rejected on the host, nothing is enqueued)."""
import pytest

from test_attention_oracle import _cache

P, ODD = 0x100000, 0x100008


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _norm(c2r, **kw):
    a = dict(x=P, xs=64, r=P, rs=64, dt=1, T=4, d=64, w=P, eps=1e-6, sum=P, ss=64, y=P, ys=64, y8=P, y8s=64, scale=P)
    assert set(kw) <= set(a)
    a.update(kw)
    return c2r.lib().c2r_add_rms_norm(*a.values(), None)


def test_norm(c2r):
    bad, no = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    for kw in (dict(dt=2), dict(T=-1), dict(d=0), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(x=ODD), dict(xs=56), dict(xs=68),
               dict(rs=63), dict(r=ODD), dict(r=None), dict(y8=None), dict(scale=None), dict(sum=None, y=None, y8=None, scale=None), dict(sum=ODD),
               dict(ss=60), dict(ys=32), dict(y=ODD), dict(y8=P + 4), dict(y8s=60), dict(y8s=68), dict(scale=P + 2), dict(w=P + 4)):
        assert _norm(c2r, **kw) == bad, kw
    for kw in (dict(d=60), dict(d=32776, xs=1 << 16), dict(T=1 << 30)):
        assert _norm(c2r, **kw) == no, kw
    assert _norm(c2r, T=0, x=None) == c2r.OK


def _adapters(c2r, **kw):
    a = dict(x=P, xs=64, x_scale=None, dt=1, T=4, d_in=64, d_out=32, adapter=P, n=3, r=16, A=P, B=P, scale=P, y=P, ys=32, out=P, os=32, ws=P,
             bytes=1 << 30)
    assert set(kw) <= set(a)
    a.update(kw)
    return c2r.lib().c2r_adapters(*a.values(), None)


def test_adapters(c2r):
    bad, no = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    for kw in (dict(dt=3), dict(T=-1), dict(d_in=0), dict(d_out=0), dict(n=0), dict(r=0), dict(x_scale=P, dt=0), dict(x=None), dict(x=ODD), dict(xs=60),
               dict(x_scale=P, x=P + 4), dict(x_scale=P, xs=56), dict(x_scale=P, xs=68), dict(x_scale=P + 1), dict(y=None), dict(out=None), dict(ys=24),
               dict(os=36), dict(adapter=None), dict(adapter=P + 2), dict(A=None), dict(B=None), dict(A=ODD), dict(B=ODD), dict(scale=P + 1)):
        assert _adapters(c2r, **kw) == bad, kw
    for kw in (dict(d_in=60), dict(d_out=36), dict(r=12), dict(r=136), dict(n=1025), dict(T=1 << 24)):
        assert _adapters(c2r, **kw) == no, kw
    need = c2r.workspace_bytes(c2r.STAGE_ADAPTERS, 4, 64, 3, 16, 0, c2r.BF16)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=P + 128), dict(bytes=need - 1)):
        assert _adapters(c2r, **kw) == c2r.ERR_WORKSPACE, kw
    assert _adapters(c2r, T=0, x=None, ws=None) == c2r.OK


def _logprobs(c2r, **kw):
    a = dict(l=P, dt=0, stride=5000, T=4, V=5000, tokens=P, given=2, n=3, lp=P, ent=P, top=P, top_lp=P, ws=P, bytes=1 << 30)
    assert set(kw) <= set(a)
    a.update(kw)
    return c2r.lib().c2r_token_logprobs(*a.values(), None)


def test_logprobs(c2r):
    bad, no = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    for kw in (dict(dt=2), dict(T=-1), dict(V=0), dict(given=-1), dict(n=-1), dict(V=2), dict(given=0, n=0, ent=None), dict(l=None), dict(l=P + 2),
               dict(stride=4999), dict(tokens=None), dict(lp=None), dict(top=None), dict(top_lp=None), dict(tokens=P + 2), dict(lp=P + 2), dict(ent=P + 2),
               dict(top=P + 2), dict(top_lp=P + 1)):
        assert _logprobs(c2r, **kw) == bad, kw
    for kw in (dict(n=65), dict(given=1025), dict(T=1 << 24), dict(V=(1 << 24) + 1, stride=1 << 25)):
        assert _logprobs(c2r, **kw) == no, kw
    need = c2r.workspace_bytes(c2r.STAGE_LOGPROBS, 4, 5000, 1, 3, 0, c2r.F32)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=P + 64), dict(bytes=4 * 16)):
        assert _logprobs(c2r, **kw) == c2r.ERR_WORKSPACE, kw
    assert _logprobs(c2r, T=0, l=None, ws=None) == c2r.OK
    assert c2r.workspace_bytes(c2r.STAGE_LOGPROBS, 1 << 20, 5000, 1, 3, 0, c2r.F32) == 0      # many rows are not cut


def _shared(c2r, cache, **kw):
    a = dict(q=P, qs=2048, heads=4, cache=cache, start=P, len=P, n=1, max_shared=0, max_own=0, scale=1.0, window=0, sinks=0, out=P, os=2048, ws=P,
             bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return c2r.lib().c2r_attention_decode_shared(*a.values(), None)


def test_shared_prefixes(c2r):
    bad, no = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    for kw in (dict(cache=None), dict(n=-1), dict(start=None), dict(len=None), dict(start=P + 2), dict(len=P + 2), dict(q=None), dict(q=ODD), dict(out=None),
               dict(qs=100), dict(window=-1), dict(sinks=-1), dict(scale=float("nan"))):
        assert _shared(c2r, **{"cache": _cache(), **kw}) == bad, kw
    assert _shared(c2r, _cache(), n=1 << 20) == no
    assert _shared(c2r, _cache(head_dim=96)) == no
    assert _shared(c2r, _cache(batch=1 << 24)) == no
    for kw in (dict(ws=None), dict(ws=P + 64), dict(bytes=1024)):
        assert _shared(c2r, _cache(), **kw) == c2r.ERR_WORKSPACE, kw
    assert _shared(c2r, _cache(batch=0)) == c2r.OK
