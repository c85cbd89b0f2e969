"""Pins of the 64-bit attention oracle, and the refusals of the attention entry points (no GPU)."""
import ctypes
import struct

import numpy as np
import pytest

from oracle import attention as oa


def test_attend_is_softmax_of_the_visible_scores():
    from scipy.special import softmax
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal(8), rng.standard_normal((20, 8)), rng.standard_normal((20, 8))
    out, size, _ = oa.attend(q, k, v, 19, 0.3)
    assert np.allclose(out, softmax(0.3 * k @ q) @ v, rtol=1e-13)
    # hidden keys may hold anything
    k2, v2 = k.copy(), v.copy()
    k2[12:], v2[13:], v2[12] = np.nan, np.inf, -np.inf
    assert np.array_equal(oa.attend(q, k2, v2, 11, 0.3)[0], oa.attend(q, k[:12], v[:12], 11, 0.3)[0])
    # equal scores average, one key is returned as it is, no key gives zeros
    assert np.allclose(oa.attend(np.zeros(8), k, v, 4, 1.0)[0], v[:5].mean(0))
    assert np.array_equal(oa.attend(q, k, v, 0, 1.0)[0], v[0])
    assert not oa.attend(q, k, v, -1, 1.0)[0].any()


def test_window_and_sinks_hand_worked():
    see = lambda p, w, s: "".join("x" if b else "." for b in oa.visible(p, 10, w, s))
    assert see(6, 0, 0) == "xxxxxxx..." == see(6, 0, 3)
    assert see(6, 3, 0) == "....xxx..."
    assert see(6, 3, 2) == "xx..xxx..."
    assert see(6, 1, 0) == "......x..."
    assert see(2, 5, 1) == "xxx......."
    assert see(1, 1, 4) == "xx........"     # a sink is not seen before its time
    assert see(-1, 3, 2) == ".........."


def test_grouped_heads_share_a_key_head():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 6, 4)), rng.standard_normal((7, 2, 4)), rng.standard_normal((7, 2, 4))
    out, _, _ = oa.attention(q, k, v, 4, 0.5)
    rep = oa.attention(q, k.repeat(3, 1), v.repeat(3, 1), 4, 0.5)[0]
    assert np.array_equal(out, rep)


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_keeps_lengths_and_depends_on_the_distance(neighbours):
    rng = np.random.default_rng(2)
    f = (10000.0 ** (-np.arange(0, 8, 2) / 8)).astype(np.float32)
    q, k = rng.standard_normal((1, 1, 12)), rng.standard_normal((1, 1, 12))
    turn = lambda x, p: oa.norm_rope(x, None, 0.0, f, [p], neighbours)[0][0, 0]
    assert np.isclose(np.linalg.norm(turn(q, 7)), np.linalg.norm(q))
    assert np.array_equal(turn(q, 0), q[0, 0]) and np.array_equal(turn(q, 5)[8:], q[0, 0, 8:])
    assert np.isclose(turn(q, 9) @ turn(k, 4), turn(q, 1009) @ turn(k, 1004), rtol=1e-9)
    # a quarter turn of the first pair
    g = np.array([np.pi / 2, 0.0], dtype=np.float32)
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    want = [-2, 1, 3, 4] if neighbours else [-3, 2, 1, 4]
    assert np.allclose(oa.norm_rope(x, None, 0.0, g, [1], neighbours)[0][0, 0], want, atol=1e-6)


def test_norm_gives_unit_mean_square():
    x = np.random.default_rng(3).standard_normal((5, 2, 16)) * 7
    y = oa.norm_rope(x, np.ones(16), 0.0, None, None, False)[0]
    assert np.allclose((y * y).mean(-1), 1.0)
    assert np.allclose(oa.norm_rope(x, 2 * np.ones(16), 0.0, None, None, False)[0], 2 * y)


# ---- refusals: rejected on the host, nothing is enqueued ----

P, NULL = 0x1000, None
CACHE = ["n_pages", "page_size", "max_pages", "batch", "kv_heads", "head_dim", "dtype", "page_stride", "slot_stride", "head_stride", "k", "v",
         "page_table", "kv_len"]


def _cache(**kw):
    v = dict(n_pages=8, page_size=16, max_pages=4, batch=2, kv_heads=2, head_dim=128, dtype=1, page_stride=4096, slot_stride=128,
             head_stride=2048, k=P, v=P, page_table=P, kv_len=P)
    assert set(kw) <= set(v)
    v.update(kw)
    return struct.pack("<10q4Q", *(v[n] for n in CACHE))


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _rope(c2r, cache=None, **kw):
    a = dict(q=P, qs=512, k=P, ks=256, v=P, vs=256, dt=1, T=2, heads=4, kv_heads=2, dim=128, qw=P, kw=P, eps=1e-6, freq=P, rot=128, nb=0,
             q_start=NULL, pos=P, qo=P, qos=512, ko=P, kos=256)
    assert set(kw) <= set(a)
    a.update(kw)
    L = c2r.lib()
    if cache is None:
        return L.c2r_qk_norm_rope(a["q"], a["qs"], a["k"], a["ks"], a["dt"], a["T"], a["heads"], a["kv_heads"], a["dim"], a["qw"], a["kw"],
                                  a["eps"], a["freq"], a["rot"], a["nb"], a["pos"], a["qo"], a["qos"], a["ko"], a["kos"], NULL)
    return L.c2r_qk_norm_rope_append(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["T"], a["heads"], a["qw"], a["kw"], a["eps"],
                                     a["freq"], a["rot"], a["nb"], a["q_start"], a["pos"], cache, a["qo"], a["qos"], NULL)


def test_norm_rope_refusals(c2r):
    bad, out = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    for form in (None, _cache()):
        r = lambda **kw: _rope(c2r, form, **kw)
        for name in ("q", "k", "qo", "freq") + (("ko", "pos") if form is None else ("v",)):
            assert r(**{name: NULL}) == bad, name
        for name in ("q", "k", "qo", "qw", "kw") + (("ko",) if form is None else ("v",)):
            assert r(**{name: P + 8}) == bad, name
        assert r(heads=0) == r(heads=3) == bad
        assert r(qs=511) == r(qs=504 + 4) == r(ks=128) == r(qos=256) == bad      # shorter than a row, not whole 16-byte pieces
        assert r(qs=516) == bad
        assert r(eps=-1.0) == r(eps=float("nan")) == r(rot=-16) == r(rot=144) == r(T=-1) == bad
        assert r(rot=24) == r(T=1 << 30) == r(heads=2048) == out
        assert r(T=0, q=NULL, k=NULL) == c2r.OK
    assert _rope(c2r, dt=2) == _rope(c2r, kv_heads=0) == bad
    assert _rope(c2r, dim=96, qs=384, ks=192, rot=96) == out
    assert _rope(c2r, _cache(), T=3) == bad                                        # one token per sequence, batch 2
    assert _rope(c2r, _cache(), T=3, q_start=P + 2) == bad


def _decode(c2r, cache, q=P, qs=512, heads=4, most=0, scale=0.1, window=0, sinks=0, out=P, os=512, ws=0x1000, n=1 << 30):
    return c2r.lib().c2r_attention_decode(q, qs, heads, cache, most, scale, window, sinks, out, os, ws, n, NULL)


def _prefill(c2r, cache, q=P, qs=512, T=100, heads=4, q_start=P, max_q=60, most=0, scale=0.1, window=0, sinks=0, out=P, os=512, ws=0x1000,
             n=1 << 30):
    return c2r.lib().c2r_attention_prefill(q, qs, T, heads, q_start, max_q, cache, most, scale, window, sinks, out, os, ws, n, NULL)


@pytest.mark.parametrize("call", [_decode, _prefill])
def test_attention_refusals(c2r, call):
    bad, out = c2r.ERR_INVALID_ARG, c2r.ERR_UNSUPPORTED
    assert call(c2r, None) == bad
    for name in ("k", "v", "page_table", "kv_len"):
        assert call(c2r, _cache(**{name: 0})) == bad, name
    for name in ("k", "v"):
        assert call(c2r, _cache(**{name: P + 8})) == bad, name
    for name in ("n_pages", "page_size", "max_pages", "kv_heads", "head_dim"):
        assert call(c2r, _cache(**{name: 0})) == bad, name
        assert call(c2r, _cache(**{name: -1})) == bad, name
    for name in ("n_pages", "page_size", "max_pages", "batch"):
        assert call(c2r, _cache(**{name: 1 << 30})) == out, name
        assert call(c2r, _cache(**{name: (1 << 32) + 4})) == out, name             # whose lower 32 bits would pass
    assert call(c2r, _cache(page_size=1 << 15, max_pages=1 << 15)) == out
    assert call(c2r, _cache(batch=-1)) == bad
    assert call(c2r, _cache(kv_heads=2048)) == call(c2r, _cache(head_dim=80)) == call(c2r, _cache(head_dim=256)) == out
    assert call(c2r, _cache(kv_heads=3)) == bad                                    # 4 query heads
    assert call(c2r, _cache(dtype=2)) == call(c2r, _cache(dtype=1 << 32)) == bad
    for name in ("page_stride", "slot_stride", "head_stride"):
        assert call(c2r, _cache(**{name: 132})) == call(c2r, _cache(**{name: -128})) == bad, name
    ok = _cache()
    assert call(c2r, ok, q=NULL) == call(c2r, ok, out=NULL) == call(c2r, ok, q=P + 2) == call(c2r, ok, out=P + 8) == bad
    assert call(c2r, ok, qs=500) == call(c2r, ok, os=256) == call(c2r, ok, qs=516) == bad
    assert call(c2r, ok, window=-1) == call(c2r, ok, sinks=-1) == call(c2r, ok, scale=float("nan")) == bad
    assert call(c2r, _cache(batch=0), q=NULL, out=NULL) == c2r.OK
    # keys that have to be split need the workspace: 64 pages of 1000 keys over 2 sequences
    long = _cache(n_pages=64, page_size=1000, max_pages=32)
    assert call(c2r, long, ws=NULL) == call(c2r, long, n=0) == call(c2r, long, ws=0x1010) == c2r.ERR_WORKSPACE


def test_prefill_refusals(c2r):
    assert _prefill(c2r, _cache(), q_start=NULL) == _prefill(c2r, _cache(), q_start=P + 2) == c2r.ERR_INVALID_ARG
    assert _prefill(c2r, _cache(), max_q=-1) == _prefill(c2r, _cache(), T=-1) == c2r.ERR_INVALID_ARG
    assert _prefill(c2r, _cache(), T=1 << 30) == c2r.ERR_UNSUPPORTED
    assert _prefill(c2r, _cache(), T=0, q=NULL, out=NULL, q_start=NULL) == c2r.OK
    assert _prefill(c2r, _cache(), max_q=0) == c2r.OK


def test_workspace_query(c2r):
    q = lambda *a: c2r.workspace_bytes(c2r.STAGE_ATTENTION, *a, c2r.BF16)
    assert q(0, 128, 16, 16, 0) == 0
    # a batch that fills the GPU needs none, one sequence little, however long its cache
    assert q(4096, 128, 16, 16, 0) == 0 and 0 < q(1, 128, 16, 16, 0) < 4 << 20
    # prompts: none where there are blocks enough, few where the keys are split
    assert q(1 << 20, 128, 16, 16, 1 << 20) == 0 and 0 < q(100, 64, 4, 4, 50) < 64 << 20


def test_struct_layout_matches_the_header(c2r):
    """Every field of c2r_kv_cache is 64 bits wide and in the order that the binding packs."""
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "c2r.h")) as f:
        body = re.search(r"typedef struct \{([^}]*)\} c2r_kv_cache;", f.read()).group(1)
    names = []
    for line in body.strip().split(";"):
        line = re.sub(r"^\s*(int64_t|void|const int32_t)\s", "", line.strip())
        names += [n.strip(" *") for n in line.split(",") if n.strip()]
    assert names == CACHE and c2r.PagedKVCache._CACHE.size == 8 * len(CACHE)
