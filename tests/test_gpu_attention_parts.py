"""Attention whose keys are cut into parts and joined: junk in hidden places, rows of which a part sees nothing, many rows, part and tile
boundaries of long contexts.  Against the definitions in 64 bits (oracle/attention.py); the terms of the tolerances are those of
test_gpu_attention.py, and a root mean square beside them where a worst case would let a key too many pass."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_attention import B8, U, Batch, _np, _randn

pytestmark = pytest.mark.gpu
SIGMA = B8 / 3 ** 0.5           # root mean square of a rounding to bf16, relative, where it is largest


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _cut(c2r, call, *args, **kw):
    """The call's result, once it is known to cut the keys: without a workspace it is refused."""
    with pytest.raises(c2r.C2RError) as e:
        call(*args, **kw, ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert e.value.code == c2r.ERR_WORKSPACE
    return call(*args, **kw)


def _tol(D, n, size, spread, ref, dtype):
    return (2 * (D + 4) * spread + 2 * max(n, 1) + 16) * U * size + 1e-37 + (B8 * (size + np.abs(ref)) if dtype == "bf16" else 0.0)


JUNK = [float("nan"), float("inf"), -float("inf"), -3.3895e38]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_in_parts_over_hidden_junk(c2r, dtype, junk, D):
    """A window of 900 and 40 sinks.  Junk behind the sinks, which no new token sees, in some of the last tokens, which the ones before
    them do not see, and wherever no token is; a sequence that is too short to be cut, one of length 0, one with nothing new."""
    rng = np.random.default_rng(61)
    new, lens, W, S = [150, 3, 0, 5, 90], [1700, 20, 100, 0, 1200], 900, 40
    bt = Batch(c2r, rng, dtype, D, 1, 16, lens, new, junk=junk)
    for b, places in ((0, [(41, 640), (1620, 1625), (1690, 1691)]), (4, [(45, 200), (1190, 1200)])):
        k, v = (x.clone() for x in bt.rows[b])
        for lo, hi in places:
            k[lo:hi], v[lo:hi] = junk, junk
        bt.write(b, k, v)
    q = _randn(rng, bt.T, 3, D, dtype=dtype)
    got = _np(_cut(c2r, c2r.attention_prefill, q, bt.cache, bt.q_start, 150, None, W, S, 1700))
    qn, t = _np(q), 0
    clean = {0: 1620 - 1550, 1: 3, 2: 0, 3: 5, 4: 1190 - 1110}           # the new tokens before the first junk among them
    for b, m in enumerate(new):
        c = clean[b]
        k, v = (_np(x) for x in bt.rows[b])
        ref, size, spread = oa.attention(qn[t:t + c], k, v, lens[b] - m, D ** -0.5, W, S)
        err = np.abs(got[t:t + c] - ref)
        assert (err <= _tol(D, len(k), size, spread, ref, dtype)).all(), b
        if junk != junk:
            assert np.isnan(got[t + c:t + m]).any(-1).all()
        t += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("window,sinks", [(700, 5), (0, 0)])
def test_token_in_parts_over_hidden_junk(c2r, dtype, junk, window, sinks):
    rng = np.random.default_rng(62)
    lens = [2400, 700, 1, 0, 1033, 3000]
    bt = Batch(c2r, rng, dtype, 128, 1, 16, lens, junk=junk)
    if window:
        for b in (0, 4, 5):
            k, v = (x.clone() for x in bt.rows[b])
            k[sinks:lens[b] - window], v[sinks:lens[b] - window] = junk, junk
            bt.write(b, k, v)
        bt.cache.page_table[0, 1:100] = -1                               # given back: they read as page 0, which is junk in part
    q = _randn(rng, 6, 6, 128, dtype=dtype)
    got = _np(_cut(c2r, c2r.attention_decode, q, bt.cache, None, window, sinks, 3000))
    for b, n in enumerate(lens):
        k, v = (_np(x) for x in bt.rows[b])
        ref, size, spread = oa.attention(_np(q[b:b + 1]), k, v, n - 1, 128 ** -0.5, window, sinks)
        assert (np.abs(got[b:b + 1] - ref) <= _tol(128, n, size, spread, ref, dtype)).all(), b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_scores_of_minus_infinity(c2r, dtype):
    """Whole parts whose keys have no weight, behind and before the others, for a token and a prompt; and rows all of whose keys have none."""
    rng = np.random.default_rng(63)
    D, n = 64, 2000
    for lo, hi in ((0, 1500), (500, 2000 - 4), (0, 2000)):
        bt = Batch(c2r, rng, dtype, D, 1, 16, [n], [4])
        k, v = bt.rows[0]
        k[lo:hi] = -float("inf")
        bt.write(0, k, v)
        q = _randn(rng, 4, 2, D, dtype=dtype).abs() + 0.1
        keep = np.ones(n, dtype=bool)
        keep[lo:hi] = False
        for got, first in ((_cut(c2r, c2r.attention_prefill, q, bt.cache, bt.q_start, 4), n - 4),
                           (_cut(c2r, c2r.attention_decode, q[-1:].contiguous(), bt.cache), n - 1)):
            if not keep.any():
                assert torch.isnan(got).all()
                continue
            kn, vn = _np(k), _np(v)
            for i in range(len(got)):
                see = keep & (np.arange(n) <= first + i)
                ref, size, spread = oa.attention(_np(q[4 - len(got) + i:][:1]), kn[see], vn[see], int(see.sum()) - 1, D ** -0.5)
                assert (np.abs(_np(got[i:i + 1]) - ref) <= _tol(D, n, size, spread, ref, dtype)).all()


# ---- many rows: the join goes through several rows' parts side by side ----

def _rows_agree(got, q, k, v, first, rows, D, window, sinks, dtype):
    kn, vn = _np(k), _np(v)
    for i in rows:
        ref, size, spread = oa.attention(_np(q[i:i + 1]), kn, vn, first + i, D ** -0.5, window, sinks)
        assert (np.abs(_np(got[i:i + 1]) - ref) <= _tol(D, len(kn), size, spread, ref, dtype)).all(), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,Hkv,new,context", [(64, 16, 4, 1100, 0), (128, 16, 4, 1100, 0), (128, 16, 16, 1031, 2000), (64, 32, 8, 520, 3000)])
def test_prompt_of_many_rows_in_parts(c2r, dtype, D, H, Hkv, new, context):
    """From 16384 rows (token, head) on; a second, short sequence whose keys are not cut; hidden NaN in the last token."""
    rng = np.random.default_rng(64 + D + new)
    lens, news = [context + new, 70], [new, 33]
    assert max(news) * H * 2 >= 16384
    bt = Batch(c2r, rng, dtype, D, Hkv, 16, lens, news)
    q = _randn(rng, bt.T, H, D, dtype=dtype)
    call = lambda: c2r.attention_prefill(q, bt.cache, bt.q_start, new, max_kv_len=context + new)
    if context or (dtype, D) == ("bf16", 128):               # (the others are not cut: their blocks fill the GPU)
        _cut(c2r, lambda **kw: c2r.attention_prefill(q, bt.cache, bt.q_start, new, max_kv_len=context + new, **kw))
    got = call()
    assert torch.isfinite(got).all() and torch.equal(got, call())
    rows = sorted({0, 1, 63, 64, 127, 128, 500, new - 2, new - 1} | set(rng.integers(0, new, 6).tolist()))
    _rows_agree(got, q, *bt.rows[0], context, rows, D, 0, 0, dtype)
    _rows_agree(got[new:], q[new:], *bt.rows[1], 37, range(0, 33, 8), D, 0, 0, dtype)
    k, v = (x.clone() for x in bt.rows[0])
    k[-1], v[-1] = float("nan"), float("nan")
    bt.write(0, k, v)
    again = call()
    assert torch.isnan(again[new - 1]).all() and torch.isfinite(again[:new - 1]).all() and torch.isfinite(again[new:]).all()
    _rows_agree(again, q, *bt.rows[0], context, [r for r in rows if r < new - 1][-5:], D, 0, 0, dtype)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_tokens_of_many_rows_in_parts(c2r, dtype, D):
    """256 sequences of 64 heads over the same pages, each with its own length: parts that are empty, one part that has all, several."""
    rng = np.random.default_rng(65)
    B, H, Hkv, page, n = 256, 64, 4, 16, 3200
    pages = n // page
    k, v = (_randn(rng, pages, Hkv, page, D, dtype=dtype) for _ in "kv")
    table = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    lens = rng.integers(0, n + 1, B).astype(np.int32)
    lens[:9] = [0, 1, 31, 32, 33, 767, 768, 769, n]
    cache = c2r.PagedKVCache(k, v, table[None].repeat(B, 1).contiguous(), torch.from_numpy(lens).cuda())
    q = _randn(rng, B, H, D, dtype=dtype)
    got = _cut(c2r, c2r.attention_decode, q, cache, max_kv_len=n)
    kn, vn = (_np(x[table.long()].transpose(1, 2).reshape(n, Hkv, D)) for x in (k, v))
    for b in list(range(9)) + [20, 100, 255]:
        ref, size, spread = oa.attention(_np(q[b:b + 1]), kn[:lens[b]], vn[:lens[b]], int(lens[b]) - 1, D ** -0.5)
        assert (np.abs(_np(got[b:b + 1]) - ref) <= _tol(D, lens[b], size, spread, ref, dtype)).all(), b


# ---- a key too many or too few ----

def _mean_square_bound(q, k, v, first, scale, window, sinks, rounded_weights):
    """(results, largest root mean square of bf16's roundings): the result's, and of independent ones of the weights, which the
    denominator has too: sum w^2 (v - out)^2 <= 2 sum w^2 (v^2 + out^2).  32-bit sums are far below (2^-24 times thousands at the most)."""
    n, H, D = q.shape
    group = H // k.shape[1]
    out, noise = np.zeros((n, H, D)), 0.0
    for i in range(n):
        see = oa.visible(first + i, len(k), window, sinks)
        for h in range(H):
            kk, vv = k[see, h // group], v[see, h // group]
            s = scale * (kk @ q[i, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vv
            if rounded_weights:
                noise += 2 * ((w * w) @ (vv * vv + out[i, h] ** 2)).sum()
    rms = np.sqrt((out ** 2).mean())
    return out, SIGMA * (rms + np.sqrt(noise / out.size))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,new,window,sinks", [
    (1023, 1, 0, 0), (1024, 1, 0, 0), (1025, 1, 0, 0), (2049, 1, 0, 0), (3000, 1, 1000, 0), (3000, 1, 1024, 64), (2500, 1, 1025, 33),
    (1024, 16, 0, 0), (1500, 65, 0, 0), (3000, 16, 1000, 0), (2500, 20, 1024, 64), (2000, 33, 961, 7)])
def test_long_rows_see_every_key_once(c2r, D, n, new, window, sinks):
    """bf16.  Scores close to each other, so that every key counts: with one key more or less at either end of what a query sees, the
    definition itself is out of the bound."""
    rng = np.random.default_rng(66 + D + n + new)
    H, Hkv, scale = 8, 4, 0.3 * D ** -0.5
    bt = Batch(c2r, rng, "bf16", D, Hkv, 16, [n], [new])
    q = _randn(rng, new, H, D, dtype="bf16")
    calls = [lambda m: c2r.attention_prefill(q, bt.cache, bt.q_start, new, scale, window, sinks, m)]
    if new == 1:
        calls.append(lambda m: c2r.attention_decode(q, bt.cache, scale, window, sinks, m))
    k, v, qn = _np(bt.rows[0][0]), _np(bt.rows[0][1]), _np(q)
    for i, call in enumerate(calls):
        ref, bound = _mean_square_bound(qn, k, v, n - new, scale, window, sinks, i == 0)
        rms = lambda x: np.sqrt(((x - ref) ** 2).mean())
        for m in (n, 0, 100):                                # the parts differ
            assert rms(_np(call(m))) <= bound, (i, m)
        wrong = [(n - new - 1, window, sinks)] + ([(n - new, window + 1, sinks), (n - new, window - 1, sinks)] if window else []) + \
            ([(n - new, window, sinks + 1), (n - new, window, sinks - 1)] if sinks else [])
        for at, W, S in wrong:
            assert rms(oa.attention(qn, k, v, at, scale, W, S)[0]) > 2 * bound, (at, W, S)


# ---- norms of zeros and of NaN ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_stays_in_its_head(c2r, dtype):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.zeros((5, 3, 64), dtype=dt, device="cuda")
    x[1, 0, 5], x[1, 1, 5], x[3, 2, 63], x[4, 1, 0] = float("nan"), 1.0, float("inf"), -2.0
    f = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda()
    pos, w = torch.arange(5, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    qo, ko = c2r.qk_norm_rope(x, x, f, pos, w, w, 1e-6)
    assert torch.equal(torch.isnan(qo), torch.isnan(ko)) and torch.equal(qo.nan_to_num(7.0), ko.nan_to_num(7.0))
    bad = torch.zeros((5, 3), dtype=torch.bool, device="cuda")
    bad[1, 0] = True
    assert torch.isnan(qo[bad]).all()
    bad[3, 2] = True                                          # infinity times 0
    assert torch.isnan(qo[3, 2]).any() and torch.isfinite(qo[~bad]).all()
    assert not qo[0].any() and not qo[2].any() and qo[1, 1].any() and qo[4, 1].any()


@pytest.mark.parametrize("most", [1 << 20, 1 << 31, (1 << 32) + 1, 1 << 62])
def test_a_most_that_is_past_every_length(c2r, most):
    """max_q_len as no limit: the workspace is the one of all T rows."""
    rng = np.random.default_rng(67)
    bt = Batch(c2r, rng, "bf16", 128, 16, 16, [1100], [1100])
    q = _randn(rng, 1100, 16, 128, dtype="bf16")
    want = _cut(c2r, c2r.attention_prefill, q, bt.cache, bt.q_start, 1100, max_kv_len=1100)
    assert torch.equal(c2r.attention_prefill(q, bt.cache, bt.q_start, most, max_kv_len=1100), want)
