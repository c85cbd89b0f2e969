"""Attention, norms and the cache where they are easiest to get wrong: roundings, keys in parts, kernels behind a size threshold,
lengths past the cache, scales of either sign.  Against the definitions in 64 bits (oracle/attention.py); the tolerances' terms are those
of test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_attention import B8, U, Batch, _np, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _sums(D, n, size, spread):
    """What 32-bit scores, weights and sums over n keys may be off."""
    return (2 * (D + 4) * spread + 2 * max(n, 1) + 16) * U * size + 1e-37


# ---- roundings ----

@pytest.mark.parametrize("D,H,Hkv,lens,window,sinks", [
    (128, 2, 2, [1, 2, 17, 300], 0, 0), (64, 8, 1, [1000, 33], 0, 0), (128, 20, 1, [4000], 0, 0), (64, 3, 3, [600, 2000], 130, 5)])
def test_decode_rounds_the_result_alone(c2r, D, H, Hkv, lens, window, sinks):
    """bf16: the weights reach the matrix pipe in two pieces, which leaves 2^-16 of each; the result's rounding is 2^-8 of it."""
    rng = np.random.default_rng(51 + D + H)
    bt = Batch(c2r, rng, "bf16", D, Hkv, 16, lens)
    q = _randn(rng, len(lens), H, D, dtype="bf16")
    got = _np(c2r.attention_decode(q, bt.cache, None, window, sinks, max(lens)))
    for b, n in enumerate(lens):
        k, v = (_np(x) for x in bt.rows[b])
        ref, size, spread = oa.attention(_np(q[b:b + 1]), k, v, n - 1, D ** -0.5, window, sinks)
        tol = _sums(D, n, size, spread) + 2.0 ** -16 * size + B8 * np.abs(ref)
        err = np.abs(got[b:b + 1] - ref)
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("page", [1, 16])
@pytest.mark.parametrize("D,H,Hkv", [(128, 2, 2), (64, 6, 2)])
def test_one_visible_key_is_its_value(c2r, D, H, Hkv, page):
    """bf16, a window of 1: whatever the weight is rounded to, it is its own denominator."""
    rng = np.random.default_rng(52 + D + page)
    new, lens = [150, 1, 40], [150, 9, 400]
    bt = Batch(c2r, rng, "bf16", D, Hkv, page, lens, new)
    q = _randn(rng, bt.T, H, D, dtype="bf16")
    want = torch.cat([v[n - m:] for (_, v), n, m in zip(bt.rows, lens, new)]).repeat_interleave(H // Hkv, 1)
    assert torch.equal(c2r.attention_prefill(q, bt.cache, bt.q_start, max(new), window=1), want)
    last = (bt.q_start[1:] - 1).long()
    assert torch.equal(c2r.attention_decode(q[last], bt.cache, window=1), want[last])


@pytest.mark.parametrize("D,nb", [(64, False), (128, True)])
def test_sine_and_cosine_in_full_precision(c2r, D, nb):
    """fp32, pairs (1, 0), which turn into (cos, sin).  Of an angle of pi/4 at most: its rounding 0.35 u of the result, the result's 0.5 u,
    those of the square and of the series 0.4 u at most: 1.5 u."""
    from test_gpu_attention import _freq
    rng = np.random.default_rng(53 + D)
    T = 3000
    q = torch.zeros((T, 1, D), device="cuda")
    if nb:
        q[..., ::2] = 1.0
    else:
        q[..., :D // 2] = 1.0
    pos = rng.integers(0, 1 << 17, T).astype(np.int32)
    f = _freq(D)
    got = c2r.qk_norm_rope(q, q, f, torch.from_numpy(pos).cuda(), neighbours=nb)[0]
    ref, _ = oa.norm_rope(_np(q), None, 0.0, f.cpu().numpy(), pos, nb)
    assert np.abs(_np(got) - ref).max() <= 1.5 * U, np.abs(_np(got) - ref).max() / U


# ---- lengths past the cache ----

def _check(got, q, bt, dtype, window, sinks, weights=0.0):
    """bt.lens: positions count from there; bt.rows: what is cached."""
    t, got, qn = 0, _np(got), _np(q)
    for b, m in enumerate(bt.new):
        k, v = (_np(x) for x in bt.rows[b])
        ref, size, spread = oa.attention(qn[t:t + m], k, v, bt.lens[b] - m, bt.D ** -0.5, window, sinks)
        tol = _sums(bt.D, len(k), size, spread) + (B8 * np.abs(ref) + weights * size if dtype == "bf16" else 0.0)
        err = np.abs(got[t:t + m] - ref)
        assert (err <= tol).all(), (b, float((err / tol).max()))
        t += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("most", [64, 2048])                  # keys that a sequence's row of the table can name: 4 pages, 128 pages
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 0), (20, 3), (700, 70), (4096, 0)])
def test_lengths_past_the_cache(c2r, dtype, most, window, sinks):
    """A chunk of which 5 tokens have no place, a token behind a full cache, one that fills it, one far behind."""
    rng = np.random.default_rng(54 + most)
    D, H, Hkv, page = 64, 4, 2, 16
    new, lens = [12, 1, 1, 3, 7], [most + 5, most + 1, most, most + 5000, 40]
    held = [min(n, most) for n in lens]
    bt = Batch(c2r, rng, dtype, D, Hkv, page, held, new, junk=3.0, extra=0)
    assert bt.table.shape[1] * page == most
    bt.cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    bt.lens = lens
    q, k, v = (_randn(rng, bt.T, h, D, dtype=dtype) for h in (H, Hkv, Hkv))
    before_k, before_v = bt.cache.k.clone(), bt.cache.v.clone()
    place = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(np.int32)
    seq = np.repeat(np.arange(5), new)
    from test_gpu_attention import _check_rope, _freq
    w, f = _randn(rng, D), _freq(D)
    got = c2r.qk_norm_rope_append(q, k, v, bt.cache, f, bt.q_start, None, w, w)
    _check_rope(got, q, w, 1e-6, f, place, False, dtype)
    ko = c2r.qk_norm_rope(q, k, f, torch.from_numpy(place).cuda(), w, w)[1]
    for t in range(bt.T):
        if place[t] < most:
            p, s, b = int(bt.table[seq[t], place[t] // page]), int(place[t] % page), seq[t]
            before_k[p, :, s], before_v[p, :, s] = ko[t], v[t]
            bt.rows[b][0][place[t]], bt.rows[b][1][place[t]] = ko[t], v[t]
    assert torch.equal(bt.cache.k, before_k) and torch.equal(bt.cache.v, before_v)       # older tokens stay where they are
    assert sum(place < most) == bt.T - 9
    for longest in (0, max(lens)):
        out = c2r.attention_prefill(q, bt.cache, bt.q_start, max(new), None, window, sinks, longest)
        _check(out, q, bt, dtype, window, sinks, weights=B8)
    if window == 20 and sinks == 0:
        assert not out[14:17].any() and out[13].any()         # the one far behind sees nothing; the one that fills the cache does
    # a token at a time
    last = (bt.q_start[1:] - 1).long()
    one = q[last].contiguous()
    bt.new = [1] * 5
    for longest in (0, max(lens)):
        _check(c2r.attention_decode(one, bt.cache, None, window, sinks, longest), one, bt, dtype, window, sinks, weights=2.0 ** -16)
    kk, vv = k[last].contiguous(), v[last].contiguous()
    c2r.qk_norm_rope_append(one, kk, vv, bt.cache, f, None, None, w, w)
    assert torch.equal(bt.cache.k, before_k) and torch.equal(bt.cache.v, before_v)       # they were there, or have no place


# ---- sizes past a grid ----

def test_norm_rope_of_more_tokens_than_a_grid_takes(c2r):
    """2^27 + 5 tokens, in place: rows everywhere have the bits that a short call gives them, so each was turned once."""
    T, D = (1 << 27) + 5, 64
    q, k = (torch.empty((T, 1, D), dtype=torch.bfloat16, device="cuda").normal_() for _ in "qk")
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 100003
    from test_gpu_attention import _freq
    f, w = _freq(D), _randn(np.random.default_rng(55), D)
    at = torch.cat([torch.arange(c - 9, c + 9) for c in (9, 1 << 24, (1 << 25) - 4, 1 << 25, 3 << 24, (1 << 26) - 8, (1 << 26) - 4, 1 << 26, T - 9)]
                   + [torch.randint(0, T, (4000,), generator=torch.Generator().manual_seed(1))]).cuda()
    want = c2r.qk_norm_rope(q[at], k[at], f, pos[at], w, w)
    c2r.qk_norm_rope(q, k, f, pos, w, w, out=(q, k))
    assert torch.equal(q[at], want[0]) and torch.equal(k[at], want[1])
    del q, k
    torch.cuda.empty_cache()


# ---- norms and rotation: every form over few and many tokens ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R", [(64, 64), (64, 16), (128, 128), (128, 64)])
@pytest.mark.parametrize("nb", [False, True])
@pytest.mark.parametrize("H,Hkv,T", [(5, 1, 2599), (30, 15, 2601), (16, 8, 8197), (1, 1, 1301)])
def test_norm_rope_forms(c2r, dtype, D, R, nb, H, Hkv, T):
    """Dense, in place and into a cache with positions of their own: the same bits.  Sizes on both sides of where a token's heads are
    spread over waves, head groups that are not full, an odd number of tokens; a few rows against 64 bits."""
    from test_gpu_attention import _check_rope, _freq
    rng = np.random.default_rng(56 + D + R + H)
    qkv = torch.randn((T, H + 2 * Hkv, D), generator=torch.Generator(device="cuda").manual_seed(H), device="cuda").to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    wq, wk, f = _randn(rng, D), _randn(rng, D), _freq(R)
    pos = rng.integers(0, 1 << 17, T).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    qo, ko = c2r.qk_norm_rope(q, k, f, p, wq, wk, 1e-5, nb)
    some = np.unique(np.concatenate([[0, 1, T - 2, T - 1], rng.integers(0, T, 60)]))
    at = torch.from_numpy(some).cuda()
    _check_rope(qo[at], q[at], wq, 1e-5, f, pos[some], nb, dtype)
    _check_rope(ko[at], k[at], wk, 1e-5, f, pos[some], nb, dtype)
    # sequences of one, of none, of odd lengths; one row before the first and two behind the last
    cuts = np.sort(np.concatenate([[1, 1, T - 2, T - 2], rng.integers(1, T - 1, 7)])).astype(np.int32)
    B, page = len(cuts) - 1, 48
    lens = np.diff(cuts)
    need = -(-lens // page)
    table = np.full((B, int(need.max())), -1, dtype=np.int32)
    table[np.arange(table.shape[1])[None] < need[:, None]] = rng.permutation(int(need.sum())).astype(np.int32)
    kk, vv = (torch.full((int(need.sum()), Hkv, page, D), 3.0, dtype=qkv.dtype, device="cuda") for _ in "kv")
    cache = c2r.PagedKVCache(kk, vv, torch.from_numpy(table).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda())
    out = torch.full((T, H, D), 9.0, dtype=qkv.dtype, device="cuda")
    c2r.qk_norm_rope_append(q, k, v, cache, f, torch.from_numpy(cuts).cuda(), p, wq, wk, 1e-5, nb, out=out)
    assert (out[:1] == 9).all() and (out[T - 2:] == 9).all() and torch.equal(out[1:T - 2], qo[1:T - 2])
    seq = np.repeat(np.arange(B), lens)
    place = np.concatenate([np.arange(n) for n in lens])
    pages, slots = torch.from_numpy(table[seq, place // page].astype(np.int64)).cuda(), torch.from_numpy(place % page).cuda()
    assert torch.equal(kk[pages, :, slots], ko[1:T - 2]) and torch.equal(vv[pages, :, slots], v[1:T - 2])
    kk[pages, :, slots], vv[pages, :, slots] = 3.0, 3.0
    assert (kk == 3).all() and (vv == 3).all()
    rest = v.clone()
    c2r.qk_norm_rope(q, k, f, p, wq, wk, 1e-5, nb, out=(q, k))
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(v, rest)


# ---- scales of either sign ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_across_parts_for_either_sign(c2r, dtype, D, sign):
    """Scores (powers of two) of 126.5 in the first tile of keys, 0 behind it but for one of 127.5 half way: the last one counts for 2 of
    66 parts, in whichever part of the keys it comes."""
    rng = np.random.default_rng(57 + D)
    new, n, scale = 8, 3000, sign * float(np.log(2.0)) / 2
    bt = Batch(c2r, rng, dtype, D, 1, 16, [n], [new])
    k, v = bt.rows[0]
    k.zero_(), v.zero_()
    k[:64, 0, 0], k[1500, 0, 0] = 253.0 * sign, 255.0 * sign
    v[1500] = 1.0
    bt.write(0, k, v)
    q = _randn(rng, new, 2, D, dtype=dtype)
    q[..., 0] = 1.0
    got = _np(c2r.attention_prefill(q, bt.cache, bt.q_start, new, scale))
    got1 = _np(c2r.attention_decode(q[-1:], bt.cache, scale))
    for g, first in ((got, n - new), (got1, n - 1)):
        ref, size, spread = oa.attention(_np(q[len(q) - len(g):]), _np(k), _np(v), first, scale)
        assert np.abs(ref - 2 / 66).max() < 1e-6
        # (a score has one term that is not zero: no sum of D roundings)
        assert (np.abs(g - ref) <= 8 * U * spread * size + (2 * n + 16) * U * size + (2 * B8 * size if dtype == "bf16" else 0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-1.0, 0.0])
def test_scales_that_are_not_positive_of_long_prompts(c2r, dtype, scale):
    """Prompts whose keys are split, with NaN in a query, in a hidden and in a visible place."""
    rng = np.random.default_rng(58)
    D, new, lens = 64, [130, 70], [1200, 70]
    bt = Batch(c2r, rng, dtype, D, 1, 16, lens, new)
    q = _randn(rng, 200, 2, D, dtype=dtype)
    q[7, 1, 5] = float("nan")
    for b, j in ((0, 1150), (1, 40)):
        bt.rows[b][0][j, 0, 3] = float("nan")
        bt.write(b, *bt.rows[b])
    got = c2r.attention_prefill(q, bt.cache, bt.q_start, 130, scale)
    nan = torch.zeros((200, 2), dtype=torch.bool, device="cuda")
    nan[80:130], nan[130 + 40:], nan[7, 1] = True, True, True
    assert torch.isnan(got[nan]).all() and torch.isfinite(got[~nan]).all()
    qn, clean = _np(q), ~nan.cpu().numpy()
    for b, (t, m) in enumerate(((0, 130), (130, 70))):
        k, v = (_np(x) for x in bt.rows[b])
        ref, size, spread = oa.attention(qn[t:t + m], k, v, lens[b] - m, scale)
        tol = _sums(D, lens[b], size, spread) + (B8 * (size + np.abs(ref)) if dtype == "bf16" else 0.0)
        ok = clean[t:t + m]
        assert (np.abs(_np(got[t:t + m]) - ref) <= tol)[ok].all()


# ---- results in the place of the queries ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,context,window", [(64, 0, 30), (128, 0, 30), (64, 1500, 900), (128, 1500, 900)])
def test_results_in_the_place_of_the_queries(c2r, dtype, D, context, window):
    """Hidden NaN make rows that are computed a second time, from their queries."""
    rng = np.random.default_rng(59 + D)
    new, lens = [170, 1, 60], [context + 170, 40, 60]
    bt = Batch(c2r, rng, dtype, D, 2, 16, lens, new, junk=float("nan"))
    k, v = (x.clone() for x in bt.rows[0])
    k[context + 90:context + 100], v[context + 90:context + 100] = float("nan"), float("nan")
    bt.write(0, k, v)
    q = _randn(rng, 231, 6, D, dtype=dtype)
    want = c2r.attention_prefill(q, bt.cache, bt.q_start, 170, None, window, 4)
    assert torch.isfinite(want[:90]).all()
    here = q.clone()
    assert c2r.attention_prefill(here, bt.cache, bt.q_start, 170, None, window, 4, out=here) is here
    assert torch.equal(here.nan_to_num(7.0), want.nan_to_num(7.0))
    last = q[(bt.q_start[1:] - 1).long()].contiguous()
    want = c2r.attention_decode(last, bt.cache, None, window, 4)
    c2r.attention_decode(last, bt.cache, None, window, 4, out=last)
    assert torch.equal(last.nan_to_num(7.0), want.nan_to_num(7.0))
