"""Norms, rotation, cache and attention on the GPU against the definitions in 64 bits (oracle/attention.py).

Tolerances, derived before the first run.  u = 2^-24, one rounding to bf16 (7 bits behind the point) is a relative 2^-8.
* norm + rotation: y_i cos a - y_j sin a with |y_i| + |y_j| = size: a mean of D squares (D/2 u), rsqrt, two products (3 u), sine
  and cosine (1.3e-7 each and 2^-25 turns of rounding in the angle: 6 u), two products and a sum (3 u): (D/2 + 16) u size; and the
  rounding of the result.
* attention: a score is a dot product of D terms, D u spread with spread = scale * sum |q_d k_d|, and its product with the
  scale and the difference to the maximum, 4 u spread; an exponential turns an absolute error of its argument into a relative
  one, both numerator and denominator have it; sums over n keys: n u; a few more roundings.  Relative to size = sum w |v|:
  (2 (D + 4) spread + 2 n + 16) u.  bf16: the weights' rounding, 2^-8 size, and the result's, 2^-8 |out|."""
import numpy as np
import pytest
import torch

from oracle import attention as oa

pytestmark = pytest.mark.gpu

U, B8 = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _randn(rng, *shape, dtype="f32", scale=1.0):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(scale))
    return t.to(DT[dtype]).cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def _check_rope(got, x, weight, eps, f, pos, nb, dtype):
    ref, size = oa.norm_rope(_np(x), None if weight is None else _np(weight), eps, None if f is None else f.cpu().numpy(), pos, nb)
    D = ref.shape[-1]
    tol = (D / 2 + 16) * U * size + (B8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-37
    err = np.abs(_np(got) - ref)
    assert (err <= tol).all(), float((err / tol).max())


def _freq(R, base=10000.0):
    return None if R == 0 else (base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float().cuda()


# ---- norms and rotation ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R,H,Hkv,T,nb,norm", [
    (128, 128, 4, 4, 1, False, True), (128, 64, 8, 2, 7, False, True), (128, 16, 5, 1, 130, False, True), (64, 64, 3, 3, 33, True, True),
    (64, 32, 7, 1, 1, True, False), (64, 64, 1, 1, 9, False, True), (128, 0, 2, 1, 5, False, True), (128, 96, 40, 8, 3, True, True),
    (64, 48, 12, 4, 2100, False, True)])
def test_norm_rope(c2r, dtype, D, R, H, Hkv, T, nb, norm):
    rng = np.random.default_rng(D + R + H + T)
    qkv = _randn(rng, T, H + 2 * Hkv, D, dtype=dtype)                # a joint projection: strided queries and keys
    q, k = qkv[:, :H], qkv[:, H:H + Hkv]
    wq, wk = (_randn(rng, D), _randn(rng, D)) if norm else (None, None)
    pos = rng.integers(0, 1 << 17, T).astype(np.int32)
    pos[0], pos[-1] = 0, (1 << 30) - 1                                # beyond any length in use
    f = _freq(R)
    keep = qkv.clone()
    qo, ko = c2r.qk_norm_rope(q, k, f, torch.from_numpy(pos).cuda(), wq, wk, 1e-5, nb)
    assert torch.equal(qkv, keep)
    _check_rope(qo, q, wq, 1e-5, f, pos, nb, dtype)
    _check_rope(ko, k, wk, 1e-5, f, pos, nb, dtype)
    # in the place of its inputs, the same bits; one norm alone
    c2r.qk_norm_rope(q, k, f, torch.from_numpy(pos).cuda(), wq, wk, 1e-5, nb, out=(q, k))
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, H + Hkv:], keep[:, H + Hkv:])
    qo2, ko2 = c2r.qk_norm_rope(keep[:, :H], keep[:, H:H + Hkv], f, torch.from_numpy(pos).cuda(), wq, None, 1e-5, nb)
    assert torch.equal(qo2, qo)
    _check_rope(ko2, keep[:, H:H + Hkv], None, 1e-5, f, pos, nb, dtype)


def test_norm_of_zeros_and_of_nan(c2r):
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    x[1, 0, 5], x[1, 1, 5] = float("nan"), 1.0
    f, pos, w = _freq(64), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    qo, ko = c2r.qk_norm_rope(x, x, f, pos, w, w, 1e-6)
    assert torch.equal(qo, ko) or torch.isnan(qo).any()
    assert not qo[0].any() and not qo[2].any() and torch.isnan(qo[1, 0]).all() and torch.isfinite(qo[1, 1]).all()


class Batch:
    """A cache with random pages, filled behind by hand: lens[b] cached tokens, of them new[b] new."""

    def __init__(self, c2r, rng, dtype, D, Hkv, page, lens, new=None, heads=None, layout="hnd", junk=float("nan"), extra=2, spare=2):
        self.c2r, self.D, self.Hkv, self.page, self.lens = c2r, D, Hkv, page, lens
        self.new = [1] * len(lens) if new is None else new
        need = [-(-max(n, 0) // page) for n in lens]
        n_pages, width = sum(need) + spare, max(need + [1]) + extra
        order = rng.permutation(n_pages)
        table = np.full((len(lens), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table
        shape = (n_pages, Hkv, page, D) if layout == "hnd" else (n_pages, page, Hkv, D)
        kk, vv = (torch.full(shape, junk, dtype=DT[dtype], device="cuda") for _ in "kv")
        if layout == "nhd":
            kk, vv = kk.transpose(1, 2), vv.transpose(1, 2)
        self.cache = c2r.PagedKVCache(kk, vv, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        self.rows = []
        for b, n in enumerate(lens):
            k, v = _randn(rng, max(n, 0), Hkv, D, dtype=dtype), _randn(rng, max(n, 0), Hkv, D, dtype=dtype)
            self.rows.append((k, v))
            self.write(b, k, v)
        self.q_start = torch.tensor([0] + list(np.cumsum(self.new)), dtype=torch.int32, device="cuda")
        self.T = int(sum(self.new))

    def write(self, b, k, v):
        n = len(k)
        if n:
            j = np.arange(n)
            pages, slots = torch.from_numpy(self.table[b, j // self.page].astype(np.int64)).cuda(), torch.from_numpy(j % self.page).cuda()
            self.cache.k[pages, :, slots] = k
            self.cache.v[pages, :, slots] = v


def _check_attention(got, q, batch, dtype, scale, window, sinks):
    D, t = batch.D, 0
    got, qn = _np(got), _np(q)
    for b, n in enumerate(batch.new):
        k, v = (_np(x) for x in batch.rows[b])
        ref, size, spread = oa.attention(qn[t:t + n], k, v, batch.lens[b] - n, scale, window, sinks)
        tol = (2 * (D + 4) * spread + 2 * max(len(k), 1) + 16) * U * size + 1e-37
        if dtype == "bf16":
            tol = tol + B8 * size + B8 * np.abs(ref)
        err = np.abs(got[t:t + n] - ref)
        assert (err <= tol).all(), (b, float((err / tol).max()))
        t += n


# ---- the cache ----

@pytest.mark.parametrize("dtype,layout", [("bf16", "hnd"), ("f32", "nhd")])
@pytest.mark.parametrize("page,D,H,Hkv", [(1, 64, 2, 1), (16, 128, 4, 4), (48, 128, 6, 2), (1000, 64, 3, 3)])
def test_append(c2r, dtype, layout, page, D, H, Hkv):
    rng = np.random.default_rng(page + D)
    new = [5, 0, 1, 40, 17]
    lens = [5, 3, 100, 41, 10]                      # the last one holds fewer than its new tokens: 7 of them are not stored
    bt = Batch(c2r, rng, dtype, D, Hkv, page, lens, new, layout=layout, junk=3.0)
    T = bt.T + 4                                    # and 4 rows of no sequence
    qkv = _randn(rng, T, H + 2 * Hkv, D, dtype=dtype)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    w, f = _randn(rng, D), _freq(D)
    before_k, before_v = bt.cache.k.clone(), bt.cache.v.clone()
    out = torch.full((T, H, D), 9.0, dtype=DT[dtype], device="cuda")
    got = c2r.qk_norm_rope_append(q, k, v, bt.cache, f, bt.q_start, None, w, w, out=out)
    place = np.concatenate([np.arange(L - n, L) for L, n in zip(lens, new)]).astype(np.int32)
    seq = np.repeat(np.arange(5), new)
    _check_rope(got[:bt.T], q[:bt.T], w, 1e-6, f, place, False, dtype)
    assert (got[bt.T:] == 9.0).all()
    ko = c2r.qk_norm_rope(q[:bt.T], k[:bt.T], f, torch.from_numpy(place).cuda(), w, w)[1]
    for t in range(bt.T):
        if place[t] >= 0:
            p, s = int(bt.table[seq[t], place[t] // page]), int(place[t] % page)
            before_k[p, :, s], before_v[p, :, s] = ko[t], v[t]
    assert torch.equal(bt.cache.k, before_k) and torch.equal(bt.cache.v, before_v)       # and nothing else was touched


def test_append_of_single_tokens_positions_and_lost_pages(c2r):
    rng = np.random.default_rng(5)
    bt = Batch(c2r, rng, "bf16", 128, 2, 16, [1, 16, 17, 0, 33], junk=3.0)
    bt.cache.page_table[1, 0] = -1                                  # pages that are none: nothing is stored, nothing is broken
    bt.cache.page_table[2, 1] = bt.cache.k.shape[0]
    q, k, v = (_randn(rng, 5, h, 128, dtype="bf16") for h in (4, 2, 2))
    w, f = _randn(rng, 128), _freq(128)
    pos = torch.tensor([7, 100, 3, 4, 99999], dtype=torch.int32, device="cuda")
    before_k, before_v = bt.cache.k.clone(), bt.cache.v.clone()
    got = c2r.qk_norm_rope_append(q, k, v, bt.cache, f, None, pos, w, w)
    _check_rope(got, q, w, 1e-6, f, pos.tolist(), False, "bf16")
    ko = c2r.qk_norm_rope(q, k, f, pos, w, w)[1]
    for b, place in ((0, 0), (4, 32)):
        before_k[bt.table[b, place // 16], :, place % 16], before_v[bt.table[b, place // 16], :, place % 16] = ko[b], v[b]
    assert torch.equal(bt.cache.k, before_k) and torch.equal(bt.cache.v, before_v)


def test_append_to_many_sequences(c2r):
    """The search for a token's sequence, past 64 and past 64 * 64 of them, empty ones between."""
    rng = np.random.default_rng(6)
    for B in (63, 64, 65, 200, 4095, 4096, 5000):
        new = rng.integers(0, 3, B)
        new[0], new[-1] = 0, 1
        lens = (new + rng.integers(0, 3, B)).astype(np.int32)
        T = int(new.sum())
        table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous()
        cache = c2r.PagedKVCache(torch.zeros((B, 1, 4, 64), device="cuda"), torch.zeros((B, 1, 4, 64), device="cuda"), table,
                                 torch.from_numpy(lens).cuda())
        start = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        k, v = _randn(rng, T, 1, 64), _randn(rng, T, 1, 64)
        c2r.qk_norm_rope_append(k, k, v, cache, None, start)
        want = torch.zeros_like(cache.v)
        seq = np.repeat(np.arange(B), new)
        place = np.concatenate([np.arange(L - n, L) for L, n in zip(lens, new)])
        want[torch.from_numpy(seq).cuda(), 0, torch.from_numpy(place).cuda()] = v[:, 0]
        assert torch.equal(cache.v, want), B


@pytest.mark.parametrize("R", [128, 64])
def test_append_of_many_tokens(c2r, R):
    """Enough tokens that a wave takes several: sequences begin at odd rows, 70 and 130 of them in a row are empty, the first rows
    and the last ones are of no sequence."""
    rng = np.random.default_rng(29 + R)
    D, H, Hkv, page, before, behind = 128, 14, 1, 64, 3, 6
    new = [2001] + [0] * 70 + [1, 1, 1, 3001] + [0] * 130 + [2048, 5, 7301, 1]
    lens = [n + int(rng.integers(0, 3)) for n in new]
    lens[-4] -= 10                                  # fewer held than new: the first of them are not stored
    bt = Batch(c2r, rng, "bf16", D, Hkv, page, lens, new, junk=3.0, spare=0)
    T = before + bt.T + behind
    assert T * -(-(H + 2 * Hkv) // 16) >= 8192
    q, k, v = _randn(rng, T, H, D, dtype="bf16"), _randn(rng, T, Hkv, D, dtype="bf16"), _randn(rng, T, Hkv, D, dtype="bf16")
    f, w = _freq(R), _randn(rng, D)
    q_start = bt.q_start + before
    out = torch.full((T, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    bt.cache.k.fill_(3.0), bt.cache.v.fill_(3.0)
    c2r.qk_norm_rope_append(q, k, v, bt.cache, f, q_start, None, w, w, 1e-6, out=out)
    assert (out[:before] == 7).all() and (out[T - behind:] == 7).all()
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)])
    inner = slice(before, before + bt.T)
    ok = pos >= 0
    _check_rope(out[inner][torch.from_numpy(ok).cuda()], q[inner][torch.from_numpy(ok).cuda()], w, 1e-6, f, pos[ok], False, "bf16")
    seq = np.repeat(np.arange(len(new)), new)
    pages = bt.table[seq[ok], pos[ok] // page]
    pages, slots = torch.from_numpy(pages.astype(np.int64)).cuda(), torch.from_numpy(pos[ok] % page).cuda()
    keep = torch.from_numpy(ok).cuda()
    _check_rope(bt.cache.k[pages, :, slots], k[inner][keep], w, 1e-6, f, pos[ok], False, "bf16")
    assert torch.equal(bt.cache.v[pages, :, slots], v[inner][keep])
    bt.cache.k[pages, :, slots], bt.cache.v[pages, :, slots] = 3.0, 3.0
    assert (bt.cache.k == 3).all() and (bt.cache.v == 3).all()      # and nothing else was written


# ---- single tokens ----

LENS = [0, 1, 15, 16, 17, 31, 32, 33, 64, 129]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,Hkv,page,lens,window,sinks,layout", [
    (128, 2, 2, 16, LENS, 0, 0, "hnd"), (64, 3, 1, 1, LENS, 0, 0, "nhd"), (128, 8, 1, 48, LENS, 7, 2, "hnd"),
    (64, 17, 1, 32, [33, 5], 0, 0, "hnd"), (128, 40, 1, 64, [70, 2, 300], 16, 0, "nhd"),     # groups of more than 16
    (128, 4, 2, 16, [3000, 1, 777, 2048], 0, 0, "hnd"), (64, 14, 2, 1000, [2500, 40], 100, 4, "hnd"),
    (128, 2, 1, 16, [1000, 999, 70], 1, 100, "hnd"), (64, 2, 2, 16, [600] * 5, 64, 33, "nhd")])
def test_decode(c2r, dtype, D, H, Hkv, page, lens, window, sinks, layout):
    rng = np.random.default_rng(D + H + page)
    bt = Batch(c2r, rng, dtype, D, Hkv, page, lens, layout=layout)
    qkv = _randn(rng, len(lens), H + 3, D, dtype=dtype)
    q, scale = qkv[:, 1:H + 1], 1.3 * D ** -0.5
    got = c2r.attention_decode(q, bt.cache, scale, window, sinks, max(lens))
    _check_attention(got, q, bt, dtype, scale, window, sinks)
    # the longest length unknown, or told wrong: the split differs, the result holds
    for most in (0, 1, 10 ** 6):
        again = c2r.attention_decode(q, bt.cache, scale, window, sinks, most)
        _check_attention(again, q, bt, dtype, scale, window, sinks)
        assert torch.equal(again, c2r.attention_decode(q, bt.cache, scale, window, sinks, most))
    # into a strided view
    out = torch.full((len(lens), H + 2, D), 5.0, dtype=DT[dtype], device="cuda")
    c2r.attention_decode(q, bt.cache, scale, window, sinks, max(lens), out=out[:, 1:H + 1])
    assert torch.equal(out[:, 1:H + 1], got) and (out[:, 0] == 5).all() and (out[:, -1] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_large_scores(c2r, dtype):
    """Scores that differ by thousands, growing and falling along the cache: the running maximum moves all the time."""
    rng = np.random.default_rng(8)
    for order in (1, -1):
        bt = Batch(c2r, rng, dtype, 64, 1, 16, [500, 257])
        for b, (k, v) in enumerate(bt.rows):
            k *= torch.linspace(0, 60, len(k), device="cuda").flip(0)[:, None, None].to(k.dtype) if order < 0 else \
                torch.linspace(0, 60, len(k), device="cuda")[:, None, None].to(k.dtype)
            bt.write(b, k, v)
        q = _randn(rng, 2, 4, 64, dtype=dtype, scale=3.0)
        _check_attention(c2r.attention_decode(q, bt.cache, 1.0), q, bt, dtype, 1.0, 0, 0)


def _poison(bt, b, lo, hi, kind):
    """Junk in the places lo .. hi - 1 of sequence b, which no query of a test sees."""
    k, v = (x.clone() for x in bt.rows[b])
    k[lo:hi], v[lo:hi] = kind, kind
    bt.write(b, k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), -3.3895e38])
def test_decode_hidden_junk(c2r, dtype, junk):
    rng = np.random.default_rng(9)
    bt = Batch(c2r, rng, dtype, 128, 2, 16, [300, 41, 700], junk=junk)
    q = _randn(rng, 3, 6, 128, dtype=dtype)
    clean = c2r.attention_decode(q, bt.cache, window=20, sinks=3)
    _poison(bt, 0, 3, 280, junk)
    _poison(bt, 1, 3, 21, junk)
    _poison(bt, 2, 3, 680, junk)
    _check_attention(c2r.attention_decode(q, bt.cache, window=20, sinks=3), q, bt, dtype, 128 ** -0.5, 20, 3)
    # pages behind the window are given back
    bt.cache.page_table[0, 1:17] = -1
    bt.cache.page_table[2, 1:42] = 10 ** 6
    _check_attention(c2r.attention_decode(q, bt.cache, window=20, sinks=3), q, bt, dtype, 128 ** -0.5, 20, 3)
    assert torch.isfinite(clean.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_visible_infinities(c2r, dtype):
    """What a query does see follows the definition: a NaN key or value, scores of -infinity."""
    rng = np.random.default_rng(10)
    bt = Batch(c2r, rng, dtype, 64, 1, 16, [40, 200, 40, 40, 300])
    q = _randn(rng, 5, 2, 64, dtype=dtype).abs() + 0.1
    k0, v0 = bt.rows[0]
    k0[7] = -float("inf")                                             # one key of score -infinity: no weight
    k1, v1 = bt.rows[1]
    v1[190, 0, 3] = float("inf")
    k2, v2 = bt.rows[2]
    k2[:] = -float("inf")                                             # every key: 0 / 0
    k3, v3 = bt.rows[3]
    k3[5] = float("nan")
    k4, v4 = bt.rows[4]
    k4[:200] = -float("inf")                                          # whole parts without weight
    for b in range(5):
        bt.write(b, *bt.rows[b])
    got = c2r.attention_decode(q, bt.cache)
    keep = torch.ones(40, dtype=torch.bool)
    keep[7] = False
    for b, (k, v) in ((0, (k0[keep.cuda()], v0[keep.cuda()])), (4, (k4[200:], v4[200:]))):
        ref, size, spread = oa.attention(_np(q[b:b + 1]), _np(k), _np(v), len(k) - 1, 0.125)
        tol = (2 * 68 * spread + 2 * 300 + 16) * U * size + (B8 * (size + np.abs(ref)) if dtype == "bf16" else 0)
        assert (np.abs(_np(got[b:b + 1]) - ref) <= tol).all()
    assert (got[1, :, 3] == float("inf")).all() and torch.isfinite(got[1, :, 4:].float()).all()
    assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all()


# ---- prompts ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,Hkv,page,new,lens,window,sinks,layout", [
    (128, 2, 2, 16, [1], [1], 0, 0, "hnd"), (64, 2, 1, 1, [1, 2, 3, 31, 32, 33], [1, 2, 3, 31, 32, 33], 0, 0, "nhd"),
    (128, 3, 1, 48, [65, 0, 128, 1], [65, 10, 130, 400], 0, 0, "hnd"), (64, 8, 2, 64, [150], [150], 0, 0, "hnd"),
    (128, 2, 2, 16, [200, 64], [200, 300], 17, 0, "hnd"), (128, 4, 1, 32, [140, 5], [333, 90], 40, 5, "nhd"),
    (64, 5, 1, 16, [70], [1100], 1, 3, "hnd"), (64, 2, 2, 1000, [130, 2], [2000, 1500], 0, 0, "hnd"),
    (128, 7, 1, 16, [20, 3], [13, 2], 0, 0, "hnd"), (128, 1, 1, 16, [257], [257], 64, 64, "hnd"),   # (more new tokens than are cached)
    (64, 1, 1, 16, [129, 129], [1500, 700], 1000, 70, "hnd")])
def test_prefill(c2r, dtype, D, H, Hkv, page, new, lens, window, sinks, layout):
    rng = np.random.default_rng(D + H + page + sum(new))
    bt = Batch(c2r, rng, dtype, D, Hkv, page, lens, new, layout=layout)
    T = bt.T + 3                                                     # 3 rows of no sequence
    qkv = _randn(rng, T, H + 2, D, dtype=dtype)
    q, scale = qkv[:, :H], 1.3 * D ** -0.5
    out = torch.full((T, H + 1, D), 7.0, dtype=DT[dtype], device="cuda")
    got = c2r.attention_prefill(q, bt.cache, bt.q_start, max(new), scale, window, sinks, max(lens), out=out[:, :H])
    _check_attention(got[:bt.T], q[:bt.T], bt, dtype, scale, window, sinks)
    assert (out[bt.T:] == 7).all() and (out[:, H] == 7).all()
    for most, longest in ((0, max(new)), (3, max(new) + 100), (10 ** 6, T)):
        again = c2r.attention_prefill(q, bt.cache, bt.q_start, longest, scale, window, sinks, most)
        _check_attention(again[:bt.T], q[:bt.T], bt, dtype, scale, window, sinks)
        assert torch.equal(again[:bt.T], c2r.attention_prefill(q, bt.cache, bt.q_start, longest, scale, window, sinks, most)[:bt.T])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_rows_past_the_stated_most_are_untouched(c2r, dtype):
    rng = np.random.default_rng(12)
    bt = Batch(c2r, rng, dtype, 64, 1, 16, [300, 20], [300, 20])
    q = _randn(rng, 320, 2, 64, dtype=dtype)
    full = c2r.attention_prefill(q, bt.cache, bt.q_start, 300)
    out = torch.full_like(q, 7.0)
    c2r.attention_prefill(q, bt.cache, bt.q_start, 100, max_kv_len=300, out=out)
    assert (out[100:300] == 7).all()
    err = (out[:100].float() - full[:100].float()).abs().max(), (out[300:].float() - full[300:].float()).abs().max()
    assert max(err) < 0.05


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("chunks", [{0: 300}, {69: 300}, {5: 129, 40: 7, 41: 200}, {30: 128, 31: 0, 32: 0, 33: 256}, {}])
def test_prefill_of_a_mixed_batch(c2r, dtype, group, chunks):
    """A few chunks among single tokens and sequences with nothing new, some rows of no sequence before and behind, one chunk with
    more rows than the stated most."""
    rng = np.random.default_rng(41 + group + len(chunks))
    B, before, behind = 70, 5, 4
    new = [chunks.get(b, 0 if b % 7 == 3 else 1) for b in range(B)]
    lens = [n + int(rng.integers(0, 200)) for n in new]
    bt = Batch(c2r, rng, dtype, 64, 2, 16, lens, new)
    T = before + bt.T + behind
    q = _randn(rng, T, 2 * group, 64, dtype=dtype)
    start = bt.q_start + before
    for most in (max(new), 250):
        out = torch.full_like(q, 7.0)
        c2r.attention_prefill(q, bt.cache, start, most, window=90, sinks=3, out=out)
        here = torch.cat([torch.arange(s, s + min(n, most)) for s, n in zip((bt.q_start + before).tolist(), new)])
        rest = torch.ones(T, dtype=torch.bool)
        rest[here] = False
        assert (out[rest.cuda()] == 7).all()

        class View:
            pass
        v = View()
        v.D, v.rows = 64, bt.rows
        if most >= max(new):
            v.new, v.lens = new, lens
            _check_attention(out[before:before + bt.T], q[before:before + bt.T], v, dtype, 64 ** -0.5, 90, 3)
        else:       # (a chunk's rows past the most are left out: its first ones stand where they stood)
            v.new, v.lens = [min(n, most) for n in new], [L - n + min(n, most) for n, L in zip(new, lens)]
            _check_attention(out[here.cuda()], q[here.cuda()], v, dtype, 64 ** -0.5, 90, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_scales_that_are_not_positive(c2r, dtype, scale):
    rng = np.random.default_rng(42)
    bt = Batch(c2r, rng, dtype, 128, 1, 16, [150], [70])
    q = _randn(rng, 70, 2, 128, dtype=dtype)
    _check_attention(c2r.attention_prefill(q, bt.cache, bt.q_start, 70, scale), q, bt, dtype, scale, 0, 0)
    bt.new = [1]
    last = q[-1:].contiguous()
    _check_attention(c2r.attention_decode(last, bt.cache, scale), last, bt, dtype, scale, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [8, 9000, 40000, 70000])
def test_prefill_with_many_rows_of_no_sequence(c2r, dtype, T):
    """Rows that are there for a larger batch: the workspace that is asked for holds the keys' parts, however many rows there are."""
    rng = np.random.default_rng(12)
    bt = Batch(c2r, rng, dtype, 64, 1, 16, [3000], [8])
    q = _randn(rng, T, 1, 64, dtype=dtype)
    out = torch.full_like(q, 7.0)
    c2r.attention_prefill(q, bt.cache, bt.q_start, 8, out=out)
    _check_attention(out[:8], q[:8], bt, dtype, 64 ** -0.5, 0, 0)
    assert (out[8:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), -3.3895e38])
@pytest.mark.parametrize("context", [0, 1500])                       # one part, and keys that are split
def test_prefill_hidden_junk(c2r, dtype, junk, context):
    """Tokens that turn to junk at some place of a prompt reach no earlier token, and none whose window has passed them."""
    rng = np.random.default_rng(13)
    new, W, S = 170, 30, 4
    bt = Batch(c2r, rng, dtype, 128, 1, 16, [context + new, 60], [new, 60], junk=junk)
    q = _randn(rng, new + 60, 2, 128, dtype=dtype)
    n0 = context + new
    k, v = (x.clone() for x in bt.rows[0])
    lo, hi = context + 90, context + 100
    k[lo:hi], v[lo:hi] = junk, junk
    bt.write(0, k, v)
    got = c2r.attention_prefill(q, bt.cache, bt.q_start, new, window=W, sinks=S, max_kv_len=n0)
    # what the definition says, token by token; those that see the junk are left out here
    ref, size, spread = oa.attention(_np(q[:new]), *(_np(x) for x in bt.rows[0]), context, 128 ** -0.5, W, S)
    blind = [i for i in range(new) if not oa.visible(context + i, n0, W, S)[lo:hi].any()]
    tol = (2 * 132 * spread + 2 * n0 + 16) * U * size + (B8 * (size + np.abs(ref)) if dtype == "bf16" else 0)
    assert (np.abs(_np(got[:new]) - ref) <= tol)[blind].all() and len(blind) == new - 10 - W + 1
    if junk != junk:
        assert torch.isnan(got[90:100 + W - 1]).any(-1).all()
    k1, v1 = (_np(x) for x in bt.rows[1])
    ref1, size1, spread1 = oa.attention(_np(q[new:]), k1, v1, 0, 128 ** -0.5, W, S)
    tol1 = (2 * 132 * spread1 + 2 * 60 + 16) * U * size1 + (B8 * (size1 + np.abs(ref1)) if dtype == "bf16" else 0)
    assert (np.abs(_np(got[new:]) - ref1) <= tol1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_of_large_scores(c2r, dtype):
    rng = np.random.default_rng(14)
    bt = Batch(c2r, rng, dtype, 64, 1, 16, [300], [300])
    k, v = bt.rows[0]
    k *= torch.linspace(0, 60, 300, device="cuda")[:, None, None].to(k.dtype)
    bt.write(0, k, v)
    q = _randn(rng, 300, 2, 64, dtype=dtype, scale=3.0)
    _check_attention(c2r.attention_prefill(q, bt.cache, bt.q_start, 300, 1.0), q, bt, dtype, 1.0, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", ["rising", "saw", "spike", "falling"])
@pytest.mark.parametrize("powers", [20, 31, 60, 140])
def test_scores_that_jump_along_the_keys(c2r, dtype, D, shape, powers):
    """Runs of 64 keys whose scores differ by so many powers of two; a prompt behind a context, and its last token alone."""
    rng = np.random.default_rng(31 + D + powers)
    new, n = 150, 900
    bt = Batch(c2r, rng, dtype, D, 1, 16, [n], [new])
    run = np.arange(n) // 64
    level = {"rising": run, "saw": run * 5 % 3, "spike": (run == 9) * 1, "falling": -run}[shape] * powers * np.log(2.0)
    k, v = bt.rows[0]
    k *= 0.3
    k[:, 0, 0] = torch.from_numpy(level).cuda().to(k.dtype)
    bt.write(0, k, v)
    q = _randn(rng, new, 2, D, dtype=dtype)
    q[:, :, 0] = 1.0
    _check_attention(c2r.attention_prefill(q, bt.cache, bt.q_start, new, 1.0), q, bt, dtype, 1.0, 0, 0)
    _check_attention(c2r.attention_prefill(q, bt.cache, bt.q_start, new, 1.0, 300, 10), q, bt, dtype, 1.0, 300, 10)
    bt.new = [1]
    last = q[-1:].contiguous()
    _check_attention(c2r.attention_decode(last, bt.cache, 1.0), last, bt, dtype, 1.0, 0, 0)


# ---- both ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(c2r, dtype):
    """A cache whose pages lie more than 4 GB from its start, and whose element offsets pass 2^31."""
    rng = np.random.default_rng(15)
    D, page, size = 128, 16, 2 if dtype == "bf16" else 4
    n_pages = (5 << 30) // (page * D * size)
    far = [n_pages - 1 - 7 * i for i in range(30)]
    kk, vv = (torch.empty((n_pages, 1, page, D), dtype=DT[dtype], device="cuda") for _ in "kv")
    kk[far], vv[far] = float("nan"), float("nan")
    table = torch.tensor([far[:20], far[20:] + [-1] * 10], dtype=torch.int32, device="cuda")
    cache = c2r.PagedKVCache(kk, vv, table, torch.tensor([300, 150], dtype=torch.int32, device="cuda"))
    k, v = _randn(rng, 450, 1, D, dtype=dtype), _randn(rng, 450, 1, D, dtype=dtype)
    start = torch.tensor([0, 300, 450], dtype=torch.int32, device="cuda")
    q = c2r.qk_norm_rope_append(k, k, v, cache, None, start)          # no norm, no rotation: keys and values as they are
    assert torch.equal(q, k)

    class View:
        pass
    bt = View()
    bt.D, bt.lens, bt.new, bt.rows = D, [300, 150], [300, 150], [(k[:300], v[:300]), (k[300:], v[300:])]
    _check_attention(c2r.attention_prefill(q, cache, start, 300), q, bt, dtype, D ** -0.5, 0, 0)
    bt.new = [1, 1]
    last = torch.stack([q[299], q[449]])
    _check_attention(c2r.attention_decode(last, cache), last, bt, dtype, D ** -0.5, 0, 0)


def test_a_stream_of_its_own_and_a_graph(c2r):
    """Everything is enqueued on the current stream; a captured decoding step replays with new lengths in place."""
    rng = np.random.default_rng(16)
    bt = Batch(c2r, rng, "bf16", 128, 2, 16, [900, 33, 500])
    q, k, v = (_randn(rng, 3, h, 128, dtype="bf16") for h in (8, 2, 2))
    f, w = _freq(128), _randn(rng, 128)

    def step():
        qo = c2r.qk_norm_rope_append(q, k, v, bt.cache, f, None, None, w, w)
        return c2r.attention_decode(qo, bt.cache, max_kv_len=1024)
    want = step().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    before_k, before_v = bt.cache.k.clone(), bt.cache.v.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for lens in ([900, 33, 500], [20, 1, 499], [901, 0, 7], [900, 33, 500]):
        bt.cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        bt.cache.k.copy_(before_k)                                   # (a step with other lengths stores elsewhere)
        bt.cache.v.copy_(before_v)
        eager = step()
        assert torch.equal(replayed, eager), lens
        bt.cache.k.copy_(before_k)
        bt.cache.v.copy_(before_v)
    assert torch.equal(replayed, want)


def test_prompt_in_chunks_and_token_by_token(c2r):
    """The same sequence as one prompt, in chunks and a token at a time, with a window and sinks."""
    rng = np.random.default_rng(17)
    n, H, Hkv, D = 150, 4, 2, 64
    q, k, v = (_randn(rng, n, h, D, dtype="f32") for h in (H, Hkv, Hkv))
    f, w = _freq(D), _randn(rng, D)
    results = []
    for cuts in ([0, n], [0, 70, 71, 140, n], list(range(n + 1))):
        cache = c2r.PagedKVCache.empty(12, 16, Hkv, D, 1, 12, torch.float32)
        cache.page_table.copy_(torch.randperm(12).int()[None])
        rows = []
        for a, b in zip(cuts, cuts[1:]):
            cache.kv_len.fill_(b)
            start = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
            single = b - a == 1
            qo = c2r.qk_norm_rope_append(q[a:b], k[a:b], v[a:b], cache, f, None if single else start, None, w, w)
            rows.append(c2r.attention_decode(qo, cache, window=50, sinks=4) if single else
                        c2r.attention_prefill(qo, cache, start, b - a, window=50, sinks=4))
        results.append(torch.cat(rows))
    for r in results[1:]:
        assert (r - results[0]).abs().max() < 2e-5
