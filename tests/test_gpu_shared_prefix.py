"""Decoding behind shared prefixes on the GPU against the definition in 64 bits (oracle/attention.py), every sequence by itself.

Tolerances, derived before the first run, those of attention over a cache: u = 2^-24, D terms of a score D u spread, its scale and
difference to the maximum 4 u spread, in numerator and denominator; sums over n keys n u; joins of parts a few more: relative to
size = sum w |v| (2 (D + 4) spread + 2 n + 64) u.  bf16: the weights' rounding, 2^-8 size at most, and the result's, 2^-8 |out|."""
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


class Batch:
    """Sequences in runs; run i has sizes[i] sequences behind prefix[i] keys, sequence b has own[b] keys behind it (or fewer than none: it
    ends inside the prefix).  Places of the cache that hold no key hold junk."""

    def __init__(self, c2r, dtype, D, H, Hkv, page, sizes, prefix, own, seed=0, junk=float("nan"), layout="hnd", before=0, after=0):
        rng = np.random.default_rng(seed)
        self.c2r, self.dtype, self.D, self.H, self.Hkv = c2r, dtype, D, H, Hkv
        B = before + sum(sizes) + after
        self.start = np.cumsum([before] + list(sizes)).astype(np.int32)
        run = [-1] * before + [i for i, n in enumerate(sizes) for _ in range(n)] + [-1] * after
        self.lens = [max(0, (prefix[r] if r >= 0 else 0) + o) for r, o in zip(run, own)]
        width = -(-max(self.lens + [1]) // page) + 2
        rows, pages, owners = [], 0, {}
        for b, (r, n) in enumerate(zip(run, self.lens)):
            whole = prefix[r] // page if r >= 0 else 0
            need = -(-max(n, prefix[r] if r >= 0 and b == self.start[r] else 0) // page)
            first = r < 0 or b == self.start[r]
            have = [] if first else rows[self.start[r]][:min(whole, need)]
            rows.append(have + list(range(pages, pages + need - len(have))))
            pages += need - len(have)
        order = rng.permutation(pages + 3)
        table = np.full((B, max(width, max(len(r) for r in rows) + 1)), -1, np.int32)
        for b, r in enumerate(rows):
            table[b, :len(r)] = order[r]
        shape = (pages + 3, Hkv, page, D) if layout == "hnd" else (pages + 3, page, Hkv, D)
        k, v = (torch.full(shape, junk, dtype=DT[dtype]).numpy() if dtype == "f32" else np.full(shape, junk, np.float32) for _ in "kv")
        rnd = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DT[dtype]).float().numpy()
        at = (lambda p, s: (p, slice(None), s)) if layout == "hnd" else (lambda p, s: (p, s))
        self.keys = []
        pre = [(rnd(n, Hkv, D), rnd(n, Hkv, D)) for n in prefix]
        for b, (r, n) in enumerate(zip(run, self.lens)):
            L = prefix[r] if r >= 0 else 0
            kk, vv = rnd(max(n - L, 0), Hkv, D), rnd(max(n - L, 0), Hkv, D)
            if r >= 0:
                kk, vv = np.concatenate([pre[r][0], kk]), np.concatenate([pre[r][1], vv])
            hold = max(n, L) if r >= 0 and b == self.start[r] else n
            for j in range(hold):
                k[at(table[b, j // page], j % page)], v[at(table[b, j // page], j % page)] = kk[j], vv[j]
            self.keys.append((kk[:n], vv[:n]))
        k, v = (torch.from_numpy(t).to(DT[dtype]).cuda() for t in (k, v))
        if layout == "nhd":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        self.cache = c2r.PagedKVCache(k, v, torch.from_numpy(table).cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda"))
        self.q = torch.from_numpy(rng.standard_normal((B, H + 2, D)).astype(np.float32)).to(DT[dtype]).cuda()[:, :H]
        self.shared_start = torch.from_numpy(self.start).cuda()
        self.shared_len = torch.tensor(prefix, dtype=torch.int32, device="cuda")
        self.prefix, self.own = prefix, own

    def run(self, **kw):
        return self.c2r.attention_decode_shared(self.q, self.cache, self.shared_start, self.shared_len, **kw)

    def check(self, out, scale=None, window=0, sinks=0, rows=None):
        scale = self.D ** -0.5 if scale is None else scale
        q, got = self.q.double().cpu().numpy(), out.double().cpu().numpy()
        for b in range(len(self.lens)) if rows is None else rows:
            k, v = self.keys[b]
            ref, size, spread = oa.attention(q[b:b + 1], k, v, self.lens[b] - 1, scale, window, sinks)
            tol = (2 * (self.D + 4) * spread + 2 * len(k) + 64) * U * size + (B8 * (size + np.abs(ref)) if self.dtype == "bf16" else 0.0) + 1e-37
            err = np.abs(got[b] - ref[0])
            assert (err <= tol[0]).all(), (b, float((err / tol[0]).max()))


SIZES = [
    # dtype-free: D, H, Hkv, page, sizes, prefix, own
    (128, 4, 4, 64, [1], [1], [1]),
    (64, 2, 1, 16, [3], [100], [1, 5, 40]),
    (128, 8, 2, 16, [5], [300], [7, 1, 64, 33, 200]),
    (64, 4, 4, 1, [4, 3], [33, 70], [1, 2, 3, 4, 50, 6, 7]),
    (128, 16, 2, 48, [20], [500], [1 + 3 * i for i in range(20)]),
    (128, 4, 1, 1000, [40], [2100], [1 + i for i in range(40)]),
    (64, 7, 1, 32, [6, 1, 9], [640, 0, 65], [1 + 11 * i for i in range(16)]),
    (128, 32, 2, 16, [9], [129], [1] * 9),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_prefixes(c2r, dtype, case):
    b = Batch(c2r, dtype, *SIZES[case], seed=case)
    b.check(b.run(max_shared_len=max(b.prefix), max_own_len=max(b.own)))
    b.check(b.run())                                          # lengths that the host does not know, or takes for shorter
    b.check(b.run(max_shared_len=1, max_own_len=1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,Hkv,each,prefix", [(64, 2, 2, 16, 1500), (64, 2, 2, 17, 1500), (128, 2, 2, 16, 1500), (128, 2, 2, 17, 1500), (128, 7, 1, 3, 700),
                                                 (64, 1, 1, 130, 4100), (128, 1, 1, 130, 4100)])
def test_rows_around_the_change_of_kernels(c2r, dtype, D, H, Hkv, each, prefix):
    """16 and 17 rows of a key head (3 x 7, too), and two blocks of them, behind a prefix long enough for many parts."""
    b = Batch(c2r, dtype, D, H, Hkv, 48, [each, each], [prefix, prefix - 65], [1 + 5 * i % 83 for i in range(2 * each)], seed=each)
    b.check(b.run(max_shared_len=prefix, max_own_len=83))
    b.check(b.run(max_shared_len=prefix, max_own_len=83, window=200, sinks=3), window=200, sinks=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 0), (200, 3), (64, 600), (5000, 1)])
@pytest.mark.parametrize("many", [False, True])
def test_windows(c2r, dtype, window, sinks, many):
    """Windows that leave all, a part or nothing of the prefix, sinks inside it and past it."""
    sizes = [26, 14] if many else [3, 2]
    own = [1 + 37 * (i % 7) for i in range(sum(sizes))]
    b = Batch(c2r, dtype, 64, 8, 2, 16, sizes, [450, 70], own, seed=window)
    b.check(b.run(window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2), (40, 2)])
def test_sequences_of_no_run_short_ones_and_empty_ones(c2r, dtype, heads):
    """Sequences before and behind the runs, ones that end inside the prefix, ones without a key, a run without a prefix and an empty run."""
    sizes, prefix = [5, 0, 3], [200, 90, 0]
    own = [30, 1, 4, -100, -200, 17, -199, 9, 65, 1, 2, 0]
    b = Batch(c2r, dtype, 128, *heads, 16, sizes, prefix, own, before=2, after=2, seed=4)
    assert min(b.lens) == 0
    out = b.run()
    b.check(out)
    assert not out[b.lens.index(0)].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("scale", [0.3, -0.2, 0.0])
def test_scales_layouts_and_results_in_the_place_of_queries(c2r, dtype, n, scale):
    b = Batch(c2r, dtype, 64, 4, 4, 24, [n], [333], [1 + i % 9 for i in range(n)], layout="nhd", seed=n)
    out = b.run(scale=scale)
    b.check(out, scale=scale)
    whole = b.q.clone()
    b.q = whole
    got = b.run(scale=scale, out=whole)
    assert got is whole and torch.equal(got, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("each", [1, 30])
def test_a_key_that_is_not_finite(c2r, dtype, n, each):
    """A NaN value in the prefix reaches exactly the sequences that see it; the places that hold no key are NaN in every test here."""
    b = Batch(c2r, dtype, 128, 4, 2, 16, [n, 2], [200, 64], [1 + each * i for i in range(n + 2)], seed=n)
    window = 60                                       # past 60 keys behind it, sequences see nothing of the prefix
    ref = b.run(window=window)
    b.check(ref, window=window)
    page, slot = int(b.cache.page_table[0, 190 // 16]), 190 % 16
    b.cache.v[page, 0, slot] = float("nan")
    out = b.run(window=window)
    sees = [i < n and 190 > b.lens[i] - 1 - window for i in range(n + 2)]
    for i, s in enumerate(sees):
        assert torch.isnan(out[i, :2]).all() if s else torch.equal(out[i], ref[i]), i
        assert torch.equal(out[i, 2:], ref[i, 2:])
    assert all(sees[:n]) == (each == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("each,group", [(1, 2), (2, 1), (3, 32)])
def test_many_runs(c2r, dtype, each, group):
    """More runs than a wave has lanes, some empty, some without a prefix; with 96 rows to each of a key head's they go through LDS in bf16."""
    n = 70
    sizes = [0 if i % 9 == 4 else each for i in range(n)]
    prefix = [0 if i % 7 == 3 else 20 + i for i in range(n)]
    b = Batch(c2r, dtype, 64, group, 1, 16, sizes, prefix, [1 + i % 40 for i in range(sum(sizes) + 3)], before=2, after=1, seed=each)
    out = b.run(max_shared_len=89, max_own_len=40)
    B = len(b.lens)
    b.check(out, rows=range(0, B, 1 if group < 32 else 11))


def test_a_large_batch_of_single_pages(c2r):
    """131072 rows of results: the workspace that is asked for is enough, and every sequence gets what it gets alone."""
    B, H, D, page, L = 4096, 32, 64, 64, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((B + 1, 1, page, D), generator=g, device="cuda").bfloat16() for _ in "kv")
    k[:, :, :L], v[:, :, :L] = k[:1, :, :L].clone(), v[:1, :, :L].clone()
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous()
    lens = (L + 1 + torch.arange(B, dtype=torch.int32, device="cuda") % (page - L)).contiguous()
    cache = c2r.PagedKVCache(k, v, table, lens)
    q = torch.randn((B, H, D), generator=g, device="cuda").bfloat16()
    i32 = dict(dtype=torch.int32, device="cuda")
    out = c2r.attention_decode_shared(q, cache, torch.tensor([0, B], **i32), torch.tensor([L], **i32), max_shared_len=L, max_own_len=page - L)
    ref = c2r.attention_decode(q, cache)
    # weights rounded to bf16 in the prefix's part, and a result's rounding on either side: 3 * 2^-8 of the largest value
    assert (out.float() - ref.float()).abs().max() <= 3 * B8 * v.abs().max().float()


def test_a_long_prefix_many_sequences(c2r):
    b = Batch(c2r, "bf16", 128, 8, 2, 16, [70], [3000], [1 + 5 * (i % 13) for i in range(70)], seed=1)
    out = b.run(max_shared_len=3000, max_own_len=61)
    b.check(out, rows=[0, 1, 33, 69])
    # each sequence by itself: two roundings of weights to bf16 apart at most
    alone = c2r.attention_decode(b.q, b.cache)
    v = max(float(np.abs(v).max()) for _, v in b.keys)
    assert (out.float() - alone.float()).abs().max() <= 4 * B8 * v
    # no run at all is decoding as it was, bit for bit
    none = c2r.attention_decode_shared(b.q, b.cache, b.shared_start[:1], b.shared_len[:0])
    assert torch.equal(none, alone)


@pytest.mark.parametrize("n", [4, 60])
def test_the_same_bits_every_time_two_streams_and_a_graph(c2r, n):
    b = Batch(c2r, "bf16", 128, 8, 2, 16, [n], [400], [1 + i % 30 for i in range(n)], seed=2)
    ref = b.run()
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(10):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(b.run())
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    out, q = torch.empty_like(ref), b.q.clone()
    ws = torch.empty(c2r.workspace_bytes(c2r.STAGE_ATTENTION_SHARED, n, 128, 8, 2, 0, c2r.BF16), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    b.q = q
    with torch.cuda.graph(g):
        b.run(out=out, ws=ws)
    for k in range(3):
        q.copy_(torch.roll(ref, k, 0))
        b.shared_len.fill_([400, 0, 130][k])              # (a shorter prefix than the keys that are alike is one, too)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, b.run())
        b.check(out, rows=[0, n - 1])
