"""Log probabilities, entropy and the likeliest tokens on the GPU against the definition in 64 bits (oracle/serving.py).

Tolerances, derived before the first run.  u = 2^-24.  Far: the largest M - l of a logit with a probability above 2^-150 (the others are 0 in
32 bits and below 2^-150 V together).  An exponent in powers of two is off by its rounding, by that of log2 e and of the reference, 4 u of the
distance; an exponential by 2 u; a lane adds V / 256 of them and the sums of 256 lanes and 64 parts go through trees: s is off by
e = (4 Far + V / 256 + 64) u of it.  log p = l - M - ln s: e + 2 u (|l - M| + |ln s|).  H = ln s + mean distance: the second is a
quotient of two such sums: e (1 + 2 D) + 2 u (|ln s| + D) with D the mean distance.
Tokens have to be equal."""
import numpy as np
import pytest
import torch

from oracle import serving as osv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _check(c2r, logits, n_top=0, given=3, seed=0, **kw):
    T, V = logits.shape
    tokens = torch.from_numpy(np.random.default_rng(seed).integers(0, V, (T, given)).astype(np.int32)).cuda() if given else None
    got = c2r.token_logprobs(logits, tokens, n_top, **kw)
    lp, ent, top, top_lp = (None if t is None else t.double().cpu().numpy() for t in got)
    l = logits.double().cpu().numpy()
    for t in range(T):
        ref, H, M, D = osv.logprobs(l[t])
        # (two finite logits can be 6.8e38 apart; below -(2 - 2^-23) 2^127 the nearest 32-bit number is -infinity)
        ref = np.where(ref < -(2 - U) * 2.0 ** 127, -np.inf, ref)
        at = osv.order(l[t])[:n_top]
        if n_top:
            want = np.full(n_top, -1)
            want[:len(at)] = at
            assert np.array_equal(top[t], want), (t, top[t], want)
        if not np.isfinite(M):
            assert ent is None or np.isnan(ent[t])
            assert lp is None or np.isnan(lp[t]).all()
            assert not n_top or np.isnan(top_lp[t]).all()
            continue
        fin = l[t][np.isfinite(l[t])]
        far = min(float((M - fin).max()), 104.0)
        ln_s = abs(float(ref[l[t] == M][0]))
        e = (4 * far + V / 256 + 64) * U
        tol = lambda x: e + 2 * U * (np.abs(x - M) + ln_s)
        if given:
            i = tokens[t].cpu().numpy()
            fine = np.isfinite(ref[i])
            assert np.array_equal(lp[t][~fine], ref[i][~fine])
            assert (np.abs(lp[t][fine] - ref[i][fine]) <= tol(l[t][i][fine])).all()
        if ent is not None:
            assert abs(ent[t] - H) <= e * (1 + 2 * D) + 2 * U * (ln_s + D), (t, ent[t], H)
        if n_top:
            fine = np.isfinite(ref[at])
            assert np.array_equal(top_lp[t][:len(at)][~fine], ref[at][~fine]) and np.isnan(top_lp[t][len(at):]).all()
            assert (np.abs(top_lp[t][:len(at)][fine] - ref[at][fine]) <= tol(l[t][at][fine])).all()
    return got


def _logits(seed, T, V, dtype, pad=0, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, V + pad, generator=g) * scale
    l[:, :: max(1, V // 5)] += 6
    return l.to(DT[dtype]).cuda()[:, :V]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,n,pad", [(1, 1, 1, 0), (3, 2, 2, 0), (2, 7, 5, 0), (5, 33, 20, 3), (4, 257, 64, 1), (3, 1000, 1, 0), (2, 2047, 64, 5),
                                       (7, 4099, 5, 0), (2, 12001, 20, 7), (1, 50257, 20, 0), (5, 50257, 64, 0), (2, 151936, 64, 0),
                                       (1, 300001, 7, 0), (2100, 515, 3, 0), (2049, 1200, 0, 0)])
def test_rows(c2r, dtype, T, V, n, pad):
    _check(c2r, _logits(T + V, T, V, dtype, pad), n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 300, 5001, 20000])
def test_equal_logits(c2r, dtype, V):
    """Ties go to the lower index: whole rows of one number, of few numbers, of zeros of either sign, and the rest ruled out."""
    n = min(64, V)
    g = torch.Generator().manual_seed(V)
    l = torch.zeros(6, V)
    l[1] = -torch.zeros(V)
    l[1, ::2] = 0.0
    l[2] = torch.randint(0, 3, (V,), generator=g).float()
    l[3] = float("-inf")
    l[3, torch.randperm(V, generator=g)[:max(1, V // 100)]] = 1.5
    l[4] = torch.finfo(DT[dtype]).min
    l[5] = torch.finfo(DT[dtype]).min
    l[5, V // 2] = -3.0
    _check(c2r, l.to(DT[dtype]).cuda(), n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits_side_by_side(c2r, dtype):
    """Orders of logits that a search by lanes finds hard: rising, falling, all the large ones in the pieces of one lane."""
    V = 40000
    l = torch.zeros(5, V)
    l[0] = torch.arange(V) / 500.0
    l[1] = -torch.arange(V) / 500.0
    g = torch.Generator().manual_seed(1)
    per = 8 if dtype == "bf16" else 4
    piece = torch.arange(V) // per
    few = (piece % 256 == 5) | (piece % 256 == 77)
    l[2] = torch.randn(V, generator=g) + 20 * few
    l[3] = torch.where(few, torch.randn(V, generator=g), torch.tensor(float("-inf")))
    l[4] = torch.where(piece % 256 == 200, torch.arange(V) / 100.0, torch.tensor(float("-inf")))
    # (a row of many parts, and the same rows as whole blocks)
    for rows in (l, l.repeat(420, 1)):
        x = rows.to(DT[dtype]).cuda()
        got = _check(c2r, x[:5], 64)
        if len(rows) > 5:
            many = c2r.token_logprobs(x, None, 64)
            assert torch.equal(many[2][:5], got[2]) and torch.equal(many[2].view(-1, 5, 64)[-1], got[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_finite(c2r, dtype):
    V = 9001
    l = _logits(3, 8, V, dtype).clone()
    l[0, 17] = float("nan")
    l[1, 8000] = float("inf")
    l[2] = float("-inf")
    l[3] = float("nan")
    l[4] = float("nan")
    l[4, [5, 4000, 8999]] = torch.tensor([1.0, -2.0, 1.0], dtype=DT[dtype], device="cuda")
    l[5] *= 0.9 * torch.finfo(DT[dtype]).max / l[5].abs().max().float()
    l[6, :] = torch.finfo(DT[dtype]).min
    l[6, 100:140] = float("-inf")
    ref = l.double().cpu().numpy()
    got = c2r.token_logprobs(l, None, 10)
    for t in range(8):
        want = np.full(10, -1)
        at = osv.order(ref[t])[:10]
        want[:len(at)] = at
        assert np.array_equal(got[2][t].cpu().numpy(), want), t
    bad = torch.tensor([True, True, True, True, True, False, False, False])
    assert torch.isnan(got[1][bad]).all() and torch.isnan(got[3][bad]).all()
    assert torch.isfinite(got[1][~bad]).all()
    _check(c2r, l[5:], 10)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 0.02])
def test_logits_close_together(c2r, scale):
    """Rows whose logits differ in their last bits only, one block's and parts of one."""
    l = 10 + scale * torch.randn(6, 30000, generator=torch.Generator().manual_seed(7))
    _check(c2r, l.cuda(), 40)
    many = l.repeat(200, 1).cuda()
    assert torch.equal(c2r.token_logprobs(many, None, 40)[2].view(200, 6, 40)[77], c2r.token_logprobs(l.cuda(), None, 40)[2])


def test_given_tokens(c2r):
    l = _logits(4, 9, 5000, "f32")
    tokens = torch.tensor([[0, -1, 4999, 5000, 2 ** 31 - 1, 77]] * 9, dtype=torch.int32, device="cuda")
    lp = c2r.token_logprobs(l, tokens)[0]
    ref = torch.log_softmax(l.double(), -1)
    assert (lp[:, [1, 3, 4]] == float("-inf")).all()
    assert (lp[:, [0, 2, 5]].double() - ref[:, [0, 4999, 77]]).abs().max() <= 2.0 ** -18
    one = c2r.token_logprobs(l, tokens[:, 0].contiguous(), entropy=False)
    assert one[0].shape == (9,) and torch.equal(one[0], lp[:, 0]) and one[1] is None and one[2] is None
    many = torch.arange(1000, dtype=torch.int32, device="cuda").repeat(9, 1)
    got = c2r.token_logprobs(l, many)[0]
    assert torch.equal(got[:, 77], lp[:, 5])
    assert c2r.token_logprobs(l[:0], None, 3)[2].shape == (0, 3)


def test_rows_of_any_alignment(c2r):
    """Every first element of a row, 16-byte pieces or not, and nothing read or written beside the rows that matters."""
    base = _logits(5, 1, 64 * 700, "bf16")[0]
    for off in range(9):
        for V in (3, 9, 100, 511):
            l = base[off:off + 40 * 517].view(40, 517)[:, :V]
            _check(c2r, l, min(V, 4))


def test_the_same_bits_every_time_two_streams_and_a_graph(c2r):
    l = _logits(6, 40, 60000, "bf16")
    tok = torch.randint(0, 60000, (40, 2), dtype=torch.int32, device="cuda")
    ref = c2r.token_logprobs(l, tok, 20)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(10):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(c2r.token_logprobs(l, tok, 20))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, ref))
    out = tuple(torch.empty_like(t) for t in ref)
    ws = torch.empty(c2r.workspace_bytes(c2r.STAGE_LOGPROBS, 40, 60000, 1, 20, 0, c2r.BF16), dtype=torch.uint8, device="cuda")
    l2, g = l.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c2r.token_logprobs(l2, tok, 20, out=out, ws=ws)
    for k in range(3):
        l2.copy_(torch.roll(l, k * 1001, 1))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, c2r.token_logprobs(l2, tok, 20)))
