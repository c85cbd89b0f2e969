"""Timed cases of the attention operators that stand beside the MoE layer in a decoder block, over their real sizes.

A case is a dict of plain values.  `op` names the operator:

* "append"   per-head RMS norms of queries and keys, the position rotation, and the new keys and values written into a
             paged cache, in one pass.  With new = 1 it is what a decoding step does before it attends.
* "rotate"   the norms and the rotation alone, dense rows in and out.
* "decode"   one new token per sequence over the paged cache.
* "prefill"  prompts, or chunks of prompts behind what is cached already.

Attention is causal; with a window W a query sees its last W keys and the first `sinks` ones.  Head counts follow the
model widths of paper_2504_01337_amd/workloads.py (2048 and 4096 with heads of 128, 256 with heads of 64); grouped heads
are generic.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BASE = 10000.0


def _case(name, op, dtype, heads, kv_heads, dim, seqs, new, context, page=64, window=0, sinks=0, rot=None, pairs="halves",
          ragged=True):
    return {"name": name, "op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "new": new,
            "context": context, "page": page, "window": window, "sinks": sinks, "rot": dim if rot is None else rot, "pairs": pairs,
            "ragged": ragged}


def listed():
    return [
        # the step of a single stream: latency and nothing else
        _case("append_1", "append", "bf16", 16, 16, 128, 1, 1, 4095),
        # prompts of a serving batch, some behind a cached prefix; grouped heads, a part of each head rotated
        _case("append_grouped_1000", "append", "bf16", 32, 8, 128, 5, 401, 700, page=16, rot=64),
        # whole prompts, 4 x 2048 tokens of the 2048-wide model
        _case("append_8192", "append", "bf16", 16, 16, 128, 4, 2048, 0, ragged=False),
        # full precision, the 256-wide model, neighbouring pairs
        _case("rotate_f32_512", "rotate", "f32", 4, 4, 64, 1, 512, 0, pairs="neighbours"),
        # one stream decoding against 4096 keys: the cache has to be split over the chip
        _case("decode_1_4096", "decode", "bf16", 16, 16, 128, 1, 1, 4095),
        # a small decoding batch of ragged lengths, odd pages
        _case("decode_16_ragged", "decode", "bf16", 32, 32, 128, 16, 1, 1500, page=48),
        # a serving batch of an odd size with grouped heads
        _case("decode_131_grouped", "decode", "bf16", 32, 8, 128, 131, 1, 8000, page=16),
        # long contexts of which a window and the first tokens are looked at
        _case("decode_window_24", "decode", "bf16", 32, 8, 128, 24, 1, 32000, window=1024, sinks=4),
        # full precision
        _case("prefill_f32_512", "prefill", "f32", 4, 4, 64, 1, 512, 0),
        # chunks of prompts behind cached prefixes
        _case("prefill_chunks_1000", "prefill", "bf16", 32, 8, 128, 5, 401, 3000, page=16),
        # whole prompts, 4 x 2048 tokens of the 2048-wide model
        _case("prefill_8192", "prefill", "bf16", 16, 16, 128, 4, 2048, 0, ragged=False),
        # one long prompt through a window with sinks
        _case("prefill_window_16000", "prefill", "bf16", 16, 16, 128, 1, 16000, 0, window=2048, sinks=16),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, its logarithm evenly spread."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "rotate", "decode", "decode", "decode", "prefill", "prefill", "prefill"])
    most = max((work(c) for c in listed() if c["op"] == {"rotate": "append"}.get(op, op)), key=lambda w: w["bytes"] + w["flops"])
    while True:
        dtype = rng.choice(["bf16"] * 4 + ["f32"])
        dim = rng.choice([64, 128, 128])
        kv_heads = rng.choice([1, 2, 4, 8, 16, 32]) if dtype == "bf16" else rng.choice([1, 2, 4])
        heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8])
        if heads > 64:
            continue
        page = rng.choice([1, 16, 16, 32, 48, 64, 64, 128, 1000])
        window = rng.choice([0, 0, 0, _spread(rng, 1, 8192)])
        sinks = rng.choice([0, 1, 4, 16, 100]) if window else 0
        rot = rng.choice([dim, dim, dim // 2])
        pairs = rng.choice(["halves", "halves", "neighbours"])
        if op == "decode":
            seqs, new, context = _spread(rng, 1, 256), 1, _spread(rng, 1, 32768) - 1
        elif op == "rotate":
            seqs, new, context = 1, _spread(rng, 1, 8192), _spread(rng, 1, 100000) - 1
        else:
            seqs, new = _spread(rng, 1, 32), _spread(rng, 1, 16384)
            context = rng.choice([0, _spread(rng, 1, 16384) - 1])
        case = _case("", op, dtype, heads, kv_heads, dim, seqs, new, context, page, window, sinks, rot, pairs)
        del case["name"]
        # the plain forms hold whole rows of scores and padded copies of the cache in 32 bits
        held = seqs * (context + new) * max(kv_heads, heads // 8) * dim * 4
        w = work(case)
        flops = w["flops"] * (8 if dtype == "f32" and op == "prefill" else 1)
        if w["bytes"] <= most["bytes"] * (1 if op != "prefill" else 4) and flops <= most["flops"] and held < 8e9 and (context + new) * new <= 3e8:
            return case


# ---- lengths: a trait of the case ----------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, cached tokens before them) of every sequence: the longest first; ragged ones spread below it."""
    rng = random.Random(7919 * case["seqs"] + 31 * case["new"] + case["context"])
    new, before = [case["new"]], [case["context"]]
    for _ in range(case["seqs"] - 1):
        new.append(max(1, int(case["new"] * rng.uniform(0.1, 1.0))) if case["ragged"] else case["new"])
        before.append(int(case["context"] * rng.uniform(0.05, 1.0)) if case["ragged"] else case["context"])
    return new, before


def _pairs_seen(case, new, before):
    """Visible (query, key) pairs of one sequence, and the keys that any of its queries sees."""
    W, S = case["window"], case["sinks"]
    end = before + new
    if not W:
        return new * before + new * (new + 1) // 2, end
    pairs = 0
    for p in range(before, end):
        lo = max(0, p - W + 1)
        pairs += p + 1 - lo + min(S, lo)
    first = max(0, before - W + 1)
    return pairs, end - first + min(S, first)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    H, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
    new, before = _lengths(case)
    T = sum(new)
    if case["op"] in ("append", "rotate"):
        rows = H + (2 if case["op"] == "append" else 1) * Hkv
        return {"bytes": 2 * size * T * rows * D + 4 * T, "flops": 8.0 * T * (H + Hkv) * D}
    seen = [_pairs_seen(case, n, b) for n, b in zip(new, before)]
    return {"bytes": 2 * size * T * H * D + 2 * size * Hkv * D * sum(k for _, k in seen), "flops": 4.0 * H * D * sum(p for p, _ in seen)}


# ---- inputs ------------------------------------------------------------------------------------------------

def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _inputs(case, seed):
    """Tensors of a case, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    H, Hkv, D, B, page = case["heads"], case["kv_heads"], case["dim"], case["seqs"], case["page"]
    new, before = _lengths(case)
    T, total = sum(new), [n + b for n, b in zip(new, before)]
    s = {"case": case, "new": new, "before": before, "total": total}
    i32 = dict(dtype=torch.int32, device="cuda")
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"], s["q_start"] = starts, torch.tensor(starts, **i32)
    if case["op"] != "rotate":
        need = [-(-t // page) for t in total]
        width, n_pages = max(need), sum(need) + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, width), -1, **i32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        s["table"], s["kv_len"] = table, torch.tensor(total, **i32)
        s["k_pages"] = _normal(gen, (n_pages, Hkv, page, D), dtype)
        s["v_pages"] = _normal(gen, (n_pages, Hkv, page, D), dtype)
    if case["op"] in ("decode", "prefill"):
        s["q"] = _normal(gen, (T, H, D), dtype)
        return s
    # one projection's output: query, key and value heads of a token in one row
    qkv = _normal(gen, (T, H + 2 * Hkv, D), dtype)
    s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    s["q_weight"] = 1.0 + 0.2 * _normal(gen, (D,), torch.float32)
    s["k_weight"] = 1.0 + 0.2 * _normal(gen, (D,), torch.float32)
    R = case["rot"]
    s["inv_freq"] = (BASE ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)).float()
    s["position"] = torch.cat([torch.arange(b, b + n, **i32) for n, b in zip(new, before)])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2504_01337_amd import c2r
        s["c2r"] = c2r
        if case["op"] != "rotate":
            s["cache"] = c2r.PagedKVCache(s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    op = case["op"]
    if op in ("append", "rotate"):
        q, k = (_norm_rope(s[n], s[n + "_weight"], s["inv_freq"], s["position"], case) for n in "qk")
        if op == "rotate":
            return {"q": q, "k": k}
        slots = _slots(s, case)
        s["k_pages"][slots[0], :, slots[1]] = k
        s["v_pages"][slots[0], :, slots[1]] = s["v"]
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return _decode(s, case) if op == "decode" else _prefill(s, case)


def _run_own(s, case):
    c2r, op = s["c2r"], case["op"]
    if op == "rotate":
        q, k = c2r.qk_norm_rope(s["q"], s["k"], s["inv_freq"], s["position"], s["q_weight"], s["k_weight"], EPS,
                                neighbours=case["pairs"] == "neighbours")
        return {"q": q, "k": k}
    if op == "append":
        q = c2r.qk_norm_rope_append(s["q"], s["k"], s["v"], s["cache"], s["inv_freq"], s["q_start"], None, s["q_weight"],
                                    s["k_weight"], EPS, neighbours=case["pairs"] == "neighbours")
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if op == "decode":
        return c2r.attention_decode(s["q"], s["cache"], window=case["window"], sinks=case["sinks"], max_kv_len=max(s["total"]))
    return c2r.attention_prefill(s["q"], s["cache"], s["q_start"], max(s["new"]), window=case["window"], sinks=case["sinks"],
                                 max_kv_len=max(s["total"]))


# ---- the plain forms ---------------------------------------------------------------------------------------

def _norm_rope(x, weight, inv_freq, position, case):
    """x[T, heads, D] in 32 bits.  The angle alone is taken in 64: at position 30000 a 32-bit product of position and
    frequency is 1e-3 radians off."""
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    R = case["rot"]
    angle = position[:, None, None].double() * inv_freq.double()
    c, sn = torch.cos(angle).float(), torch.sin(angle).float()
    if case["pairs"] == "halves":
        a, b = y[..., :R // 2], y[..., R // 2:R]
        out = [a * c - b * sn, b * c + a * sn]
    else:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        out = [torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)]
    return torch.cat(out + [y[..., R:]], -1).to(x.dtype)


def _slots(s, case):
    """(page, slot in it) of every new token."""
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), s["q_start"].diff())
    index = s["position"].long()
    return s["table"][seq, index // case["page"]].long(), index % case["page"]


def _sees(p, j, case):
    see = j <= p
    if case["window"]:
        see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    return see


def _softmax_sum(score, see, v):
    """sum_j softmax_j(score) v_j over the visible j."""
    score = score.masked_fill(~see, float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _decode(s, case):
    H, Hkv, D, B = case["heads"], case["kv_heads"], case["dim"], case["seqs"]
    pages = s["table"].long().clamp(min=0)
    k, v = (s[n][pages].transpose(1, 2).reshape(B, Hkv, -1, D) for n in ("k_pages", "v_pages"))
    j = torch.arange(k.shape[2], device="cuda")
    see = _sees(s["kv_len"][:, None, None, None] - 1, j, case)
    score = torch.matmul(s["q"].float().view(B, Hkv, H // Hkv, D), k.float().transpose(2, 3)) * D ** -0.5
    return _softmax_sum(score, see, v.float()).view(B, H, D).to(s["q"].dtype)


def _gather(s, b, kind):
    """[Hkv, cached tokens, D] of sequence b."""
    page = s["case"]["page"]
    rows = s[kind][s["table"][b, :-(-s["total"][b] // page)].long()]
    return rows.transpose(0, 1).flatten(1, 2)[:, :s["total"][b]]


def _prefill(s, case):
    H, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
    G, out = H // Hkv, torch.empty_like(s["q"])
    for b, (n, before) in enumerate(zip(s["new"], s["before"])):
        q = s["q"][s["starts"][b]:s["starts"][b + 1]].float()
        k, v = _gather(s, b, "k_pages").float(), _gather(s, b, "v_pages").float()
        p = torch.arange(before, before + n, device="cuda")[:, None]
        see = _sees(p, torch.arange(before + n, device="cuda"), case)
        for h in range(H):
            o = _softmax_sum(torch.matmul(q[:, h], k[h // G].t()) * D ** -0.5, see, v[h // G])
            out[s["starts"][b]:s["starts"][b + 1], h] = o.to(out.dtype)
    return out


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    D, R, page = case["dim"], case["rot"], case["page"]
    if case["op"] in ("append", "rotate"):
        half = R // 2
        first = torch.arange(half, device="cuda") if case["pairs"] == "halves" else 2 * torch.arange(half, device="cuda")
        second = first + (half if case["pairs"] == "halves" else 1)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           torch.outer(s["position"].double(), s["inv_freq"].double()))[:, None]
        res = {}
        for n in "qk":
            x = s[n].double()
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * s[n + "_weight"].double()
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            res[n] = x
        if case["op"] == "rotate":
            return res
        out = {"q": res["q"]}
        for n, rows in (("k", res["k"]), ("v", s["v"].double())):
            cache = s[n + "_pages"].double()
            for b in range(case["seqs"]):
                for at in range(s["before"][b] // page, -(-s["total"][b] // page)):
                    lo, hi = max(at * page, s["before"][b]), min((at + 1) * page, s["total"][b])
                    t = s["starts"][b] + lo - s["before"][b]
                    cache[int(s["table"][b, at]), :, lo - at * page:hi - at * page] = rows[t:t + hi - lo].transpose(0, 1)
            out[n + "_pages"] = cache
        return out
    G, W, S = case["heads"] // case["kv_heads"], case["window"], case["sinks"]
    if work(case)["flops"] > 2e12:
        return None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (n, before) in enumerate(zip(s["new"], s["before"])):
        k, v = _gather(s, b, "k_pages"), _gather(s, b, "v_pages")
        for lo in range(0, n, 2048):
            hi = min(n, lo + 2048)
            # of this block of queries: the keys up to its last one, from its first one's window on and the first ones
            start = max(0, before + lo - W + 1) if W else 0
            keys = torch.arange(start, before + hi, device="cuda")
            if W and S:
                keys = torch.cat([torch.arange(min(S, start), device="cuda"), keys])
            p = torch.arange(before + lo, before + hi, device="cuda")[:, None]
            hidden = keys > p
            if W:
                hidden |= (keys <= p - W) & (keys >= S)
            for h in range(case["heads"]):
                kk, vv = k[h // G][keys].double(), v[h // G][keys].double()
                rows = slice(s["starts"][b] + lo, s["starts"][b] + hi)
                e = (s["q"][rows, h].double() @ kk.t()) / math.sqrt(D)
                e[hidden] = -math.inf
                out[rows, h] = torch.softmax(e, -1) @ vv
    return out
