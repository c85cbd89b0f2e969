"""Timed cases of what a serving step of many requests needs around the blocks' two halves, over its real sizes.

A case is a dict of plain values.  `op` names the operator:

* "norm"      the residual's sum and the norm of whole rows that stand before each half of a block, with the rows in 8 bits and
              a scale each where a projection takes them so.
* "adapters"  low-rank adapters of the requests beside a projection that they share: out[t] = y[t] + c_a B_a (A_a x[t]), a the
              adapter of row t's request, if it has one.
* "shared"    one new token per sequence over the paged cache, where runs of sequences begin with the same long prefix.
* "logprobs"  log probabilities of given tokens, the entropy and the likeliest tokens, from the logits of every row.

Widths and head counts follow paper_2504_01337_amd/workloads.py (2048 and 4096 with heads of 128, 256 with heads of 64);
vocabularies, ranks and grouped heads are generic.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
E4M3_MOST = 448.0
INF = float("inf")


def _norm(name, dtype, rows, d, residual=True, dense=True, bits8=False):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "d": d, "residual": residual, "dense": dense, "bits8": bits8}


def _adapters(name, dtype, rows, d_in, d_out, rank, adapters, per_request=1, without=0.0, bits8=False):
    return {"name": name, "op": "adapters", "dtype": dtype, "rows": rows, "d_in": d_in, "d_out": d_out, "rank": rank,
            "adapters": adapters, "per_request": per_request, "without": without, "bits8": bits8}


def _shared(name, dtype, heads, kv_heads, dim, seqs, groups, prefix, after, page=64, window=0, sinks=0):
    return {"name": name, "op": "shared", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs,
            "groups": groups, "prefix": prefix, "after": after, "page": page, "window": window, "sinks": sinks}


def _logprobs(name, dtype, rows, vocab, top, given=1, stride=None, banned=0.0):
    return {"name": name, "op": "logprobs", "dtype": dtype, "rows": rows, "vocab": vocab, "stride": stride or vocab, "top": top,
            "given": given, "banned": banned}


def listed():
    return [
        # a single stream's step: latency and nothing else
        _norm("norm_1", "bf16", 1, 2048),
        # full precision, an odd number of rows of the 256-wide model, no residual yet
        _norm("norm_f32_517", "f32", 517, 256, residual=False),
        # prompts, rows for the router and, in 8 bits, for the projections
        _norm("norm_8bits_8192", "bf16", 8192, 2048, bits8=True),
        # a single request with an adapter beside the query, key and value projection
        _adapters("adapters_1", "bf16", 1, 2048, 6144, 16, 8),
        # a decoding batch of an odd size, a row for each request, many adapters of a high rank, some requests without
        _adapters("adapters_131", "bf16", 131, 4096, 6144, 64, 20, without=0.2),
        # prompts whose rows come in 8 bits
        _adapters("adapters_8bits_8192", "bf16", 8192, 2048, 6144, 16, 5, per_request=500, bits8=True),
        # four answers to one prompt
        _shared("shared_4_2000", "bf16", 16, 16, 128, 4, 1, 2000, 200),
        # a serving batch of an odd size behind one long system prompt, grouped heads
        _shared("shared_131_8000", "bf16", 32, 8, 128, 131, 1, 8000, 500, page=16),
        # several prompts with ragged numbers of sequences behind them, odd pages
        _shared("shared_groups_64", "bf16", 16, 16, 128, 64, 5, 4000, 2000, page=48),
        # the last row of a single stream, with alternatives
        _logprobs("logprobs_1", "bf16", 1, 151936, 20),
        # a decoding batch in full precision, a vocabulary of an odd size, some of it ruled out
        _logprobs("logprobs_251_odd", "f32", 251, 50257, 5, banned=0.3),
        # every row of prompts: answers scored among choices
        _logprobs("logprobs_4096", "bf16", 4096, 128200, 1, given=4, stride=128256),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, its logarithm evenly spread."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "adapters", "adapters", "shared", "shared", "logprobs", "logprobs"])
    most = max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["bytes"] + w["flops"])
    while True:
        dtype = rng.choice(["bf16"] * 4 + ["f32"])
        if op == "norm":
            dense, bits8 = rng.choice([(True, False), (True, False), (False, True), (True, True)])
            case = _norm("", dtype, _spread(rng, 1, 16384), 8 * _spread(rng, 8, 2048), rng.random() < 0.8, dense, bits8)
        elif op == "adapters":
            case = _adapters("", dtype, _spread(rng, 1, 8192), 8 * _spread(rng, 16, 1024), 8 * _spread(rng, 16, 2048), 8 * _spread(rng, 1, 16),
                             _spread(rng, 1, 64), rng.choice([1, 1, 1, _spread(rng, 2, 2000)]), rng.choice([0.0, 0.0, 0.3, 0.9]),
                             dtype == "bf16" and rng.random() < 0.4)
            # (the plain form takes every adapter for every row)
            if case["rows"] * case["adapters"] * case["rank"] * (case["d_in"] + case["d_out"]) > 2e13:
                continue
        elif op == "shared":
            dim = rng.choice([64, 128, 128])
            kv_heads = rng.choice([1, 2, 4, 8, 16, 32]) if dtype == "bf16" else rng.choice([1, 2, 4])
            heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8])
            seqs = _spread(rng, 1, 256)
            window = rng.choice([0, 0, 0, 0, _spread(rng, 1, 8192)])
            case = _shared("", dtype, heads, kv_heads, dim, seqs, min(seqs, rng.choice([1, 1, 2, 3, 8])), _spread(rng, 1, 32768),
                           _spread(rng, 1, 4096), rng.choice([1, 16, 16, 32, 48, 64, 64, 128, 1000]), window,
                           rng.choice([0, 1, 4, 16, 100]) if window else 0)
            # the plain form holds the scores, and padded copies of the keys, in 32 bits
            members = max(_members(case))
            held = 4 * (case["groups"] * case["prefix"] * (kv_heads * dim + members * heads) + seqs * case["after"] * kv_heads * dim)
            if heads > 64 or held > 8e9:
                continue
        else:
            vocab = _spread(rng, 1000, 200000)
            case = _logprobs("", dtype, _spread(rng, 1, 8192), vocab, rng.choice([0, 1, 5, 20, 64]), rng.choice([0, 1, 1, 1, 4]),
                             rng.choice([vocab, -(-vocab // 64) * 64]), rng.choice([0.0, 0.0, 0.3, 0.99]))
        del case["name"]
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] * (16 if dtype == "f32" and op == "shared" else 1) <= most["flops"]:
            return case


# ---- traits of a case --------------------------------------------------------------------------------------

def _rng(case, *names):
    return random.Random(sum(7919 ** i * int(case[n]) for i, n in enumerate(names)))


def _members(case):
    """Sequences of every group: ragged numbers, one at least."""
    rng, G = _rng(case, "seqs", "groups"), case["groups"]
    cuts = sorted(rng.sample(range(1, case["seqs"]), G - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [case["seqs"]])]


def _lengths(case):
    """(prefix of every group, keys behind it of every sequence): the first ones longest, the last of several groups without a prefix."""
    rng, G = _rng(case, "seqs", "groups", "prefix", "after"), case["groups"]
    prefix = [case["prefix"]] + [int(case["prefix"] * rng.uniform(0.2, 1.0)) for _ in range(G - 1)]
    if G > 2:
        prefix[-1] = 0
    return prefix, [case["after"]] + [max(1, int(case["after"] * rng.uniform(0.05, 1.0))) for _ in range(case["seqs"] - 1)]


def _adapter_of(case):
    """The adapter of every row, -1: none.  Requests have per_request rows each, or from a tenth of it on."""
    rng = _rng(case, "rows", "adapters", "per_request", "rank")
    rows = []
    while len(rows) < case["rows"]:
        n = case["per_request"] if not rows else max(1, int(case["per_request"] * rng.uniform(0.1, 1.0)))
        a = rng.randrange(case["adapters"])
        rows += [-1 if rows and rng.random() < case["without"] else a] * n
    return rows[:case["rows"]]


def _seen(case, length, lo, hi):
    """How many of the keys lo .. hi - 1 the token at the end of `length` keys sees."""
    hi = min(hi, length)
    first = max(0, length - case["window"]) if case["window"] else 0
    return max(0, hi - max(lo, first)) + max(0, min(hi, first, case["sinks"]) - lo)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        T, d = case["rows"], case["d"]
        return {"bytes": T * d * (size * (1 + 2 * case["residual"] + case["dense"]) + case["bits8"]) + 4 * d + 4 * T * case["bits8"],
                "flops": 6.0 * T * d}
    if case["op"] == "adapters":
        ids = _adapter_of(case)
        with_one, used, r = sum(a >= 0 for a in ids), len(set(a for a in ids if a >= 0)), case["rank"]
        return {"bytes": with_one * case["d_in"] * (1 if case["bits8"] else size) + used * r * (case["d_in"] + case["d_out"]) * size
                + 2 * case["rows"] * case["d_out"] * size + 4 * case["rows"], "flops": 2.0 * with_one * r * (case["d_in"] + case["d_out"])}
    if case["op"] == "shared":
        H, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
        prefix, after = _lengths(case)
        keys, pairs, b = 0, 0, 0
        for n, L in zip(_members(case), prefix):
            mine = [(_seen(case, L + a, 0, L), _seen(case, L + a, L, L + a)) for a in after[b:b + n]]
            keys += max(p for p, _ in mine) + sum(s for _, s in mine)
            pairs += sum(p + s for p, s in mine)
            b += n
        return {"bytes": 2 * size * case["seqs"] * H * D + 2 * size * Hkv * D * keys, "flops": 4.0 * H * D * pairs}
    T, V = case["rows"], case["vocab"]
    return {"bytes": size * T * V + T * (4 + 8 * case["given"] + 8 * case["top"]), "flops": 8.0 * T * V}


# ---- inputs ------------------------------------------------------------------------------------------------

def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _inputs(case, seed):
    """Tensors of a case, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    i32 = dict(dtype=torch.int32, device="cuda")
    s = {"case": case}
    if case["op"] == "norm":
        T, d = case["rows"], case["d"]
        s["x"] = _normal(gen, (T, d), dtype)
        s["residual"] = _normal(gen, (T, d), dtype) * 3 if case["residual"] else None
        s["weight"] = 1.0 + 0.2 * _normal(gen, (d,), torch.float32)
    elif case["op"] == "adapters":
        T, n, r, d_in, d_out = case["rows"], case["adapters"], case["rank"], case["d_in"], case["d_out"]
        x = _normal(gen, (T, d_in), dtype)
        s["x_scale"] = None
        if case["bits8"]:
            s["x_scale"] = x.float().abs().amax(1) / E4M3_MOST
            x = (x.float() / s["x_scale"][:, None]).to(torch.float8_e4m3fn)
        s["x"] = x
        s["adapter"] = torch.tensor(_adapter_of(case), **i32)
        s["A"] = _normal(gen, (n, r, d_in), dtype) * d_in ** -0.5
        s["B"] = _normal(gen, (n, d_out, r), dtype) * r ** -0.5
        s["scale"] = 0.25 + torch.rand(n, generator=gen, device="cuda")
        s["y"], s["out"] = _normal(gen, (T, d_out), dtype), torch.empty((T, d_out), dtype=dtype, device="cuda")
    elif case["op"] == "shared":
        _shared_inputs(s, case, gen, dtype)
    else:
        T, V = case["rows"], case["vocab"]
        rows = _normal(gen, (T, case["stride"]), dtype).mul_(2.5)
        # a few likely tokens in every row
        rows.scatter_add_(1, torch.randint(V, (T, 8), generator=gen, device="cuda"), 12 * torch.rand((T, 8), generator=gen, device="cuda").to(dtype))
        if case["banned"]:
            rows[:, torch.rand(case["stride"], generator=gen, device="cuda") < case["banned"]] = -INF
        s["logits"] = rows[:, :V]
        s["tokens"] = torch.randint(V, (T, case["given"]), generator=gen, device="cuda", dtype=torch.int32)
    return s


def _shared_inputs(s, case, gen, dtype):
    i32 = dict(dtype=torch.int32, device="cuda")
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    members, (prefix, after) = _members(case), _lengths(case)
    start = [0]
    for n in members:
        start.append(start[-1] + n)
    group = [g for g, n in enumerate(members) for _ in range(n)]
    total = [prefix[g] + a for g, a in zip(group, after)]
    # whole pages of a prefix are the same ones for all sequences behind it; a page that it ends in is copied
    width, pages, rows, copies = max(-(-t // page) for t in total), 0, [], []
    for b, (g, t) in enumerate(zip(group, total)):
        common, need = prefix[g] // page, -(-t // page)
        first = b == start[g]
        row = list(range(pages, pages + need)) if first else rows[start[g]][:common] + list(range(pages, pages + need - common))
        pages += need if first else need - common
        if not first and prefix[g] % page:
            copies.append((row[common], rows[start[g]][common], prefix[g] % page))
        rows.append(row)
    order = torch.randperm(pages + 3, generator=gen, device="cuda").to(torch.int32)
    table = torch.tensor([r + [pages] * (width - len(r)) for r in rows], device="cuda")
    s["table"] = order[table].contiguous()
    for n in ("k_pages", "v_pages"):
        t = s[n] = _normal(gen, (pages + 3, Hkv, page, D), dtype)
        for to, of, slots in copies:
            t[order[to], :, :slots] = t[order[of], :, :slots]
    s["q"] = _normal(gen, (case["seqs"], H, D), dtype)
    s["total"], s["prefix"], s["after"], s["members"], s["start"] = total, prefix, after, members, start
    # the group of every sequence, and its place in it
    s["group"], s["place"] = torch.tensor(group, device="cuda"), torch.tensor([i for n in members for i in range(n)], device="cuda")
    s["kv_len"], s["shared_start"], s["shared_len"] = torch.tensor(total, **i32), torch.tensor(start, **i32), torch.tensor(prefix, **i32)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2504_01337_amd import c2r
        s["c2r"] = c2r
        if case["op"] == "shared":
            s["cache"] = c2r.PagedKVCache(s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"norm": _plain_norm, "adapters": _plain_adapters, "shared": _plain_shared, "logprobs": _plain_logprobs}[case["op"]](s, case)


def _run_own(s, case):
    c2r, op = s["c2r"], case["op"]
    if op == "norm":
        y, total, y8, scale = c2r.add_rms_norm(s["x"], s["residual"], s["weight"], EPS, dense=case["dense"], bits8=case["bits8"])
        return {"y": y, "sum": total, "y8": y8, "scale": scale}
    if op == "adapters":
        return c2r.adapters(s["x"], s["adapter"], s["A"], s["B"], s["y"], scale=s["scale"], x_scale=s["x_scale"], out=s["out"])
    if op == "shared":
        return c2r.attention_decode_shared(s["q"], s["cache"], s["shared_start"], s["shared_len"], window=case["window"], sinks=case["sinks"],
                                           max_shared_len=max(s["prefix"]), max_own_len=max(s["after"]))
    logprob, entropy, top_token, top_logprob = c2r.token_logprobs(s["logits"], s["tokens"], case["top"])
    return {"logprob": logprob, "entropy": entropy, "top_token": top_token, "top_logprob": top_logprob}


# ---- the plain forms ---------------------------------------------------------------------------------------

def _plain_norm(s, case):
    x, total = s["x"], None
    if s["residual"] is not None:
        x = total = (x.float() + s["residual"].float()).to(x.dtype)
    f = x.float()
    y = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * s["weight"]
    y8 = scale = None
    if case["bits8"]:
        scale = y.abs().amax(-1) / E4M3_MOST
        y8 = (y / scale[:, None]).to(torch.float8_e4m3fn)
    return {"y": y.to(x.dtype) if case["dense"] else None, "sum": total, "y8": y8, "scale": scale}


def _plain_adapters(s, case):
    """All adapters as one product each way; a row keeps what its own adapter gives."""
    n, r, d_in, d_out = case["adapters"], case["rank"], case["d_in"], case["d_out"]
    x = s["x"].float()
    if s["x_scale"] is not None:
        x = x * s["x_scale"][:, None]
    keep = (s["adapter"][:, None] == torch.arange(n, device="cuda")) * s["scale"]
    h = torch.matmul(x, s["A"].float().view(n * r, d_in).t()).view(-1, n, r) * keep[..., None]
    more = torch.matmul(h.view(-1, n * r), s["B"].float().transpose(1, 2).reshape(n * r, d_out))
    s["out"].copy_(s["y"].float() + more)
    return s["out"]


def _sees(p, j, case):
    see = j <= p
    if case["window"]:
        see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    return see


def _plain_shared(s, case):
    """The prefixes' keys against the queries of their groups, the sequences' own keys against theirs, and one softmax over both."""
    H, Hkv, D, B, G, page = case["heads"], case["kv_heads"], case["dim"], case["seqs"], case["groups"], case["page"]
    q = s["q"].float().view(B, Hkv, H // Hkv, D) * D ** -0.5
    L, M = max(s["prefix"]), max(s["members"])
    p = (s["kv_len"] - 1).long()
    # the prefixes
    pages = s["table"][s["shared_start"][:G].long(), :max(1, -(-L // page))].long()
    k, v = (s[n][pages].transpose(1, 2).reshape(G, Hkv, -1, D).float() for n in ("k_pages", "v_pages"))
    q_group = torch.zeros((G, M, Hkv, H // Hkv, D), device="cuda")
    q_group[s["group"], s["place"]] = q
    q_group = q_group.transpose(1, 2).reshape(G, Hkv, -1, D)
    of_prefix = torch.matmul(q_group, k.transpose(2, 3).contiguous()).view(G, Hkv, M, H // Hkv, -1)
    of_prefix = of_prefix[s["group"], :, s["place"]]                       # [B, Hkv, heads of a group, keys]
    j = torch.arange(k.shape[2], device="cuda")
    see = _sees(p[:, None], j, case) & (j < s["shared_len"][s["group"]][:, None])
    of_prefix = of_prefix.masked_fill(~see[:, None, None], -INF)
    # the sequences' own keys
    j = s["shared_len"][s["group"]].long()[:, None] + torch.arange(max(s["after"]), device="cuda")
    see = _sees(p[:, None], j, case)
    j = torch.minimum(j, p[:, None])
    page_of = torch.gather(s["table"].long(), 1, j // page)
    k_own, v_own = (s[n][page_of, :, j % page].float().transpose(1, 2) for n in ("k_pages", "v_pages"))   # [B, Hkv, keys, D]
    of_own = torch.matmul(q, k_own.transpose(2, 3).contiguous()).masked_fill(~see[:, None, None], -INF)
    top = torch.maximum(of_prefix.amax(-1, keepdim=True), of_own.amax(-1, keepdim=True))
    w_prefix, w_own = torch.exp(of_prefix - top), torch.exp(of_own - top)
    w_group = torch.zeros((G, M, Hkv, H // Hkv, k.shape[2]), device="cuda")
    w_group[s["group"], s["place"]] = w_prefix
    o = torch.matmul(w_group.transpose(1, 2).reshape(G, Hkv, -1, k.shape[2]), v).view(G, Hkv, M, H // Hkv, D)[s["group"], :, s["place"]]
    o = (o + torch.matmul(w_own, v_own)) / (w_prefix.sum(-1, keepdim=True) + w_own.sum(-1, keepdim=True))
    return o.reshape(B, H, D).to(s["q"].dtype)


def _plain_logprobs(s, case):
    l = s["logits"].float()
    top = l.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(l - top).sum(-1, keepdim=True))
    out = {"logprob": torch.gather(l, 1, s["tokens"].long()) - lse if case["given"] else None}
    lp = l - lse
    out["entropy"] = -(torch.exp(lp) * lp.clamp(min=-1e30)).sum(-1)
    out["top_token"] = out["top_logprob"] = None
    if case["top"]:
        # whole numbers in the order of the logits, the lower index first among equals
        bits = l.contiguous().view(torch.int32).long()
        order = torch.where(bits < 0, -0x80000000 - bits, bits) * 2 ** 32 + (2 ** 31 - torch.arange(case["vocab"], device="cuda"))
        at = torch.topk(order, case["top"], -1).indices
        out["top_token"], out["top_logprob"] = at.int(), torch.gather(lp, 1, at)
    return out


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "adapters": _exact_adapters, "shared": _exact_shared, "logprobs": _exact_logprobs}[case["op"]](s, case)


def _exact_norm(s, case):
    out = {"y": None, "sum": None, "y8": None, "scale": None}
    x = s["x"].double()
    if s["residual"] is not None:
        out["sum"] = x + s["residual"].double()
        x = out["sum"].to(s["x"].dtype).double()      # the norm is that of the sum as it is kept
    y = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["d"] + EPS) * s["weight"].double()
    if case["dense"]:
        out["y"] = y
    if case["bits8"]:
        c = y.abs().max(-1).values / E4M3_MOST
        out["scale"], out["y8"] = c, y / c[:, None]
    return out


def _exact_adapters(s, case):
    out = s["y"].double()
    for a in range(case["adapters"]):
        rows = (s["adapter"] == a).nonzero()[:, 0]
        if len(rows):
            x = s["x"][rows].to(torch.float64) if s["x_scale"] is None else s["x"].float()[rows].double() * s["x_scale"][rows, None].double()
            out[rows] += s["scale"][a].double() * ((x @ s["A"][a].double().t()) @ s["B"][a].double().t())
    return out


def _exact_shared(s, case):
    if work(case)["flops"] > 2e12:
        return None
    G, D, page = case["heads"] // case["kv_heads"], case["dim"], case["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["total"]):
        j = torch.arange(n, device="cuda")
        if case["window"]:
            j = j[(j >= n - case["window"]) | (j < case["sinks"])]
        page_of = s["table"][b].long()[j // page]
        k, v = (s[x][page_of, :, j % page].double() for x in ("k_pages", "v_pages"))     # [keys, kv heads, D]
        for h in range(case["heads"]):
            e = k[:, h // G] @ s["q"][b, h].double() / math.sqrt(D)
            out[b, h] = torch.softmax(e, 0) @ v[:, h // G]
    return out


def _exact_logprobs(s, case):
    T, parts = case["rows"], []
    for lo in range(0, T, 256):
        l = s["logits"][lo:lo + 256].double()
        lp = torch.log_softmax(l, -1)
        p = torch.softmax(l, -1)
        best = lp.sort(-1, descending=True).values[:, :case["top"]] if case["top"] > 1 else lp.max(-1, keepdim=True).values
        parts.append((torch.gather(lp, 1, s["tokens"][lo:lo + 256].long()), -torch.where(p > 0, p * lp, 0.0).sum(-1), best))
    logprob, entropy, best = (torch.cat(x) for x in zip(*parts))
    return {"logprob": logprob if case["given"] else None, "entropy": entropy, "top_token": None, "top_logprob": best if case["top"] else None}
