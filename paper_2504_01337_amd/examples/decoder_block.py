"""A decoder block around the MoE layer, and a stack of them that takes prompts and then a token at a time.

    x = x + attention(norm(x)) . W_o        add_rms_norm, qk_norm_rope_append, then attention_prefill or attention_decode
    x = x + moe(norm(x))                    C2RLayer

Requests may have low-rank adapters of their own beside the two projections (adapters), may begin with one prompt that is kept and read once
for all of them (Decoder.share, attention_decode_shared), and their answers are scored against a vocabulary (Decoder.logprobs, token_logprobs).

    python -m paper_2504_01337_amd.examples.decoder_block                     # small, fp32
    python -m paper_2504_01337_amd.examples.decoder_block --workload C3       # 2048 wide, 60 experts + shared, bf16
    python -m paper_2504_01337_amd.examples.decoder_block --adapters 3 --common 400 --vocab 1000

Weights are random (workloads.py); hidden states stand in for embedded tokens, and the last block's output is the next token's
input.  The projections are torch's."""
import argparse
import time

import torch

from paper_2504_01337_amd import c2r, workloads as wl


def rms_norm(x, eps=1e-6):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps)).to(x.dtype)


class DecoderBlock:
    """One block's weights; its cache belongs to the batch that is being served."""

    LAYERS = 4      # row counts whose MoE layer (buffers of its own, made for one number of rows) is kept, the last ones used

    def __init__(self, w: wl.Workload, heads, kv_heads, head_dim, window=0, sinks=0, seed=0, device="cuda"):
        self.w, self.heads, self.kv_heads, self.head_dim, self.window, self.sinks = w, heads, kv_heads, head_dim, window, sinks
        self.dtype = torch.bfloat16 if w.dtype == "bf16" else torch.float32
        gen = torch.Generator(device=device).manual_seed(seed)
        on = lambda a, dtype=None: None if a is None else torch.from_numpy(a).to(device, dtype)
        normal = lambda *s: torch.randn(s, generator=gen, device=device).mul_(s[1] ** -0.5).to(self.dtype)
        self.w_qkv, self.w_o = normal((heads + 2 * kv_heads) * head_dim, w.d), normal(w.d, heads * head_dim)
        self.q_weight, self.k_weight = (1 + 0.1 * torch.randn(head_dim, generator=gen, device=device) for _ in "qk")
        self.inv_freq = (10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().to(device)
        Wg, bias = wl.router(w)
        self.Wg, self.bias = on(Wg), on(bias)
        self.experts = [on(a, self.dtype) for a in wl.expert_weights(w)]
        self.shared = [on(a, self.dtype) for a in wl.shared_expert_weights(w)] if w.F_shared else None
        # collaborator lists of each expert, profiled on random rows
        idx, _, _ = c2r.route(on(wl.hidden(w, max(w.T_profile // 16, w.T)), self.dtype), self.Wg, self.bias, w.K)
        self.collab, _ = c2r.collaborators(c2r.build_coactivation(idx, w.E), w.Tc)
        self.moe = {}
        self.adapters = None

    def add_adapters(self, n, rank, scale=1.0, seed=0):
        """n adapters beside both projections, for requests to choose from: (A, B) of each, and their scales."""
        dev = self.w_qkv.device
        gen = torch.Generator(device=dev).manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device=dev).mul_(s[2] ** -0.5).to(self.dtype)
        pair = lambda w: (normal(n, rank, w.shape[1]), normal(n, w.shape[0], rank))
        self.adapters = (pair(self.w_qkv), pair(self.w_o), torch.full((n,), scale, device=dev))

    def _project(self, x, which, adapter):
        """Rows through the query, key and value projection (0) or the output's (1), with the requests' adapters."""
        y = torch.nn.functional.linear(x, (self.w_qkv, self.w_o)[which])
        if adapter is not None and self.adapters is not None:
            A, B = self.adapters[which]
            c2r.adapters(x, adapter, A, B, y, self.adapters[2], out=y)
        return y

    def cache(self, n_pages, page_size, batch, max_pages):
        return c2r.PagedKVCache.empty(n_pages, page_size, self.kv_heads, self.head_dim, batch, max_pages, self.dtype)

    def forward(self, x, cache, q_start=None, max_new=1, max_kv_len=0, adapter=None, shared=None):
        """x[T, d]: the new rows of all sequences, which cache.kv_len already counts.  q_start[batch + 1]: where each sequence's
        begin; None: one of each.  adapter: int32[T], each row's.  shared: (shared_start, shared_len, the longest) of runs of sequences
        that begin with the same keys, for single new rows."""
        T, H, Hkv, D = len(x), self.heads, self.kv_heads, self.head_dim
        rows = c2r.add_rms_norm(x)[0]
        qkv = self._project(rows, 0, adapter).view(T, H + 2 * Hkv, D)
        q = c2r.qk_norm_rope_append(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], cache, self.inv_freq, q_start, None,
                                    self.q_weight, self.k_weight)
        if q_start is None and shared is not None:
            start, keys, longest = shared
            o = c2r.attention_decode_shared(q, cache, start, keys, window=self.window, sinks=self.sinks, max_shared_len=longest,
                                            max_own_len=max(max_kv_len - longest, 1))
        elif q_start is None:
            o = c2r.attention_decode(q, cache, window=self.window, sinks=self.sinks, max_kv_len=max_kv_len)
        else:
            o = c2r.attention_prefill(q, cache, q_start, max_new, window=self.window, sinks=self.sinks, max_kv_len=max_kv_len)
        rows, x, _, _ = c2r.add_rms_norm(self._project(o.view(T, H * D), 1, adapter), x)
        return x + self._layer(T).forward(rows)

    def _layer(self, T):
        layer = self.moe.pop(T, None)
        if layer is None:
            while len(self.moe) >= self.LAYERS:
                del self.moe[next(iter(self.moe))]
            w = self.w
            layer = c2r.C2RLayer(T, w.d, w.E, w.K, w.F, self.dtype, self.Wg, self.bias, self.collab, *self.experts, shared=self.shared)
        self.moe[T] = layer         # (a dict keeps its order: the last one used comes last)
        return layer


class Decoder:
    """Blocks and their caches.  All blocks of a batch share the page table and the lengths: a page is the same slots in each."""

    def __init__(self, blocks, batch, max_len, page_size=64, adapter=None, vocab=0):
        """adapter: int32[batch] on the device, each sequence's (see DecoderBlock.add_adapters; -1: none).  vocab: tokens that logprobs
        scores against (random rows)."""
        self.blocks, self.max_len, self.adapter, self.shared = blocks, max_len, adapter, None
        d = blocks[0].w.d
        self.head = torch.randn((vocab, d), generator=torch.Generator().manual_seed(vocab)).mul_(d ** -0.5).to(blocks[0].w_qkv) if vocab else None
        per = -(-max_len // page_size)
        first = blocks[0].cache(batch * per, page_size, batch, per)
        first.page_table.copy_(torch.randperm(batch * per, dtype=torch.int32).view(batch, per))
        first.kv_len.zero_()
        self.kv_len = first.kv_len
        self.caches = [first]
        for b in blocks[1:]:
            c = b.cache(batch * per, page_size, batch, per)
            self.caches.append(c2r.PagedKVCache(c.k, c.v, first.page_table, first.kv_len))
        self.lengths = [0] * batch      # kv_len as the host knows it

    def _grow(self, new):
        """The lengths with `new` more rows of each sequence; a row past max_len would have no place in the caches."""
        if len(new) != len(self.lengths) or min(new) < 0:
            raise ValueError(f"{len(self.lengths)} sequences, new rows {new}")
        lengths = [n + m for n, m in zip(self.lengths, new)]
        if max(lengths) > self.max_len:
            raise ValueError(f"sequence {lengths.index(max(lengths))} would have {max(lengths)} rows, the caches hold {self.max_len}")
        self.lengths = lengths

    def share(self, x):
        """A common beginning x[n, d] of all sequences, while they are empty: its rows go through the blocks once, as the first sequence's (with no
        adapter), whole pages of its keys become everyone's, and steps read them once for all.  Returns the last block's rows."""
        if any(self.lengths):
            raise ValueError("a common beginning comes first")
        n, batch = len(x), len(self.lengths)
        y = self._prompt(x, [n] + [0] * (batch - 1), None)
        table, size = self.caches[0].page_table, self.caches[0].k.shape[2]
        whole, part = n // size, n % size
        table[1:, :whole] = table[0, :whole]
        if part:
            here, there = table[0, whole].long(), table[1:, whole].long()
            for c in self.caches:
                c.k[there, :, :part], c.v[there, :, :part] = c.k[here, :, :part], c.v[here, :, :part]
        self.kv_len[1:] = n
        self.lengths = [n] * batch
        i32 = dict(dtype=torch.int32, device=x.device)
        self.shared = (torch.tensor([0, batch], **i32), torch.tensor([n], **i32), n)
        return y

    def logprobs(self, x, tokens=None, n_top=0):
        """token_logprobs of the last block's rows x[T, d]."""
        return c2r.token_logprobs(torch.nn.functional.linear(c2r.add_rms_norm(x)[0], self.head), tokens, n_top)

    def reset(self):
        """Empty sequences."""
        if self.shared is not None:             # (pages that were everyone's: each has its own again)
            table = self.caches[0].page_table
            table.copy_(torch.randperm(table.numel(), dtype=torch.int32).view(table.shape))
            self.shared = None
        self.kv_len.zero_()
        self.lengths = [0] * len(self.lengths)

    def prompt(self, x, lengths):
        """x[sum(lengths), d]: the next lengths[b] rows of each sequence."""
        return self._prompt(x, lengths, self.adapter)

    def _prompt(self, x, lengths, adapter):
        self._grow(lengths)
        new = torch.tensor(lengths, dtype=torch.int32)
        q_start = torch.zeros(len(lengths) + 1, dtype=torch.int32)
        q_start[1:] = new.cumsum(0)
        q_start, new = q_start.cuda(), new.cuda()
        self.kv_len += new
        if adapter is not None:
            adapter = torch.repeat_interleave(adapter, new, output_size=len(x))
        for block, cache in zip(self.blocks, self.caches):
            x = block.forward(x, cache, q_start, max(lengths), self.max_len, adapter)
        return x

    def step(self, x):
        """x[batch, d]: the next row of each sequence."""
        self._grow([1] * len(self.lengths))
        self.kv_len += 1
        for block, cache in zip(self.blocks, self.caches):
            x = block.forward(x, cache, max_kv_len=self.max_len, adapter=self.adapter, shared=self.shared)
        return x


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="C1", choices=[n for n, w in wl.WORKLOADS.items() if w.F and not w.E_local])
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--prompts", type=int, nargs="+", default=[500, 37, 1, 260])
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--adapters", type=int, default=0, help="low-rank adapters that the sequences have in turn")
    ap.add_argument("--common", type=int, default=0, help="rows that all sequences begin with")
    ap.add_argument("--vocab", type=int, default=0, help="score the last rows against so many tokens")
    a = ap.parse_args()
    w = wl.WORKLOADS[a.workload]
    head_dim = 64 if w.d < 1024 else 128
    def block(i):
        b = DecoderBlock(w, w.d // head_dim, w.d // head_dim, head_dim, a.window, a.sinks, seed=i)
        if a.adapters:
            b.add_adapters(a.adapters, 16, 0.1, seed=i)
        return b
    adapter = (torch.arange(len(a.prompts), dtype=torch.int32) % a.adapters).cuda() if a.adapters else None
    dec = Decoder([block(i) for i in range(a.blocks)], len(a.prompts), a.common + max(a.prompts) + a.steps + 1, adapter=adapter, vocab=a.vocab)
    common = torch.randn(a.common, w.d, device="cuda").to(dec.blocks[0].dtype)
    x = torch.randn(sum(a.prompts), w.d, device="cuda").to(dec.blocks[0].dtype)

    def timed(f, *args):
        torch.cuda.synchronize()
        t = time.perf_counter()
        y = f(*args)
        torch.cuda.synchronize()
        return y, time.perf_counter() - t
    dec.prompt(x, a.prompts)                    # (first calls load the kernels)
    dec.reset()
    if a.common:
        dec.share(common)
    y, t = timed(dec.prompt, x, a.prompts)
    print(f"{w.name}: {len(x)} rows of {len(a.prompts)} prompts through {a.blocks} blocks: {t * 1e3:.2f} ms")
    last = rms_norm(y[torch.tensor(a.prompts).cumsum(0).cuda() - 1])
    last = rms_norm(dec.step(last))

    def steps(row):
        for _ in range(a.steps):
            row = rms_norm(dec.step(row))
        return row
    last, t = timed(steps, last)
    assert torch.isfinite(last).all()
    print(f"{a.steps} steps of {len(a.prompts)} sequences: {t / a.steps * 1e3:.3f} ms a step")
    if a.vocab:
        _, entropy, top, logprob = dec.logprobs(last, n_top=min(3, a.vocab))
        print("likeliest tokens", top.tolist(), "log probabilities", [[round(v, 3) for v in r] for r in logprob.tolist()],
              "entropy", [round(v, 3) for v in entropy.tolist()])


if __name__ == "__main__":
    main()
