"""Token generation through decoder layers with the Mixture-of-Experts feed-forward layer, on this library's operators:

    h, y   = moe_add_norm(delta, h)           residual stream and its norm (also in 8 bits for the projection, with --qkv e4m3)
    q,k,v  = y W_qkv                          a plain product (torch)
    q, k   = moe_rope(q, k)                   rotary positions, in their places (--rotary)
    cache  = moe_kv_write(k, v)               into the pages, quantised where the cache is e4m3
    o      = moe_attn_decode(q, cache)        one new token per sequence over everything cached (moe_attn_decode_scored with --cap or --slopes)
    h, y   = moe_add_norm(o W_o, h)
    delta  = moe_layer_forward(y)             gate, batching, expert FFNs, combine

A prompt's tokens go through the same layers at once, with moe_attn_prompt over the cache that they have been written to.

    python examples/decode.py                                    # the CPM-2-MoE layer's sizes, 40 sequences
    python examples/decode.py --batch 8 --layers 4 --cache e4m3 --qkv e4m3 --length 8000
    python examples/decode.py --batch 4 --length 4000 --prompt --rotary --cap 30
"""
import argparse
import math
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2106_10715_amd as M  # noqa: E402


class Weights:
    """One layer's weights, random: norms, projections, gate and experts as the library packs them."""

    def __init__(self, d, heads, kv_heads, dim, moe, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda std, *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)
        self.norm_attn, self.norm_moe = 1.0 + new(0.1, d), 1.0 + new(0.1, d)
        self.qkv = new(d ** -0.5, (heads + 2 * kv_heads) * dim, d)              # [out, in]
        self.o = new((heads * dim) ** -0.5, d, heads * dim)
        self.gate = new(d ** -0.5, moe.d, moe.E)
        self.packed_gate = torch.empty(M.moe_gate_bytes(moe), dtype=torch.uint8, device="cuda")
        M.moe_pack_gate(moe, self.gate, self.packed_gate)
        self.experts = torch.empty((moe.E, M.moe_expert_bytes(moe)), dtype=torch.uint8, device="cuda")
        self.expert = lambda e: Weights.matrices(moe, seed, e)
        for e in range(moe.E):
            M.moe_pack_weights(moe, *self.expert(e), self.experts[e])
        top = self.qkv.float().abs().amax(1, keepdim=True) / 448.0
        self.qkv8, self.qkv8_scale = (self.qkv.float() / top).to(torch.float8_e4m3fn), top

    @staticmethod
    def matrices(moe, seed, e):
        g = torch.Generator(device="cuda").manual_seed(1000 * seed + e + 1)
        return [torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)
                for shape, std in (((moe.d, moe.f), moe.d ** -0.5), ((moe.d, moe.f), moe.d ** -0.5), ((moe.f, moe.d), moe.f ** -0.5))]


class Decoder:
    """A stack of layers with a paged cache for `batch` sequences of up to `room` tokens."""

    def __init__(self, batch, layers, d, heads, kv_heads, dim, f, E, k, room, page=64, cache="bf16", qkv="bf16", eps=1e-6, seed=1, rotary=None, cap=0.0,
                 slopes=False):
        """rotary: what M.RopeCfg.make takes beside the heads, or None; cap, slopes: the scores' (ALiBi's slopes: 2^(-8 (h + 1) / heads))."""
        assert heads * dim == d
        per = -(-room // page)
        self.batch, self.heads, self.kv_heads, self.dim, self.page, self.qkv = batch, heads, kv_heads, dim, page, qkv
        self.moe = M.MoeCfg.make(batch, d, f, E, k).with_packed_gate()
        self.norm = M.NormCfg.make(batch, d, "bf16", eps=eps)
        self.kv = M.KvCfg.make(batch * per, page, kv_heads, dim, "bf16", cache)
        self.attn = M.AttnCfg.make(batch, heads, per)
        self.weights = [Weights(d, heads, kv_heads, dim, self.moe, seed + i) for i in range(layers)]
        self.caches = [self.kv.empty() for _ in range(layers)]
        self.table = torch.randperm(batch * per, device="cuda").int().reshape(batch, per)
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
        self.h, self.delta, self.y, self.o = new(batch, d), new(batch, d), new(batch, d), new(batch, heads, dim)
        self.y8, self.y8_scale = (new(batch, d, dtype=torch.float8_e4m3fn), new(batch, 1, dtype=torch.float32)) if qkv == "e4m3" else (None, None)
        self.ws = new(M.moe_workspace_bytes(self.moe), dtype=torch.uint8)
        self.attn_ws = new(M.moe_attn_workspace_bytes(self.kv, self.attn), dtype=torch.uint8)
        self.rope = None if rotary is None else M.RopeCfg.make(heads, kv_heads, dim, **rotary)
        self.freqs = None if rotary is None else M.moe_rope_frequencies(self.rope).cuda()
        self.scores = M.ScoresCfg.make(cap) if cap else None
        self.slopes = torch.exp2(-8.0 * torch.arange(1, heads + 1, device="cuda") / heads) if slopes else None

    def project(self, w, y, y8, y8_scale):
        if self.qkv == "e4m3":
            return torch._scaled_mm(y8, w.qkv8.t(), scale_a=y8_scale, scale_b=w.qkv8_scale.t().contiguous(), out_dtype=torch.bfloat16)
        return torch.mm(y, w.qkv.t())

    def places(self, seq, at):
        """Slots of the tokens at these places of these sequences."""
        return self.table[seq, at // self.page] * self.page + (at % self.page).int()

    def heads_of(self, rows, positions):
        """Queries, keys and values in a projection's rows, the first two turned by their positions."""
        q, k, v = rows.view(rows.shape[0], self.heads + 2 * self.kv_heads, self.dim).split([self.heads, self.kv_heads, self.kv_heads], 1)
        if self.rope is not None:
            M.moe_rope(self.rope, positions, self.freqs, q, q, k, k)
        return q, k, v

    @staticmethod
    def in_calls(counts, most):
        """The counts of calls of prompt() that take these tokens in, up to `most` in each: the layer's buffers grow with a call's tokens."""
        left, call = list(counts), [0] * len(counts)
        for b in range(len(left)):
            while left[b] > 0:
                take = min(left[b], most - sum(call))
                call[b] += take
                left[b] -= take
                if sum(call) == most:
                    yield call
                    call = [0] * len(counts)
        if any(call):
            yield call

    def prompt(self, x, counts, first=None, end=None):
        """counts[b] further tokens of each sequence, their embeddings x [sum, d] -> their hidden states [sum, d].  first, end: what moe_attn_prompt's mask takes."""
        n = x.shape[0]
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
        counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
        starts = torch.zeros(self.batch + 1, dtype=torch.int32, device="cuda")
        starts[1:] = torch.cumsum(counts, 0)
        seq = torch.repeat_interleave(torch.arange(self.batch, device="cuda"), counts.long(), output_size=n)
        at = self.lens.long()[seq] + torch.arange(n, device="cuda") - starts.long()[seq]
        slots, positions = self.places(seq, at), at.int()
        self.lens += counts
        moe = M.MoeCfg.make(n, self.moe.d, self.moe.f, self.moe.E, self.moe.k).with_packed_gate()
        norm, attn = M.NormCfg.make(n, self.norm.d, "bf16", eps=self.norm.eps), M.PromptCfg.make(n, self.batch, self.heads, self.table.shape[1])
        ws, attn_ws = new(M.moe_workspace_bytes(moe), dtype=torch.uint8), new(M.moe_attn_prompt_workspace_bytes(self.kv, attn), dtype=torch.uint8)
        h, y, o, delta = new(n, moe.d), new(n, moe.d), new(n, self.heads, self.dim), x
        y8, y8_scale = (new(n, moe.d, dtype=torch.float8_e4m3fn), new(n, 1, dtype=torch.float32)) if self.qkv == "e4m3" else (None, None)
        residual, out = None, new(n, moe.d)
        for w, cache in zip(self.weights, self.caches):
            M.moe_add_norm(norm, delta, residual, w.norm_attn, h, None if y8 is not None else y, y8, y8_scale)
            q, k, v = self.heads_of(self.project(w, y, y8, y8_scale), positions)
            M.moe_kv_write(self.kv, k, v, slots, *cache)
            M.moe_attn_prompt(self.kv, attn, self.scores, q, *cache, self.table, self.lens, starts, first, end, self.slopes, None, o, None, attn_ws)
            torch.mm(o.view(n, -1), w.o.t(), out=out)
            M.moe_add_norm(norm, out, h, w.norm_moe, h, y)
            M.moe_layer_forward(moe, y, w.packed_gate, None, w.experts, None, out, ws)
            delta, residual = out, h
        return h.add(out)

    def step(self, x):
        """One token per sequence, its embedding x [batch, d] -> its hidden state [batch, d] (a buffer of the decoder's)."""
        at = self.lens.long()
        slots, positions = self.places(torch.arange(self.batch, device="cuda"), at), at.int()
        self.lens += 1
        delta, h = x, None
        for w, cache in zip(self.weights, self.caches):
            M.moe_add_norm(self.norm, delta, h, w.norm_attn, self.h, None if self.y8 is not None else self.y, self.y8, self.y8_scale)
            q, k, v = self.heads_of(self.project(w, self.y, self.y8, self.y8_scale), positions)
            M.moe_kv_write(self.kv, k, v, slots, *cache)
            if self.scores is not None or self.slopes is not None:
                M.moe_attn_decode_scored(self.kv, self.attn, self.scores, q, *cache, self.table, self.lens, self.slopes, None, self.o, None, self.attn_ws)
            else:
                M.moe_attn_decode(self.kv, self.attn, q, *cache, self.table, self.lens, self.o, None, self.attn_ws)
            torch.mm(self.o.view(self.batch, -1), w.o.t(), out=self.delta)
            M.moe_add_norm(self.norm, self.delta, self.h, w.norm_moe, self.h, self.y)
            M.moe_layer_forward(self.moe, self.y, w.packed_gate, None, w.experts, None, self.delta, self.ws)
            delta, h = self.delta, self.h
        return self.h.add(self.delta)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 40), ("layers", 2), ("heads", 64), ("kv-heads", 64), ("dim", 64), ("d-ff", 10240), ("experts", 32),
                        ("top", 1), ("length", 2000), ("steps", 20), ("page", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--qkv", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--prompt", action="store_true", help="take prompts of `length` tokens in first (else the caches start with random rows)")
    ap.add_argument("--rotary", action="store_true")
    ap.add_argument("--cap", type=float, default=0.0)
    ap.add_argument("--slopes", action="store_true")
    a = ap.parse_args()
    D = Decoder(a.batch, a.layers, a.heads * a.dim, a.heads, a.kv_heads, a.dim, a.d_ff, a.experts, a.top, a.length + a.steps + 8, a.page, a.cache, a.qkv,
                rotary={} if a.rotary else None, cap=a.cap, slopes=a.slopes)
    if a.prompt:
        calls = list(D.in_calls([a.length] * a.batch, min(1 << 16, (2 ** 31 - 1) // (D.moe.k * max(D.moe.d, D.moe.f)))))
        x = torch.empty((max(map(sum, calls)), a.heads * a.dim), dtype=torch.bfloat16, device="cuda").normal_()
        for _ in range(2):                                   # (the first is the warm-up)
            D.lens.zero_()
            torch.cuda.synchronize()
            t = time.perf_counter()
            for counts in calls:
                D.prompt(x[:sum(counts)], counts)
            torch.cuda.synchronize()
            s = time.perf_counter() - t
        print(f"{a.batch} prompts of {a.length} tokens, {a.layers} layers: {s * 1e3:.3f} ms, {a.batch * a.length / s:.0f} tokens/s")
    else:
        for cache in D.caches:                               # as if `length` tokens had been generated already
            for t in cache:
                if t is not None:
                    t.copy_(torch.empty(t.shape, dtype=torch.bfloat16, device="cuda").normal_()) if t.dtype != torch.float32 else t.fill_(1.0 / math.sqrt(a.dim))
        D.lens.fill_(a.length)
    x = torch.empty((a.batch, a.heads * a.dim), dtype=torch.bfloat16, device="cuda").normal_()
    for _ in range(4):
        D.step(x)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        D.step(x)
    torch.cuda.synchronize()
    s = (time.perf_counter() - t) / a.steps
    print(f"{a.batch} sequences of {a.length} tokens, {a.layers} layers: {s * 1e3:.3f} ms a step, {a.batch / s:.0f} tokens/s")


if __name__ == "__main__":
    main()
