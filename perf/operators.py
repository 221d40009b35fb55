"""The operators that stand around the MoE feed-forward layer in a decoder layer, for a token being generated: sizes, inputs, one
pass through the public entry points or through plain torch operations, and what the result is in 64-bit arithmetic.

A case's "op":

  norm   moe_add_norm: residual addition, root-mean-square norm, output in the activations' type and in e4m3 with scales
  write  moe_kv_write: new keys and values into the pages of a cache, quantised on the way where the cache is e4m3
  read   moe_kv_read: rows of the cache gathered back into a plain tensor
  attn   moe_attn_decode: attention of one new token per sequence over the paged cache

4096 columns and 64 heads of 64 are the CPM-2-MoE layer; groups of query heads over heads of 128 are ordinary decoders.
"""
import math

import torch

own = False

_MAX = 448.0             # largest e4m3 value
_TINY = 2.0 ** -126      # a scale is a normal number
_EPS = 1e-6


def _norm(name, T, d, dtype="bf16", residual=1, y=1, q=0, group=0):
    return dict(name=name, op="norm", T=T, d=d, dtype=dtype, residual=residual, y=y, q=q, group=group)


def _rows(name, op, n, heads, dim, page, dtype="bf16", cache="bf16", skip=0):
    return dict(name=name, op=op, n=n, heads=heads, dim=dim, page=page, dtype=dtype, cache=cache, skip=skip)


def _attn(name, B, length, heads, kv_heads, dim, page, dtype="bf16", cache="bf16", ragged=1, window=0):
    return dict(name=name, op="attn", B=B, length=length, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype,
                cache=cache, ragged=ragged, window=window)


def listed():
    return [
        # one token being generated: the smallest call
        _norm("norm-1", 1, 4096),
        # a prompt of 4096 tokens, also in 8 bits for the projection that follows
        _norm("norm-4096-e4m3", 4096, 4096, q=1),
        # a large batch of tokens
        _norm("norm-65536", 65536, 4096),
        # forty sequences generating one token each
        _rows("write-40", "write", 40, 64, 64, 16),
        # the keys and values of a prompt into an 8-bit cache, with some padding tokens that have no slot
        _rows("write-16384-e4m3", "write", 16384, 8, 128, 64, cache="e4m3", skip=13),
        # a short odd stretch of an 8-bit cache
        _rows("read-777-e4m3", "read", 777, 8, 128, 16, cache="e4m3"),
        # a long sequence's keys and values as a plain tensor
        _rows("read-32768", "read", 32768, 64, 64, 32),
        # one sequence of some hundred tokens
        _attn("attn-1x500", 1, 500, 64, 64, 64, 16, ragged=0),
        # forty sequences of up to 2048 tokens, every head with keys of its own
        _attn("attn-40x2048", 40, 2048, 64, 64, 64, 16),
        # one very long sequence, four query heads to a key head: all of the work is in the split of its length
        _attn("attn-1x131072", 1, 131072, 32, 8, 128, 64, ragged=0),
        # a full server: 256 sequences of up to 8192 tokens in an 8-bit cache, eight query heads to a key head
        _attn("attn-256x8192-e4m3", 256, 8192, 64, 8, 128, 64, cache="e4m3"),
        # single precision, an odd group, a head width between the usual ones, a sliding window
        _attn("attn-f32-9x3001", 9, 3001, 12, 4, 80, 32, dtype="f32", cache="f32", window=1500),
    ]


def _log_int(rng, lo, hi):
    n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))
    return min(hi, n | 1) if n < 10 or rng.random() < 0.5 else n - n % 10


def _drawn(c):
    del c["name"]
    return c


def draw(rng):
    pick = rng.random()
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if pick < 0.25:
        d = rng.choice([64, 72, 320, 512, 1000, 1024, 2048, 4096, 4096, 5120, 8192, 12288])
        q = rng.choice([0, 1])
        return _drawn(_norm("", _log_int(rng, 1, min(65536, (1 << 27) // d)), d, dtype, rng.choice([1, 1, 0]), 1 if not q else rng.choice([0, 1]), q,
                            rng.choice([0, 0, 64, 128]) if q and d % 128 == 0 else 0))
    cache = rng.choice(["bf16", "bf16", "e4m3", "e4m3"] if dtype == "bf16" else ["f32", "f32", "bf16", "e4m3"])
    dim = rng.choice([64, 64, 80, 112, 128, 128, 128, 160, 256])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if pick < 0.5:
        heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40, 64])
        return _drawn(_rows("", "write" if pick < 0.375 else "read", _log_int(rng, 1, min(65536, (1 << 27) // (heads * dim))), heads, dim, page,
                            dtype, cache, rng.choice([0, 0, 7])))
    kv_heads, group = rng.choice([(64, 1), (40, 1), (32, 1), (16, 2), (8, 4), (8, 4), (8, 8), (8, 5), (4, 7), (4, 8), (2, 16), (1, 32), (1, 71)])
    B = _log_int(rng, 1, 256)
    most = (1 << 29) // (B * kv_heads * dim)
    return _drawn(_attn("", B, _log_int(rng, 1, max(2, min(131072, most))), kv_heads * group, kv_heads, dim, page, dtype, cache,
                        rng.choice([0, 1, 1]), rng.choice([0, 0, 0, 100, 1024])))


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def _width(name):
    return {"bf16": 2, "f32": 4, "e4m3": 1}[name]


def _lens(case):
    """The sequences' lengths: all alike, or spread evenly from 0 to the longest, in an order that mixes them."""
    B, length = case["B"], case["length"]
    if not case["ragged"] or B == 1:
        return [length] * B
    return [length * ((b * 157) % B) // (B - 1) if B % 157 else length * b // (B - 1) for b in range(B)]


def _spans(case):
    """How many cached tokens each sequence attends to."""
    return [min(n, case["window"]) if case["window"] else n for n in _lens(case)]


def work(case):
    es = _width(case["dtype"])
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        moved = T * d * (es * (1 + 2 * case["residual"] + case["y"]) + case["q"]) + d * es
        moved += 4 * T * (d // case["group"] if case["group"] else 1) * case["q"]
        return {"bytes": moved, "flops": 6 * T * d}
    cs = _width(case["cache"])
    if case["op"] in ("write", "read"):
        n = case["n"] - (case["n"] // case["skip"] if case["skip"] else 0)
        rows = 2 * n * case["heads"]
        return {"bytes": rows * (case["dim"] * (es + cs) + (4 if cs == 1 else 0)) + 4 * case["n"], "flops": 3 * rows * case["dim"]}
    rows = 2 * sum(_spans(case)) * case["kv_heads"]
    heads = case["B"] * case["heads"]
    return {"bytes": rows * (case["dim"] * cs + (4 if cs == 1 else 0)) + heads * (2 * es * case["dim"] + 4),
            "flops": 4 * sum(_spans(case)) * case["heads"] * case["dim"]}


def _normal(seed, tensor, shape, dtype, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + tensor)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _pages(seed, tensor, case, pages, heads):
    """Pages [pages, heads, page, dim] as a program's earlier tokens have filled them, and the rows' scales."""
    shape = (pages, heads, case["page"], case["dim"])
    if case["cache"] != "e4m3":
        return _normal(seed, tensor, shape, _type(case["cache"])), None
    rows = _normal(seed, tensor, shape, torch.bfloat16)
    scale = (rows.abs().amax(3).float() / _MAX).clamp_min(_TINY)
    return (rows.float() / scale[..., None]).to(torch.float8_e4m3fn), scale


def _permutation(seed, tensor, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + tensor)
    return torch.randperm(n, generator=g, device="cuda")


def prepare(case, seed):
    dt = _type(case["dtype"])
    state = {"case": case}
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        state["x"] = _normal(seed, 1, (T, d), dt)
        state["residual"] = _normal(seed, 2, (T, d), dt, 3.0) if case["residual"] else None
        state["weight"] = _normal(seed, 3, (d,), dt, 0.1).add_(1.0)
        state["sum"] = torch.empty_like(state["x"]) if case["residual"] else None
        state["y"] = torch.empty_like(state["x"]) if case["y"] else None
        state["q"] = torch.empty((T, d), dtype=torch.float8_e4m3fn, device="cuda") if case["q"] else None
        groups = d // case["group"] if case["group"] else 1
        state["q_scale"] = torch.empty((T, groups), dtype=torch.float32, device="cuda") if case["q"] else None
        return state
    page = case["page"]
    if case["op"] in ("write", "read"):
        n, heads, dim = case["n"], case["heads"], case["dim"]
        pages = -(-n // page) + 3
        state["k_pages"], state["k_scale"] = _pages(seed, 1, case, pages, heads)
        state["v_pages"], state["v_scale"] = _pages(seed, 2, case, pages, heads)
        at = torch.arange(n, device="cuda")
        slots = _permutation(seed, 3, pages)[at // page] * page + at % page
        if case["skip"]:
            slots[case["skip"] - 1::case["skip"]] = -1
        state["slots"] = slots.int()
        if case["op"] == "write":
            # the keys and values lie in the rows of one projection's output
            kv = _normal(seed, 4, (n, 2, heads, dim), dt)
            state["k"], state["v"] = kv[:, 0], kv[:, 1]
        else:
            state["k"] = torch.empty((n, heads, dim), dtype=dt, device="cuda")
            state["v"] = torch.empty((n, heads, dim), dtype=dt, device="cuda")
        return state
    lens = _lens(case)
    per = max(1, -(-case["length"] // page))
    pages = case["B"] * per
    state["k_pages"], state["k_scale"] = _pages(seed, 1, case, pages, case["kv_heads"])
    state["v_pages"], state["v_scale"] = _pages(seed, 2, case, pages, case["kv_heads"])
    state["table"] = _permutation(seed, 3, pages).int().reshape(case["B"], per)
    state["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # logits with a spread of two: attention that picks some of its tokens
    state["q"] = _normal(seed, 4, (case["B"], case["heads"], case["dim"]), dt, 2.0)
    state["out"] = torch.empty_like(state["q"])
    state["lse"] = torch.empty((case["B"], case["heads"]), dtype=torch.float32, device="cuda")
    return state


def _quantised(v):
    """v [..., n] as e4m3 values and one scale for each last axis."""
    scale = (v.abs().amax(-1) / _MAX).clamp_min(_TINY)
    return (v / scale[..., None]).clamp(-_MAX, _MAX).to(torch.float8_e4m3fn), scale


def _plain_norm(s):
    c = s["case"]
    total = s["x"].float() + s["residual"].float() if c["residual"] else s["x"].float()
    n = total * torch.rsqrt(total.square().mean(1, keepdim=True) + _EPS) * s["weight"].float()
    out = {}
    if c["residual"]:
        out["sum"] = total.to(s["x"].dtype)
    if c["y"]:
        out["y"] = n.to(s["x"].dtype)
    if c["q"]:
        q, scale = _quantised(n.reshape(c["T"], -1, c["group"] or c["d"]))
        out["q"], out["q_scale"] = q.reshape(n.shape), scale
    return out


def _plain_write(s):
    page = s["case"]["page"]
    at = s["slots"].long()
    at = at[at >= 0]
    for name in ("k", "v"):
        rows = s[name][s["slots"] >= 0].float()
        if s["case"]["cache"] == "e4m3":
            rows, scale = _quantised(rows)
            s[name + "_scale"][at // page, :, at % page] = scale
            s[name + "_pages"].view(torch.uint8)[at // page, :, at % page] = rows.view(torch.uint8)
        else:
            s[name + "_pages"][at // page, :, at % page] = rows.to(s[name + "_pages"].dtype)
    return _cache(s)


def _cache(s):
    return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale") if s[n] is not None}


def _values(s, name, index, slot, real=torch.float32):
    """Rows of the cache as `real` numbers: [..., heads, dim] for the pages `index` and the places `slot` in them."""
    pages = s[name + "_pages"]
    raw = pages.view(torch.uint8)[index, :, slot].view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else pages[index, :, slot]
    return raw.to(real) if s[name + "_scale"] is None else raw.to(real) * s[name + "_scale"][index, :, slot].to(real)[..., None]


def _plain_read(s):
    at = s["slots"].long().clamp_min(0)
    there = (s["slots"] >= 0)[:, None, None]
    page = s["case"]["page"]
    return {n: torch.where(there, _values(s, n, at // page, at % page), 0.0).to(s[n].dtype) for n in ("k", "v")}


def _attention(s, real):
    c = s["case"]
    B, heads, dim = s["q"].shape
    kv = c["kv_heads"]
    at = torch.arange(c["length"], device="cuda")
    index, slot = s["table"].long()[:, at // c["page"]], (at % c["page"]).expand(B, -1)
    lens = s["lens"][:, None]
    seen = at < lens
    if c["window"]:
        seen = seen & (at >= lens - c["window"])
    k = _values(s, "k", index, slot, real).permute(0, 2, 1, 3).contiguous()              # [B, kv, length, dim]
    q = s["q"].to(real).reshape(B, kv, -1, dim).transpose(2, 3).contiguous()             # [B, kv, dim, group]
    logits = torch.matmul(k, q).transpose(2, 3) / math.sqrt(dim)                         # [B, kv, group, length]
    del k
    logits = logits.masked_fill(~seen[:, None, None], -math.inf)
    top = logits.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(logits - top)
    del logits
    total = p.sum(3, keepdim=True)
    v = _values(s, "v", index, slot, real).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(p.contiguous(), v) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).reshape(B, heads)
    return out.reshape(B, heads, dim), lse


def _plain_attn(s):
    out, lse = _attention(s, torch.float32)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _keep(s):
    """The descriptions and the workspace that a program makes once for its cache."""
    import paper_2106_10715_amd as M
    c = s["case"]
    s["M"] = M
    if c["op"] == "norm":
        s["cfg"] = M.NormCfg.make(c["T"], c["d"], c["dtype"], eps=_EPS, q_group=c["group"])
        return
    pages, heads, page, dim = s["k_pages"].shape
    s["cfg"] = M.KvCfg.make(pages, page, heads, dim, c["dtype"], c["cache"])
    if c["op"] == "attn":
        s["attn"] = M.AttnCfg.make(c["B"], c["heads"], s["table"].shape[1], window=c["window"])
        s["ws"] = torch.empty(M.moe_attn_workspace_bytes(s["cfg"], s["attn"]), dtype=torch.uint8, device="cuda")


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[op](s)
    if "M" not in s:
        _keep(s)
    M = s["M"]
    if op == "norm":
        M.moe_add_norm(s["cfg"], s["x"], s["residual"], s["weight"], s["sum"], s["y"], s["q"], s["q_scale"])
        return {n: s[n] for n in ("sum", "y", "q", "q_scale") if s[n] is not None}
    if op == "write":
        M.moe_kv_write(s["cfg"], s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
        return _cache(s)
    if op == "read":
        M.moe_kv_read(s["cfg"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["slots"], s["k"], s["v"])
        return {"k": s["k"], "v": s["v"]}
    M.moe_attn_decode(s["cfg"], s["attn"], s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["lens"],
                      s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _exact_quantised(v):
    """Rows of 64-bit values: the nearest e4m3 value (ties to even) of each over its row's scale, and the scales."""
    scale = (v.abs().amax(-1) / _MAX).clamp_min(_TINY)
    r = v / scale[..., None]
    e = torch.frexp(r).exponent.clamp_min(-5) - 4          # three bits below the leading one; 2^-9 is the smallest step
    return torch.ldexp(torch.round(torch.ldexp(r, -e)), e).clamp(-_MAX, _MAX), scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        v = s["x"].double()
        out = {}
        if case["residual"]:
            v = v + s["residual"].double()
            out["sum"] = v
        n = s["weight"].double() * v / torch.sqrt((v * v).sum(1, keepdim=True) / case["d"] + _EPS)
        if case["y"]:
            out["y"] = n
        if case["q"]:
            q, scale = _exact_quantised(n.view(case["T"], -1, case["group"] or case["d"]))
            out["q"], out["q_scale"] = q.view(n.shape), scale
        return out
    page = case["page"]
    if case["op"] == "write":
        out = {n: t.double() for n, t in _cache(s).items()}
        keep = s["slots"] >= 0
        at = s["slots"][keep].long()
        for name in ("k", "v"):
            rows = s[name][keep].double()
            if case["cache"] == "e4m3":
                rows, out[name + "_scale"][at // page, :, at % page] = _exact_quantised(rows)
            out[name + "_pages"][at // page, :, at % page] = rows
        return out
    if case["op"] == "read":
        out = {}
        for name in ("k", "v"):
            flat = s[name + "_pages"].transpose(1, 2).double()                       # [pages, page, heads, dim]
            if s[name + "_scale"] is not None:
                flat = flat * s[name + "_scale"].transpose(1, 2).double().unsqueeze(3)
            flat = torch.cat([flat.flatten(0, 1), flat.new_zeros((1, *flat.shape[2:]))])
            out[name] = flat[s["slots"].long()]                                      # slot -1 is the row of zeros
        return out
    # one sequence after the other, one key head after the other where sequences are long
    B, heads, dim = s["q"].shape
    kv = case["kv_heads"]
    out = torch.zeros((B, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((B, heads), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        used = s["table"][b, first // page:-(-n // page)].long()
        cut = slice(first % page, first % page + n - first)
        rows = {}
        for name in ("k", "v"):
            r = s[name + "_pages"].view(torch.uint8)[used].view(s[name + "_pages"].dtype).double()       # [pages, kv, page, dim]
            if s[name + "_scale"] is not None:
                r = r * s[name + "_scale"][used].double()[..., None]
            rows[name] = r.transpose(0, 1).reshape(kv, -1, dim)[:, cut]
        q = s["q"][b].double().view(kv, heads // kv, dim)
        w = (q.unsqueeze(2) * rows["k"].unsqueeze(1)).sum(3) * dim ** -0.5 if n * heads * dim < 1 << 27 else torch.bmm(q, rows["k"].transpose(1, 2).contiguous()) * dim ** -0.5
        lse[b] = torch.logsumexp(w, 2).reshape(-1)
        out[b] = torch.bmm(torch.exp(w - lse[b].view(kv, -1, 1)), rows["v"].contiguous()).reshape(heads, dim)
    return {"out": out, "lse": lse}
