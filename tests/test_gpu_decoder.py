"""GPU parity of the operators around the expert layer with the fp64 oracle (oracle/decoder_oracle.py) on the same stored inputs.

Tolerances, per element.  A rounding to a type is off by half a step, eps / 2 relative (bf16 2^-8, fp32 2^-24).
  norm       fp32 from the addition on: up to 54 additions of a sum of squares (one lane's, the wave's, the block's) count half in the
             root, plus the root, the addition and two products: 64 * 2^-24, and the output's rounding.
  e4m3       the scale as the norm, plus a division; a value is within half a step (2^-4 relative, 2^-10 below 2^-6) of n / scale,
             wider by what n and the scale may be off.
  attention  with A = sum p |v| and M the largest |l|: a logit is off by (D + 8) 2^-24 sum |q k| scale from its sum and 4 * 2^-24 M
             from its scaling, which changes p by as much relatively (times 2: numerator and total); sums over n tokens of
             a wave's runs, its lanes, waves and parts: (n / 16 + 64) 2^-24; weights in bf16: 2^-8; and the output's rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def normal(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TORCH[dtype]).cuda()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def within(got, ref, tol, what):
    got = np.asarray(got, np.float64)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - ref) - tol
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}: {got[at]} for {ref[at]} at {at}, off by {abs(got[at] - ref[at]):.3e} of {np.broadcast_to(tol, ref.shape)[at]:.3e}"


# ------------------------------------------------------------------------------------------- norm

NORM_REL = 64 * 2.0 ** -24


def run_norm(cfg, x, r, w, with_sum=True, with_y=True, with_q=False):
    new = lambda dt, shape: torch.full(shape, 7, dtype=torch.uint8 if dt == torch.float8_e4m3fn else dt, device="cuda").view(dt)
    T, d, dt = cfg.T, cfg.d, x.dtype
    out = dict(sum=new(dt, (T, d)) if with_sum else None, y=new(dt, (T, d)) if with_y else None,
               q=new(torch.float8_e4m3fn, (T, d)) if with_q else None,
               q_scale=new(torch.float32, (T, d // cfg.q_group if cfg.q_group else 1)) if with_q else None)
    M.moe_add_norm(cfg, x, r, w, out["sum"], out["y"], out["q"], out["q_scale"])
    torch.cuda.synchronize()
    return out


def check_norm(cfg, dtype, x, r, w, out):
    s, n = D.add_norm(f64(x), None if r is None else f64(r), f64(w), cfg.eps)
    half = HALF[dtype]
    if out["sum"] is not None:
        within(f64(out["sum"]), s, np.abs(s) * (half + 2 ** -23), "sum")
    if out["y"] is not None:
        within(f64(out["y"]), n, np.abs(n) * (half * (1 + NORM_REL) + NORM_REL), "y")
    if out["q"] is not None:
        groups = n.reshape(cfg.T, -1, cfg.q_group or cfg.d)
        scale = D.e4m3_scale(groups)
        within(f64(out["q_scale"]), scale, scale * (NORM_REL + 2 ** -23), "q_scale")
        ratio = groups / scale[..., None]
        within(f64(out["q"]).reshape(groups.shape), ratio, np.maximum(np.abs(ratio) * 2 ** -4, 2 ** -10) * (1 + 2 ** -10) + np.abs(ratio) * 4 * NORM_REL, "q")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,group", [(1, 8, 0), (1, 4096, 0), (3, 64, 32), (257, 72, 0), (5, 320, 64), (63, 512, 128), (2, 1000, 0), (33, 1024, 128),
                                       (9, 2048, 0), (4, 2056, 0), (17, 4096, 64), (3, 8192, 32), (2, 8200, 0), (5, 12288, 128), (2, 16384, 0), (3, 32768, 128), (1, 32760, 0)])
def test_norm(T, d, group, dtype):
    x, r, w = normal(1, (T, d), dtype), normal(2, (T, d), dtype, 3.0), normal(3, (d,), dtype, 0.5)
    cfg = M.NormCfg.make(T, d, dtype, q_group=group)
    check_norm(cfg, dtype, x, r, w, run_norm(cfg, x, r, w, with_q=True))
    check_norm(cfg, dtype, x, None, w, run_norm(cfg, x, None, w, with_sum=False))
    check_norm(cfg, dtype, x, r, w, run_norm(cfg, x, r, w, with_sum=False, with_y=False, with_q=True))


def test_norm_of_zeros_of_tiny_and_of_large_rows():
    """Rows of zeros have the smallest scale and no NaN; rows of denormal size and rows near the root of the largest value are exact."""
    d = 512
    x = normal(4, (6, d), "f32")
    x[0] = 0.0
    x[1] *= 1e-30
    x[2] *= 1e15
    x[3, :] = 0.0
    x[3, 77] = -5.0
    x[4] = 1.0
    w = torch.ones(d, device="cuda")
    cfg = M.NormCfg.make(6, d, "f32", eps=1e-5)
    out = run_norm(cfg, x, None, w, with_q=True)
    check_norm(cfg, "f32", x, None, w, out)
    assert f64(out["q_scale"])[0, 0] == 2.0 ** -126 and (f64(out["q"])[0] == 0).all()


def test_norm_may_write_over_its_inputs_and_keeps_nan_to_its_row():
    for T, d, dtype in ((5, 4096, "bf16"), (300, 320, "f32"), (2, 20000, "bf16")):
        x, r, w = normal(5, (T, d), dtype), normal(6, (T, d), dtype), normal(7, (d,), dtype)
        cfg = M.NormCfg.make(T, d, dtype)
        want = run_norm(cfg, x, r, w)
        x2, r2 = x.clone(), r.clone()
        M.moe_add_norm(cfg, x2, r2, w, r2, x2)
        assert torch.equal(r2, want["sum"]) and torch.equal(x2, want["y"])
        x[1, 3] = float("nan")
        got = run_norm(cfg, x, r, w, with_q=True)
        assert torch.isnan(got["y"][1]).all() and torch.isnan(got["q"][1].float()).all()
        keep = [t for t in range(T) if t != 1]
        assert torch.equal(got["y"][keep], want["y"][keep])


# ------------------------------------------------------------------------------------------- cache

TYPES = [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "bf16"), ("f32", "e4m3")]


def filled(cfg, value):
    """A cache of this value's bytes everywhere (0xff: NaN in every type)."""
    out = cfg.empty()
    for t in out:
        if t is not None:
            t.view(torch.uint8).fill_(value)
    return out


def take(pages, slots, page_size):
    raw = pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages
    rows = raw.transpose(1, 2).flatten(0, 1)[slots.long()]
    return rows.view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else rows


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,heads,dim,page", [(1, 1, 16, 16), (1, 64, 64, 16), (7, 3, 80, 32), (130, 8, 128, 64), (33, 2, 144, 16), (1000, 5, 256, 128), (5, 40, 48, 1024)])
def test_cache_write_and_read(n, heads, dim, page, dtype, cache):
    pages = (n + 40) // page + 2
    cfg = M.KvCfg.make(pages, page, heads, dim, dtype, cache)
    g = torch.Generator().manual_seed(n)
    slots = torch.randperm(pages * page, generator=g)[:n].int()
    if n > 4:
        slots[1], slots[3] = -1, pages * page                                   # no place: before and past the cache
    real = (slots >= 0) & (slots < pages * page)
    slots_d, used = slots.cuda(), slots[real].cuda()
    wide = normal(8, (n, 3 * heads * dim + 8), dtype, 4.0)                      # k and v are stretches of wider rows
    k = wide[:, heads * dim:2 * heads * dim].view(n, heads, dim)
    v = wide[:, 2 * heads * dim + 8:].view(n, heads, dim)
    if n > 4:
        k[4, 0] = 0.0
    arrays = filled(cfg, 0x5a)
    before = [None if t is None else t.clone() for t in arrays]
    M.moe_kv_write(cfg, k, v, slots_d, *arrays)
    torch.cuda.synchronize()
    left = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    left[used.long()] = False
    others = left.nonzero()[:, 0]
    for rows, t, scale, b, bs in ((k, arrays[0], arrays[2], before[0], before[2]), (v, arrays[1], arrays[3], before[1], before[3])):
        assert torch.equal(take(t, others, page).view(torch.uint8), take(b, others, page).view(torch.uint8)), "a slot that was not given has changed"
        rows = rows[real.cuda()]
        if cache != "e4m3":
            assert torch.equal(take(t, used, page), rows.to(TORCH[cache]))
            continue
        sc = f64(scale.transpose(1, 2).flatten(0, 1)[used.long()])
        want = D.e4m3_scale(f64(rows))
        within(sc, want, want * 2 ** -23, "scale")
        assert torch.equal(scale.transpose(1, 2).flatten(0, 1)[others], bs.transpose(1, 2).flatten(0, 1)[others])
        ratio = f64(rows) / want[..., None]
        within(f64(take(t, used, page)), ratio, np.maximum(np.abs(ratio) * 2 ** -4, 2 ** -10) * (1 + 2 ** -10) + np.abs(ratio) * 2 ** -21, "e4m3 value")
    # and back, into stretches of wider rows
    back = torch.full((n, 2 * heads * dim + 8), 7, dtype=TORCH[dtype], device="cuda")
    kb, vb = back[:, :heads * dim].view(n, heads, dim), back[:, heads * dim + 8:].view(n, heads, dim)
    M.moe_kv_read(cfg, *arrays, slots_d, kb, vb)
    torch.cuda.synchronize()
    assert (back[:, heads * dim:heads * dim + 8] == 7).all()
    for got, t, scale in ((kb, arrays[0], arrays[2]), (vb, arrays[1], arrays[3])):
        assert (got[~real.cuda()] == 0).all()
        want = f64(take(t, used, page))
        if scale is not None:
            want = want * f64(scale.transpose(1, 2).flatten(0, 1)[used.long()])[..., None]
        within(f64(got[real.cuda()]), want, np.abs(want) * (HALF[dtype] + 2 ** -23), "read")


def test_cache_offsets_past_32_bits():
    """A pool of over 2^32 bytes and 2^31 elements a side: rows at its far end, and attention over them."""
    pages, page, heads, dim = 33100, 64, 8, 128
    cfg = M.KvCfg.make(pages, page, heads, dim)
    arrays = cfg.empty()
    assert arrays[0].numel() > 2 ** 31
    n = 150
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32)
    at = torch.arange(n)
    slots = (table[0][at // page] * page + at % page).int().cuda()
    k, v = normal(9, (n, heads, dim), "bf16"), normal(10, (n, heads, dim), "bf16")
    M.moe_kv_write(cfg, k, v, slots, *arrays)
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    M.moe_kv_read(cfg, *arrays, slots, kb, vb)
    torch.cuda.synchronize()
    assert torch.equal(kb, k) and torch.equal(vb, v)
    q = normal(11, (1, heads, dim), "bf16")
    run_and_check(cfg, arrays, q, table.cuda(), [n])


# ------------------------------------------------------------------------------------------- attention

def cache_of(seed, cfg, table, lens, k_std=1.0, window=0):
    """A cache whose every place that is not attended to holds NaN (pages, scales), the others normal values."""
    arrays = filled(cfg, 0xff)
    page, dt = cfg.page_size, {0: "f32", 1: "bf16"}[cfg.dtype]
    slots = []
    for b, n in enumerate(lens):
        at = torch.arange(max(0, n - window) if window else 0, n)
        slots.append(table[b][at // page].long() * page + at % page)
    slots = torch.cat(slots).int().cuda()
    if slots.numel():
        k = normal(seed, (slots.numel(), cfg.heads, cfg.head_dim), dt, k_std)
        v = normal(seed + 1, (slots.numel(), cfg.heads, cfg.head_dim), dt)
        M.moe_kv_write(cfg, k, v, slots, *arrays)
    return arrays


def run_attention(cfg, arrays, q, table, lens, window=0, scale=0.0, want_lse=True):
    B, heads, dim = q.shape
    attn = M.AttnCfg.make(B, heads, table.shape[1], scale=scale, window=window)
    n = M.moe_attn_workspace_bytes(cfg, attn)
    ws = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((B, heads, dim), 7, dtype=q.dtype, device="cuda")
    lse = torch.full((B, heads), 7, dtype=torch.float32, device="cuda") if want_lse else None
    M.moe_attn_decode(cfg, attn, q, *arrays, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, ws)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xff).all(), "written past the workspace"
    return out, lse


def run_and_check(cfg, arrays, q, table, lens, window=0, scale=0.0, only=None):
    """`only`: the sequences that are compared with the oracle (all)."""
    out, lse = run_attention(cfg, arrays, q, table, lens, window, scale)
    dt = {0: "f32", 1: "bf16"}[cfg.dtype]
    B, heads, dim = q.shape
    group = heads // cfg.heads
    c = scale or 1 / math.sqrt(dim)
    pages = [f64(t) for t in arrays[:2]] if arrays[0].numel() < 1 << 26 else None
    scales = [None if t is None else f64(t) for t in arrays[2:]]
    tab = table.cpu().numpy()
    for b in range(B) if only is None else only:
        n = min(max(lens[b], 0), table.shape[1] * cfg.page_size)
        first = max(0, n - window) if window else 0
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        if pages is None:                                                       # a pool that is too large for the host
            used = torch.unique(table[b, :-(-n // cfg.page_size)].long())
            small = np.zeros(cfg.pages, np.int64)
            small[used.cpu().numpy()] = np.arange(len(used))
            k, v = (D.paged_rows(f64(t.view(torch.uint8)[used].view(t.dtype)), None if s is None else f64(s[used]), small[tab[b]], first, n)
                    for t, s in zip(arrays[:2], arrays[2:]))
        else:
            k, v = (D.paged_rows(t, s, tab[b], first, n) for t, s in zip(pages, scales))
        for j in range(heads):
            h = j // group
            qj = f64(q[b, j])
            ref, ref_lse, p = D.attention(qj, k[h], v[h], c)
            logits = c * (k[h] @ qj)
            off = (dim + 8) * 2 ** -24 * c * (np.abs(k[h]) @ np.abs(qj)).max() + 4 * 2 ** -24 * np.abs(logits).max()
            sums = (len(p) / 16 + 64) * 2 ** -24
            A = p @ np.abs(v[h])
            weights = 2 ** -8 if dt == "bf16" else 0.0
            within(f64(out[b, j]), ref, HALF[dt] * np.abs(ref) + (weights + 2 * off + 2 * sums) * A * (1 + HALF[dt]), f"sequence {b}, head {j}")
            assert abs(float(lse[b, j]) - ref_lse) <= off + sums + 2 ** -22 * abs(ref_lse) + 2 ** -22, f"lse of sequence {b}, head {j}"
    return out, lse


def tables(seed, B, per, pages):
    return torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:B * per].reshape(B, per).int()


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 255, 257, 400]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,window", [(4, 1, 64, 16, 0), (2, 3, 128, 32, 0), (1, 8, 16, 64, 0), (3, 5, 80, 16, 100), (2, 16, 48, 512, 1),
                                                         (1, 17, 128, 16, 33), (1, 33, 64, 32, 0), (2, 4, 256, 16, 0), (1, 20, 144, 128, 130)])
def test_attention_at_the_edges_of_runs_pages_and_windows(heads, group, dim, page, window, dtype, cache):
    B, per = len(EDGES), -(-400 // page)
    cfg = M.KvCfg.make(B * per + 3, page, heads, dim, dtype, cache)
    table = tables(1, B, per, cfg.pages)
    arrays = cache_of(20, cfg, table, EDGES, window=window)
    for b, n in enumerate(EDGES):                              # pages that no token of the window lies in: not even numbers of pages
        first = max(0, n - window) if window else 0
        table[b, -(-n // page):] = 2 ** 31 - 1
        table[b, :first // page] = -7
    wide = normal(22, (B, heads * group * dim + 24), dtype, 2.0)
    q = wide[:, 8:8 + heads * group * dim].view(B, heads * group, dim)
    run_and_check(cfg, arrays, q, table.cuda(), EDGES, window)


@pytest.mark.parametrize("B,length,heads,group,dim,page,dtype,cache", [
    (1, 40000, 1, 71, 128, 64, "bf16", "bf16"), (1, 33001, 2, 4, 64, 16, "bf16", "e4m3"), (2, 9999, 4, 1, 80, 32, "f32", "f32"),
    (1, 5000, 40, 1, 128, 256, "bf16", "bf16"), (3, 3001, 1, 32, 256, 16, "bf16", "e4m3"), (1, 20000, 1, 1, 256, 16, "f32", "bf16"), (65, 700, 3, 2, 64, 16, "f32", "e4m3")])
def test_attention_split_over_long_sequences(B, length, heads, group, dim, page, dtype, cache):
    per = -(-length // page)
    cfg = M.KvCfg.make(B * per, page, heads, dim, dtype, cache)
    table = tables(2, B, per, cfg.pages)
    lens = [length - (37 * b) % length for b in range(B)]
    arrays = cache_of(30, cfg, table, lens)
    q = normal(32, (B, heads * group, dim), dtype, 2.0)
    a = run_and_check(cfg, arrays, q, table.cuda(), lens, only=sorted({0, B // 2, B - 1}))
    b = run_attention(cfg, arrays, q, table.cuda(), lens)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), "two runs differ"


@pytest.mark.parametrize("B,heads,group,dim,cache,most", [
    (1, 3, 2, 64, "bf16", 768), (2, 32, 1, 64, "bf16", 1024), (16, 8, 1, 64, "e4m3", 1536), (4, 64, 1, 64, "bf16", 2048), (32, 8, 8, 128, "e4m3", 2048),
    (5, 2, 16, 128, "bf16", 768), (16, 4, 4, 128, "bf16", 1024), (3, 1, 40, 128, "bf16", 768), (64, 1, 40, 96, "e4m3", 1536), (2, 1, 20, 256, "bf16", 512)])
def test_attention_where_sequences_begin_to_be_split(B, heads, group, dim, cache, most):
    """Tables of the most tokens that a block takes whole, and of one page more: ragged, with a sequence that fills its table and an empty one."""
    page = 32
    for room in (most, most + page):
        per = room // page
        cfg = M.KvCfg.make(B * per, page, heads, dim, "bf16", cache)
        attn = M.AttnCfg.make(B, heads * group, per)
        assert (M.moe_attn_workspace_bytes(cfg, attn) == 256) == (room == most)
        table = tables(7, B, per, cfg.pages)
        lens = [room if b == 0 else (room * b * 7) // (B * 7 + 3) % room for b in range(B)]
        if B > 2:
            lens[1] = 0
        arrays = cache_of(34, cfg, table, lens)
        q = normal(36, (B, heads * group, dim), "bf16", 2.0)
        run_and_check(cfg, arrays, q, table.cuda(), lens, only=sorted({0, 1 % B, B - 1}))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("B,room,heads,group,dim,window", [
    (45, 32, 8, 1, 64, 0), (24, 128, 32, 3, 128, 0), (70, 256, 4, 33, 80, 0), (40, 512, 32, 2, 128, 100), (24, 128, 16, 17, 256, 0), (66, 512, 64, 1, 64, 0)])
def test_attention_of_many_short_sequences(B, room, heads, group, dim, window, dtype, cache):
    """A wave for each sequence and group of query heads: lengths of all kinds, a number of items that does not fill the last block."""
    page = 16
    per = room // page
    cfg = M.KvCfg.make(B * per, page, heads, dim, dtype, cache)
    table = tables(8, B, per, cfg.pages)
    lens = [min(room, n) for n in [0, 1, 15, 17, 31, 32, 33, 64, 65, 127, 128, 129, 255, 300, room, room - 1]]
    lens += [(37 * b) % (room + 1) for b in range(B - len(lens))]
    arrays = cache_of(38, cfg, table, lens, window=window)
    q = normal(40, (B, heads * group, dim), dtype, 2.0)
    run_and_check(cfg, arrays, q, table.cuda(), lens, window, only=[*range(16), B - 1])


def test_attention_of_as_many_sequences_as_there_may_be():
    """4096 sequences of 0 to 40 tokens, and 1000 of which one is long: the stretches of a block begin and end anywhere."""
    for B, lens, heads in ((4096, [(b * 29) % 41 for b in range(4096)], 1), (1000, [(b % 3) * 20 if b != 777 else 4000 for b in range(1000)], 2)):
        page = 16
        cfg = M.KvCfg.make(sum(-(-n // page) for n in lens) + 1, page, heads, 64)
        per = -(-max(lens) // page)
        table, at = torch.zeros((B, per), dtype=torch.int32), 0
        for b, n in enumerate(lens):
            used = -(-n // page)
            table[b, :used] = torch.arange(at, at + used)
            at += used
        arrays = cache_of(40, cfg, table, lens)
        q = normal(42, (B, 2 * heads, 64), "bf16", 2.0)
        out, _ = run_and_check(cfg, arrays, q, table.cuda(), lens, only=[0, 1, 2, 100, 776, 777, 778, B - 1])
        assert all((out[b] == 0).all() == (n == 0) for b, n in enumerate(lens[:200]))


def test_attention_of_growing_falling_and_far_logits():
    """The running maximum rises in every run, never rises, and logits lie thousands apart; lengths outside of the table are taken as within it."""
    page, n, dim = 32, 900, 64
    cfg = M.KvCfg.make(29, page, 1, dim, "f32", "f32")
    table = tables(3, 1, 29, 29)
    for slope in (0.05, -0.05, 8.0, -8.0):
        arrays = cache_of(50, cfg, table, [n], 0.1)
        at = torch.arange(n)
        arrays[0][table[0][at // page].long(), 0, at % page, 0] = (slope * at.float()).cuda()
        q = torch.zeros((1, 3, dim), device="cuda")
        q[:, :, 0] = 8.0
        run_and_check(cfg, arrays, q, table.cuda(), [n])
        arrays[0][table[0][28].long(), 0, n % page:] = arrays[1][table[0][28].long(), 0, n % page:] = 0.0
        for odd, as_if in ((10 ** 9, 29 * page), (-5, 0)):
            out, lse = run_attention(cfg, arrays, q, table.cuda(), [odd])
            want, want_lse = run_attention(cfg, arrays, q, table.cuda(), [as_if])
            assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_attention_scale_no_lse_and_not_finite_values_that_count():
    cfg = M.KvCfg.make(8, 16, 2, 64)
    table = tables(4, 2, 4, 8)
    arrays = cache_of(60, cfg, table, [50, 60])
    q = normal(62, (2, 4, 64), "bf16")
    out, _ = run_and_check(cfg, arrays, q, table.cuda(), [50, 60], scale=0.7)
    again, _ = run_attention(cfg, arrays, q, table.cuda(), [50, 60], scale=0.7, want_lse=False)
    assert torch.equal(out, again)
    arrays[0][table[0, 1].long(), 0, 3] = float("nan")                          # token 19 of sequence 0, key head 0
    bad, _ = run_attention(cfg, arrays, q, table.cuda(), [50, 60], scale=0.7)
    assert torch.isnan(bad[0, :2]).all() and torch.equal(bad[0, 2:], out[0, 2:]) and torch.equal(bad[1], out[1])
    shorter, _ = run_attention(cfg, arrays, q, table.cuda(), [19, 60], scale=0.7)
    assert torch.isfinite(shorter).all()


@pytest.mark.parametrize("n", [20, 5000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_to_logits_of_minus_infinity(n, dtype):
    """Tokens whose logit is -infinity weigh nothing; a head with no other tokens is as one without tokens (one launch, and split)."""
    cfg = M.KvCfg.make(-(-n // 16), 16, 2, 64, dtype)
    table = tables(6, 1, cfg.pages, cfg.pages)
    arrays = cache_of(64, cfg, table, [n])
    q = normal(66, (1, 4, 64), dtype).abs()
    at = torch.arange(n)
    place = (table[0][at // 16].long(), at % 16)
    arrays[0][place[0], 0, place[1], 0] = -math.inf                             # key head 0: all tokens
    arrays[0][place[0][7:], 1, place[1][7:], 63] = -math.inf                    # key head 1: all from the eighth on
    out, lse = run_attention(cfg, arrays, q, table.cuda(), [n])
    assert (out[0, :2] == 0).all() and (lse[0, :2] == -math.inf).all()
    want, want_lse = run_attention(cfg, arrays, q, table.cuda(), [7])
    tol = 2 * HALF[dtype] if dtype == "bf16" else 2.0 ** -18                    # the same seven weights in sums of another order
    within(f64(out[0, 2:]), f64(want[0, 2:]), tol * (f64(want[0, 2:]).__abs__() + 4), "seven tokens")
    assert torch.allclose(lse[0, 2:], want_lse[0, 2:], atol=2.0 ** -20)


def test_empty_calls_through_the_binding():
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    M.moe_add_norm(M.NormCfg.make(0, 64), x, x, w, x, x)
    cfg = M.KvCfg.make(2, 16, 1, 64)
    arrays, rows, slots = cfg.empty(), x.view(0, 1, 64), torch.empty(0, dtype=torch.int32, device="cuda")
    M.moe_kv_write(cfg, rows, rows, slots, *arrays)
    M.moe_kv_read(cfg, *arrays, slots, rows, rows)
    attn = M.AttnCfg.make(0, 2, 2)
    ws = torch.empty(M.moe_attn_workspace_bytes(cfg, attn), dtype=torch.uint8, device="cuda")
    M.moe_attn_decode(cfg, attn, rows.expand(0, 2, 64), *arrays, slots.view(0, 2), slots, rows.expand(0, 2, 64), None, ws)


# ------------------------------------------------------------------------------------------- together

def test_calls_on_another_stream_and_in_a_graph():
    """norm -> cache -> attention, recorded into a graph and replayed on new inputs, against the eager calls on another stream."""
    B, heads, group, dim, page = 5, 4, 2, 64, 16
    d = heads * group * dim
    cfg = M.KvCfg.make(B * 20, page, heads, dim, "bf16", "e4m3")
    table = tables(5, B, 20, cfg.pages)
    lens = [0, 17, 130, 299, 40]
    arrays = cache_of(70, cfg, table, lens)
    table, norm = table.cuda(), M.NormCfg.make(B, d, "bf16")
    attn = M.AttnCfg.make(B, heads * group, 20)
    x, r, w = normal(71, (B, d), "bf16"), normal(72, (B, d), "bf16"), normal(73, (d,), "bf16")
    kv = normal(74, (B, 2, heads, dim), "bf16")
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s, y, out = torch.empty_like(x), torch.empty_like(x), torch.empty((B, heads * group, dim), dtype=torch.bfloat16, device="cuda")
    slots = torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(M.moe_attn_workspace_bytes(cfg, attn), dtype=torch.uint8, device="cuda")

    def calls():
        M.moe_add_norm(norm, x, r, w, s, y)
        M.moe_kv_write(cfg, kv[:, 0], kv[:, 1], slots, *arrays)
        M.moe_attn_decode(cfg, attn, y.view(B, heads * group, dim), *arrays, table, lens_d, out, None, ws)

    def place():
        at = lens_d.long()
        slots.copy_(table[torch.arange(B, device="cuda"), at // page] * page + at % page)
        lens_d.add_(1)

    place()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        place()
        x.copy_(normal(80 + step, (B, d), "bf16"))
        kv.copy_(normal(90 + step, (B, 2, heads, dim), "bf16"))
        kept = [t.clone() for t in arrays]
        graph.replay()
        torch.cuda.synchronize()
        got, cache = out.clone(), [t.clone() for t in arrays]
        for t, k in zip(arrays, kept):
            t.copy_(k)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            calls()
        side.synchronize()
        assert torch.equal(got, out) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache, arrays))
        q = y.view(B, heads * group, dim)
        run_and_check(cfg, arrays, q, table, lens_d.tolist())
