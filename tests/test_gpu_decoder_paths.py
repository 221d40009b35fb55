"""Every way that a size can choose: attention whose sequences are split over the device at short lengths, window edges and with as many
sequences as there may be; norm and cache with the accesses that large calls take.  A call that is split needs a workspace of more than the
256 bytes that every call asks for, which says which way it takes.  Tolerances as in test_gpu_decoder.py, with weights of 16 bits."""
import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from test_gpu_decoder import EDGES, HALF, TYPES, cache_of, check_norm, f64, filled, normal, run_and_check, run_attention, tables, take, within

pytestmark = pytest.mark.gpu


def is_split(cfg, B, q_heads, per, window=0):
    return M.moe_attn_workspace_bytes(cfg, M.AttnCfg.make(B, q_heads, per, window=window)) > 256


# ------------------------------------------------------------------------------------------- attention

LENGTHS = EDGES + [513, 600, 1499, 1500, 1501, 1516, 2048, 2049, 2064, 2500, 3000]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,window", [
    (4, 1, 64, 16, 0), (2, 3, 128, 32, 1501), (1, 8, 16, 64, 2064), (3, 5, 80, 16, 1500), (2, 16, 48, 512, 2049), (1, 17, 128, 16, 1100), (1, 33, 64, 32, 2033),
    (2, 4, 256, 16, 515), (1, 20, 144, 128, 513), (12, 1, 48, 64, 2990)])
def test_split_attention_at_the_edges_of_runs_pages_and_windows(heads, group, dim, page, window, dtype, cache):
    """Tables with room for 3000 tokens: short sequences among long ones, windows that begin anywhere in a run of 16, numbers of pages that are
    none beside the attended ones."""
    B, per = len(LENGTHS), -(-3000 // page)
    cfg = M.KvCfg.make(B * per + 3, page, heads, dim, dtype, cache)
    assert is_split(cfg, B, heads * group, per, window)
    table = tables(1, B, per, cfg.pages)
    arrays = cache_of(20, cfg, table, LENGTHS, window=window)
    for b, n in enumerate(LENGTHS):
        first = max(0, n - window) if window else 0
        table[b, -(-n // page):] = 2 ** 31 - 1
        table[b, :first // page] = -7
    wide = normal(22, (B, heads * group * dim + 24), dtype, 2.0)
    q = wide[:, 8:8 + heads * group * dim].view(B, heads * group, dim)
    run_and_check(cfg, arrays, q, table.cuda(), LENGTHS, window)


@pytest.mark.parametrize("heads,cache", [(1, "bf16"), (2, "e4m3")])
def test_as_many_sequences_as_there_may_be_are_split(heads, cache):
    """4096 sequences of 0 to 40 tokens and some of up to 2500, each with a table for 2560: stretches begin and end anywhere in them, and the list
    of lengths is as long as it gets."""
    B, page, per = 4096, 16, 160
    lens = [(b * 29) % 41 for b in range(B)]
    for b, n in ((0, 0), (63, 777), (64, 0), (65, 2500), (1000, 2049), (2047, 1300), (4032, 2500), (4095, 2111)):
        lens[b] = n
    cfg = M.KvCfg.make(sum(-(-n // page) for n in lens) + 1, page, heads, 64, "bf16", cache)
    assert is_split(cfg, B, 2 * heads, per)
    table, at = torch.full((B, per), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        used = -(-n // page)
        table[b, :used] = torch.arange(at, at + used)
        at += used
    arrays = cache_of(40, cfg, table, lens)
    q = normal(42, (B, 2 * heads, 64), "bf16", 2.0)
    only = [0, 1, 2, 62, 63, 64, 65, 66, 100, 999, 1000, 1001, 2047, 2048, 4031, 4032, 4033, 4094, 4095]
    out, lse = run_and_check(cfg, arrays, q, table.cuda(), lens, only=only)
    assert all((out[b] == 0).all() == (n == 0) for b, n in enumerate(lens[:200]))
    # the rest of them against the same sequences with tables that are not split
    short = [b for b in range(B) if lens[b] <= 40]
    narrow = table[short][:, :3].contiguous()
    assert not is_split(cfg, len(short), 2 * heads, 3)
    want, want_lse = run_attention(cfg, arrays, q[short].contiguous(), narrow.cuda(), [lens[b] for b in short])
    assert torch.allclose(out[short].float(), want.float(), rtol=2 ** -7, atol=2 ** -12)
    assert torch.allclose(lse[short], want_lse, rtol=2 ** -20, atol=2 ** -20)


def test_no_sequence_with_tokens_is_split():
    """All of them empty, in tables that are split."""
    cfg = M.KvCfg.make(4, 16, 2, 64)
    arrays, table = filled(cfg, 0xff), torch.full((300, 256), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    assert is_split(cfg, 300, 4, 256)
    out, lse = run_attention(cfg, arrays, normal(1, (300, 4, 64), "bf16"), table, [0] * 300)
    assert (out == 0).all() and (lse == -float("inf")).all()


# ------------------------------------------------------------------------------------------- norm and cache

def sampled(n):
    return sorted({0, 1, n // 3, n // 2, n - 2, n - 1})


@pytest.mark.parametrize("dtype,T,d,group", [
    ("bf16", 4096, 4096, 0), ("bf16", 4001, 4096, 128), ("bf16", 16384, 4096, 0), ("bf16", 50001, 1000, 0), ("bf16", 6000, 12288, 64), ("bf16", 130001, 512, 32),
    ("f32", 2048, 4096, 0), ("f32", 8192, 4096, 128), ("f32", 40001, 1000, 0), ("f32", 1600, 32768, 0), ("f32", 60000, 256, 64)])
def test_norm_of_many_rows(dtype, T, d, group):
    """From 100 MiB on stores, and from 320 MiB on loads, leave the caches to others: the same bits as in pieces that do not, and the oracle's
    values in some rows; in place too."""
    x, r, w = (torch.empty(s, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32) for s in ((T, d), (T, d), (d,)))
    g = torch.Generator(device="cuda").manual_seed(T)
    for t in (x, r, w):
        t.normal_(generator=g)
    groups = d // group if group else 1
    new = lambda dt, *shape: torch.zeros(shape, dtype=dt, device="cuda")
    outs = [dict(sum=new(x.dtype, T, d), y=new(x.dtype, T, d), q=new(torch.float8_e4m3fn, T, d), q_scale=new(torch.float32, T, groups)) for _ in range(2)]
    cfg = M.NormCfg.make(T, d, dtype, q_group=group)
    es, each = x.element_size(), T * d
    assert each * (4 * es + 1) > 100 << 20
    M.moe_add_norm(cfg, x, r, w, *outs[0].values())
    step = (64 << 20) // (d * (4 * es + 1)) & ~3                   # (scales 16-byte aligned)
    for at in range(0, T, step):
        cut = slice(at, min(T, at + step))
        M.moe_add_norm(M.NormCfg.make(cut.stop - at, d, dtype, q_group=group), x[cut], r[cut], w, *(t[cut] for t in outs[1].values()))
    torch.cuda.synchronize()
    for name in outs[0]:
        assert torch.equal(*(o[name].view(torch.uint8) for o in outs)), name
    rows = sampled(T)
    check_norm(M.NormCfg.make(len(rows), d, dtype, q_group=group), dtype, x[rows], r[rows], w, {n: t.view(torch.uint8)[rows].view(t.dtype) for n, t in outs[0].items()})
    M.moe_add_norm(cfg, x, r, w, r, x)
    torch.cuda.synchronize()
    assert torch.equal(r, outs[0]["sum"]) and torch.equal(x, outs[0]["y"])


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("megabytes", [130, 270, 540])
@pytest.mark.parametrize("heads,dim", [(32, 64), (16, 128), (8, 256), (9, 144)])
def test_cache_of_many_tokens(heads, dim, megabytes, dtype, cache):
    """From 80 MiB on stores, from 200 (written) or 320 (read into bf16) on loads, leave the caches to others: the same bits as token by token in
    pieces that do not, with tokens that have no place, and the oracle's values in some rows."""
    page = 64
    width = {"bf16": 2, "f32": 4, "e4m3": 1}
    n = megabytes * 10 ** 6 // (2 * heads * dim * (width[dtype] + width[cache])) | 1
    pages = -(-n // page) + 2
    cfg = M.KvCfg.make(pages, page, heads, dim, dtype, cache)
    g = torch.Generator(device="cuda").manual_seed(n)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n].int()
    slots[5::11] = -1
    slots[6::13] = pages * page
    there = (slots >= 0) & (slots < pages * page)
    kv = torch.empty((n, 2, heads, dim), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda").normal_(generator=g)
    k, v = kv[:, 0], kv[:, 1]
    whole, pieces = filled(cfg, 0x5a), filled(cfg, 0x5a)
    M.moe_kv_write(cfg, k, v, slots, *whole)
    step = n * 48 // megabytes
    for at in range(0, n, step):
        cut = slice(at, min(n, at + step))
        M.moe_kv_write(cfg, k[cut], v[cut], slots[cut], *pieces)
    torch.cuda.synchronize()
    for a, b in zip(whole, pieces):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    rows = torch.tensor([i for i in sampled(n) if there[i]], device="cuda")
    for t, pages_, scale in ((k, whole[0], whole[2]), (v, whole[1], whole[3])):
        got = take(pages_, slots[rows], page)
        if cache != "e4m3":
            assert torch.equal(take(pages_, slots[there], page), t[there].to(pages_.dtype))
            continue
        want = D.e4m3_scale(f64(t[rows]))
        within(f64(scale.transpose(1, 2).flatten(0, 1)[slots[rows].long()]), want, want * 2 ** -23, "scale")
        ratio = f64(t[rows]) / want[..., None]
        within(f64(got), ratio, np.maximum(np.abs(ratio) * 2 ** -4, 2 ** -10) * (1 + 2 ** -10), "e4m3 value")
    back = [torch.full_like(kv, 7) for _ in range(2)]
    M.moe_kv_read(cfg, *whole, slots, back[0][:, 0], back[0][:, 1])
    for at in range(0, n, step):
        cut = slice(at, min(n, at + step))
        M.moe_kv_read(cfg, *whole, slots[cut], back[1][cut, 0], back[1][cut, 1])
    torch.cuda.synchronize()
    assert torch.equal(*back) and (back[0][~there] == 0).all()
    for i, (pages_, scale) in enumerate(((whole[0], whole[2]), (whole[1], whole[3]))):
        want = f64(take(pages_, slots[rows], page))
        if scale is not None:
            want = want * f64(scale.transpose(1, 2).flatten(0, 1)[slots[rows].long()])[..., None]
        within(f64(back[0][rows, i]), want, np.abs(want) * (HALF[dtype] + 2 ** -23), "read")
