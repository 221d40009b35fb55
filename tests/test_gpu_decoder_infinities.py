"""Infinite keys and queries: a token whose logit is -infinity weighs nothing, and a head with no other tokens is as one without tokens.

The logits are -infinity by their formula: in the infinite column keys and queries are not zero and of the signs that give it.  What is
left of a head's tokens is compared with the oracle on those tokens alone, with the tolerances of test_gpu_decoder.py (the fewer tokens, the
narrower)."""
import math

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from test_gpu_decoder import HALF, cache_of, f64, normal, run_attention, tables, within

pytestmark = pytest.mark.gpu


def check_head(out, lse, q, k, v, scale, dtype, what):
    if len(k) == 0:
        assert (f64(out) == 0).all() and float(lse) == -math.inf, what
        return
    ref, ref_lse, p = D.attention(q, k, v, scale)
    logits = scale * (k @ q)
    off = (len(q) + 8) * 2 ** -24 * scale * (np.abs(k) @ np.abs(q)).max() + 4 * 2 ** -24 * np.abs(logits).max()
    sums = (len(p) / 16 + 64) * 2 ** -24
    weights = 2 ** -16 if dtype == "bf16" else 0.0
    within(f64(out), ref, HALF[dtype] * np.abs(ref) + (weights + 2 * off + 2 * sums) * (p @ np.abs(v)) * (1 + HALF[dtype]), what)
    assert abs(float(lse) - ref_lse) <= off + sums + 2 ** -22 * abs(ref_lse) + 2 ** -22, what


def place(table, n, page):
    at = torch.arange(n)
    return table[0][at // page].long().cuda(), (at % page).cuda()


def infinite_keys(dtype, cache, dim, n, column):
    """Key head 0: every token has -infinity in `column`.  Key head 1: all but seven.  Key head 2: none."""
    page = 16
    cfg = M.KvCfg.make(-(-n // page), page, 3, dim, dtype, cache)
    table = tables(6, 1, cfg.pages, cfg.pages)
    arrays = cache_of(64, cfg, table, [n])
    q = normal(66, (1, 6, dim), dtype).abs() + 2 ** -10
    q[0, :, column] = torch.tensor([0.3, 1.0, 0.7, 5.0, 0.7, 1.0], device="cuda").to(q.dtype)
    index, at = place(table, n, page)
    arrays[0][index, 0, at, column] = -math.inf
    left = torch.zeros(n, dtype=torch.bool)
    left[torch.linspace(0, n - 1, 7).long()] = True
    gone = ~left.cuda()
    arrays[0][index[gone], 1, at[gone], column] = -math.inf
    out, lse = run_attention(cfg, arrays, q, table.cuda(), [n])
    k, v = (t[index, :, at].float().cpu().numpy().astype(np.float64) for t in arrays[:2])
    for head in range(6):
        keep = (np.zeros(n, bool), left.numpy(), np.ones(n, bool))[head // 2]
        check_head(out[0, head], lse[0, head], f64(q[0, head]), k[keep, head // 2], v[keep, head // 2], 1 / math.sqrt(dim), dtype, f"head {head}")


@pytest.mark.parametrize("n", [20, 5000])
@pytest.mark.parametrize("dim", [16, 48, 80, 112, 144, 208, 240])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32")])
def test_infinite_keys_in_the_last_column_of_odd_widths(dtype, cache, dim, n):
    infinite_keys(dtype, cache, dim, n, dim - 1)


@pytest.mark.parametrize("n", [20, 5000])
@pytest.mark.parametrize("dim,column", [(16, 0), (48, 47), (64, 33), (80, 79), (128, 5), (144, 143), (256, 200)])
def test_infinite_keys_under_fp32_queries_in_parts(dim, column, n):
    """The parts of 0.3 have two signs, those of 1.0 are zeros but for the first."""
    infinite_keys("f32", "bf16", dim, n, column)


@pytest.mark.parametrize("n", [20, 5000])
@pytest.mark.parametrize("dim", [48, 64, 128, 144, 256])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "bf16"), ("f32", "e4m3")])
def test_infinite_queries(dtype, cache, dim, n):
    """-infinity against keys above zero: logits of -infinity alone; +infinity: no number; the other heads of the same keys as they were."""
    page = 16
    cfg = M.KvCfg.make(-(-n // page), page, 1, dim, dtype, cache)
    table = tables(6, 1, cfg.pages, cfg.pages)
    k, v = normal(70, (n, 1, dim), dtype), normal(71, (n, 1, dim), dtype)
    k[:, :, dim - 1] = k[:, :, dim - 1].abs() + 0.5
    arrays = cfg.empty()
    index, at = place(table, n, page)
    M.moe_kv_write(cfg, k, v, (index * page + at).int(), *arrays)
    q = normal(72, (1, 4, dim), dtype)
    want, want_lse = run_attention(cfg, arrays, q, table.cuda(), [n])
    q[0, 1, dim - 1], q[0, 2, dim - 1] = -math.inf, math.inf
    out, lse = run_attention(cfg, arrays, q, table.cuda(), [n])
    assert (out[0, 1] == 0).all() and lse[0, 1] == -math.inf
    assert torch.isnan(out[0, 2]).all()
    assert torch.equal(out[0, ::3], want[0, ::3]) and torch.equal(lse[0, ::3], want_lse[0, ::3])


@pytest.mark.parametrize("n", [20, 5000])
@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_the_largest_finite_query(cache, n):
    """3.4e38 is past the largest value of 16 bits that is not infinite."""
    page, dim = 16, 64
    cfg = M.KvCfg.make(-(-n // page), page, 1, dim, "f32", cache)
    table = tables(6, 1, cfg.pages, cfg.pages)
    k, v = normal(73, (n, 1, dim), "f32"), normal(74, (n, 1, dim), "f32")
    k[:, :, 3] *= 2.0 ** -124
    arrays = cfg.empty()
    index, at = place(table, n, page)
    M.moe_kv_write(cfg, k, v, (index * page + at).int(), *arrays)
    q = normal(75, (1, 2, dim), "f32")
    q[0, 0, 3], q[0, 1, 3] = torch.finfo(torch.float32).max, -3.3962e38
    out, lse = run_attention(cfg, arrays, q, table.cuda(), [n])
    k, v = (t[index, 0, at].float().cpu().numpy().astype(np.float64) for t in arrays[:2])
    for head in range(2):
        check_head(out[0, head], lse[0, head], f64(q[0, head]), k, v, 1 / math.sqrt(dim), "f32", f"head {head}")
