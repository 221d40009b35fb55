"""e4m3 outputs are quotients: with the scale that is stored, every value is the e4m3 value nearest to row / scale, both steps rounded to the
nearest.  A product with a rounded 1 / scale is off by a bit of fp32 now and then, which at a border between two e4m3 values is a whole step of
2^-3.  So the values are compared bit by bit, with quotients that numpy forms (IEEE, fp32)."""
import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D

pytestmark = pytest.mark.gpu


def f32(t):
    return t.float().cpu().numpy()


def quotients(rows, scale):
    return D.e4m3((rows.astype(np.float32) / scale[..., None].astype(np.float32)))


def scales(rows):
    return np.maximum(np.abs(rows).max(-1) / np.float32(448), np.float32(2.0 ** -126))


def rows_with_borders(seed, shape):
    """Normal values rounded to bf16, whose quotients often lie at a border or within a bit of fp32 from it."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * 4.0).to(torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,dim", [(8, 128), (3, 80), (2, 256), (4, 16)])
def test_cache_values_are_the_quotients(heads, dim, dtype):
    n, page = 2000, 64
    cfg = M.KvCfg.make(-(-n // page), page, heads, dim, "bf16" if dtype is torch.bfloat16 else "f32", "e4m3")
    k, v = (rows_with_borders(s, (n, heads, dim)).to(dtype).cuda() for s in (1, 2))
    arrays = cfg.empty()
    M.moe_kv_write(cfg, k, v, torch.arange(n, dtype=torch.int32, device="cuda"), *arrays)
    torch.cuda.synchronize()
    for rows, pages, scale in ((k, arrays[0], arrays[2]), (v, arrays[1], arrays[3])):
        got = f32(pages).transpose(0, 2, 1, 3).reshape(-1, heads, dim)[:n]
        sc = f32(scale).transpose(0, 2, 1).reshape(-1, heads)[:n]
        assert np.array_equal(sc, scales(f32(rows)))
        assert np.array_equal(got, quotients(f32(rows), sc))


@pytest.mark.parametrize("T,d,group", [(600, 4096, 0), (600, 4096, 128), (2000, 512, 32), (64, 12288, 64), (1000, 1000, 0)])
def test_norm_values_are_the_quotients(T, d, group):
    """fp32 activations, so that what is divided is an output too."""
    cfg = M.NormCfg.make(T, d, "f32", q_group=group)
    x, w = rows_with_borders(3, (T, d)).float().cuda(), rows_with_borders(4, (d,)).float().cuda()
    y, q = torch.empty_like(x), torch.empty((T, d), dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.empty((T, d // group if group else 1), dtype=torch.float32, device="cuda")
    M.moe_add_norm(cfg, x, None, w, None, y, q, sc)
    torch.cuda.synchronize()
    rows = f32(y).reshape(T, -1, group or d)
    assert np.array_equal(f32(sc), scales(rows))
    assert np.array_equal(f32(q).reshape(rows.shape), quotients(rows, f32(sc)))


def test_rows_of_every_size():
    """Rows from the smallest that have a scale of their own to the largest: the scales' whole range."""
    n, dim = 240, 64
    cfg = M.KvCfg.make(n // 16, 16, 1, dim, "f32", "e4m3")
    g = torch.Generator().manual_seed(5)
    rows = torch.rand((n, 1, dim), generator=g) + 0.5
    rows = torch.ldexp(rows * torch.randint(0, 2, rows.shape, generator=g).mul(2).sub(1), torch.arange(n)[:, None, None] - 120)
    rows = torch.ldexp(rows, torch.randint(-14, 1, rows.shape, generator=g))
    arrays = cfg.empty()
    M.moe_kv_write(cfg, rows.cuda(), rows.cuda(), torch.arange(n, dtype=torch.int32, device="cuda"), *arrays)
    torch.cuda.synchronize()
    sc = f32(arrays[2]).transpose(0, 2, 1).reshape(n, 1)
    assert np.array_equal(sc, scales(rows.numpy()))
    assert np.array_equal(f32(arrays[0]).transpose(0, 2, 1, 3).reshape(n, 1, dim), quotients(rows.numpy(), sc))


def test_a_row_with_an_infinity_stores_zeros_and_nan():
    """Over a scale of infinity finite values are 0 and the infinity is NaN: read back, all of the row is NaN, and no other row."""
    cfg = M.KvCfg.make(1, 16, 2, 32, "f32", "e4m3")
    rows = torch.ones((3, 2, 32))
    rows[1, 0, 5] = -float("inf")
    arrays = cfg.empty()
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    M.moe_kv_write(cfg, rows.cuda(), rows.cuda(), slots, *arrays)
    k, v = torch.empty((3, 2, 32), device="cuda"), torch.empty((3, 2, 32), device="cuda")
    M.moe_kv_read(cfg, *arrays, slots, k, v)
    torch.cuda.synchronize()
    raw = f32(arrays[0])[0, 0, 1]
    assert np.isnan(raw[5]) and (np.delete(raw, 5) == 0).all()
    for got in (k, v):
        assert torch.isnan(got[1, 0]).all()
        got[1, 0] = 1.0
        assert torch.allclose(got, torch.ones_like(got))
