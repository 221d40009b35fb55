"""moe_rope on calls that move more than the caches hold, which leave these to others by their stores (from 100 MB on) and by their loads too (from 300 MB on):
against the same formula in fp64 on the same device.  Tolerance as in test_gpu_rope.py."""
import pytest
import torch

import paper_2106_10715_amd as M
from test_gpu_decoder import HALF

pytestmark = pytest.mark.gpu


def turned(x, angle, rot, neighbours):
    """In fp64: rows x turned by angle [n, 1, pairs], and |a| + |b| of each element's pair (|a| of its own past the turned columns)."""
    x = x.double()
    at = torch.arange(rot, device="cuda")
    at = at.view(-1, 2).t() if neighbours else at.view(2, -1)
    a, b = x[..., at[0]], x[..., at[1]]
    ref, size = x.clone(), x.abs()
    ref[..., at[0]], ref[..., at[1]] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
    size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
    return ref, size


@pytest.mark.parametrize("place", ["apart", "in place"])
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("dtype,n,q_heads,k_heads,dim,rot", [
    ("bf16", 6001, 32, 8, 128, 128), ("bf16", 16001, 32, 8, 128, 128), ("bf16", 30001, 12, 4, 80, 32), ("bf16", 70001, 12, 4, 80, 32), ("bf16", 40001, 7, 2, 96, 6),
    ("bf16", 100001, 7, 2, 96, 6), ("f32", 3001, 32, 8, 128, 128), ("f32", 8001, 32, 8, 128, 128), ("f32", 9001, 16, 1, 112, 28), ("f32", 25001, 16, 1, 112, 28)])
def test_calls_past_the_caches(dtype, n, q_heads, k_heads, dim, rot, pairs, place):
    heads, dt = q_heads + k_heads, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    moved = 2 * n * heads * dim * dt.itemsize
    assert 100 << 20 < moved < 280 << 20 or moved > 310 << 20                  # between the two sizes, or past both
    cfg = M.RopeCfg.make(q_heads, k_heads, dim, rot, dtype, pairs=pairs)
    freqs = M.moe_rope_frequencies(cfg).cuda()
    g = torch.Generator(device="cuda").manual_seed(81)
    x = torch.empty((n, heads * dim + 16), dtype=dt, device="cuda").normal_(generator=g)
    positions = torch.randint(0, 200000, (n,), generator=g, device="cuda").int()
    q, k = x[:, :q_heads * dim].view(n, q_heads, dim), x[:, q_heads * dim + 8:-8].view(n, k_heads, dim)
    y = x if place == "in place" else torch.full_like(x, 7)
    q_out, k_out = y[:, :q_heads * dim].view(n, q_heads, dim), y[:, q_heads * dim + 8:-8].view(n, k_heads, dim)
    before = x.clone()
    M.moe_rope(cfg, positions, freqs, q, q_out, k, k_out)
    torch.cuda.synchronize()
    for gap in (slice(q_heads * dim, q_heads * dim + 8), slice(heads * dim + 8, None)):
        assert torch.equal(y[:, gap], before[:, gap]) if place == "in place" else (y[:, gap] == 7).all()
    q, k = before[:, :q_heads * dim].view(n, q_heads, dim), before[:, q_heads * dim + 8:-8].view(n, k_heads, dim)
    for name, rows, got in (("q", q, q_out), ("k", k, k_out)):
        for i in range(0, n, 8192):
            part = slice(i, min(i + 8192, n))
            ref, size = turned(rows[part], positions[part].double()[:, None, None] * freqs, rot, pairs == "neighbours")
            tol = ref.abs() * HALF[dtype] + size * (32 * 2.0 ** -24 + 200000 * 2.0 ** -49)
            tol[..., rot:] = 0.0
            over = ((got[part].double() - ref).abs() - tol).max()
            assert over <= 0, f"{name}, rows from {i}: off by {float(over):.3e} more than they may be"
