"""The bits that moe_attn_decode_scored's products keep: the check of test_gpu_decoder_parts.py, which results with a part fewer do not pass, of scores that change
no logit (slopes of zero, a table of zeros)."""
import pytest
import torch

import paper_2106_10715_amd as M
from test_gpu_decoder import TORCH, TYPES, f64, filled, tables
from test_gpu_decoder_parts import B, DIM, H, check, inputs, values


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["slopes", "table"])
@pytest.mark.parametrize("room", [32, 8192])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_all_promised_bits_enter(dtype, cache, room, score):
    """In one launch, and in tables that are split."""
    page, per = 16, room // 16
    cfg, attn = M.KvCfg.make(B, page, H, DIM, dtype, cache), M.AttnCfg.make(B, H, per)
    assert (M.moe_attn_workspace_bytes(cfg, attn) > 256) == (room > 32)
    scores, slopes, bias = (None, torch.zeros(H, device="cuda"), None) if score == "slopes" else (M.ScoresCfg.make(0.0, 4, 2), None, torch.zeros((H, 7), device="cuda"))
    q, k2 = inputs(dtype)
    arrays = filled(cfg, 0)
    table = torch.zeros((B, per), dtype=torch.int32)
    table[:, :1] = tables(3, B, 1, B)
    pages, slots = table[:, 0].numpy(), ((table[:, 0] * page)[:, None] + torch.arange(2)).int()
    ws = torch.empty(M.moe_attn_workspace_bytes(cfg, attn), dtype=torch.uint8, device="cuda")

    def put(k, v, slots):
        """k, v [B, tokens, H, DIM] into the cache."""
        M.moe_kv_write(cfg, k.reshape(-1, H, DIM).to(TORCH[dtype]).cuda(), v.reshape(-1, H, DIM).to(TORCH[dtype]).cuda(), slots.reshape(-1).cuda(), *arrays)

    def stored(pages_of, scales):
        """[B, 2, H, DIM]: the first two tokens' rows as the cache has them."""
        rows = f64(pages_of)[pages].transpose(0, 2, 1, 3)[:, :2]
        return rows if scales is None else rows * f64(scales)[pages].transpose(0, 2, 1)[:, :2, :, None]

    def run(n):
        out, lse = torch.empty((B, H, DIM), dtype=TORCH[dtype], device="cuda"), torch.empty((B, H), device="cuda")
        M.moe_attn_decode_scored(cfg, attn, scores, q.cuda(), *arrays, table.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"), slopes, bias, out, lse, ws)
        torch.cuda.synchronize()
        return f64(out), f64(lse)

    k = torch.stack([torch.zeros_like(k2), k2], 1)
    put(k, torch.zeros_like(k), slots)
    k_stored = stored(arrays[0], arrays[2])[:, 1]
    put(k, values(dtype, q, torch.from_numpy(k_stored)).transpose(0, 1), slots)
    v_stored = stored(arrays[1], arrays[3]).swapaxes(0, 1)
    got, got_lse = run(2)
    put(k2[:, None], k2[:, None], slots[:, :1])                                # the second token alone, where the first was
    check(dtype, f64(q), k_stored, v_stored, got, got_lse, run(1)[1])
