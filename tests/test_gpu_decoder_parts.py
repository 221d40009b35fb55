"""The bits that attention's products keep: weights exp(l - m) of 16 bits for bf16 outputs, fp32 queries and weights with all of theirs.

Two tokens per sequence and one column of the queries that is not zero, so that a logit is one product and errors stay small enough to tell:
  fp32  out of values 0 and 1 is w / (1 + w): a logit of at most 2 is off by 8 roundings, 2^-20, the exponential, its argument, sum,
        quotient and products by some 8 of 2^-24 more: 2^-19 in all.  The log-sum of one token is its logit: 2^-20 of it.  A part of 8 bits
        fewer of the weight is off by up to 2^-18, of the query by up to 2^-17 of the logit.
  bf16  values 1 and minus the weight as it would be with 8 bits cancel all but what those leave out: off by 2^-16 of the sum of
        magnitudes and half a step of what is left, 2^-8 of that; with 8 bits nothing would be left, or all of it would be wrong.
The same check is made of results computed here with a part fewer, which it has to refuse."""
import math

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from test_gpu_decoder import TORCH, TYPES, f64, filled, tables

B, H, DIM, COLUMN = 32, 16, 64, 37
SCALE = 1 / math.sqrt(DIM)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def held(x, parts):
    """x as the sum of this many bf16 values."""
    left, out = x.copy(), np.zeros_like(x)
    for _ in range(parts):
        p = bf16(left)
        out, left = out + p, left - p
    return out


def inputs(dtype):
    """q [B, H, DIM] and the second tokens' keys [B, H, DIM] of the activations' type: logits between -2 and 2, the first tokens' are 0."""
    g = torch.Generator().manual_seed(9)
    q, k = torch.zeros((B, H, DIM)), torch.zeros((B, H, DIM))
    q[..., COLUMN] = (torch.rand((B, H), generator=g) + 0.5) * 4.0 * torch.randint(0, 2, (B, H), generator=g).mul(2).sub(1)
    k[..., COLUMN] = torch.rand((B, H), generator=g) * 2.0 + 0.5
    return q.to(TORCH[dtype]), k.to(TORCH[dtype])


def weights(q, k):
    """exp of the second tokens' logits in 64 bits."""
    return np.exp(SCALE * (q[..., COLUMN] * k[..., COLUMN]))


def check(dtype, q, k, v, out, lse, lse_of_one):
    """q, k [B, H, DIM], v [2, B, H, DIM]: as stored.  lse_of_one: where the second token is the only one."""
    logit, w = SCALE * (q[..., COLUMN] * k[..., COLUMN]), weights(q, k)
    ref = (v[0] + w[..., None] * v[1]) / (1 + w)[..., None]
    size = (np.abs(v[0]) + w[..., None] * np.abs(v[1])) / (1 + w)[..., None]
    if dtype == "f32":
        assert (np.abs(out - ref) <= 2 ** -19 * size).all(), "out"
        assert (np.abs(lse_of_one - logit) <= 2 ** -20 * np.abs(logit)).all(), "log-sum of one token"
    else:
        assert (np.abs(out - ref) <= 2 ** -16 * size + 2 ** -8 * np.abs(ref)).all(), "out"
    assert (np.abs(lse - np.log1p(w)) <= 2 ** -19).all(), "log-sum of two"


def values(dtype, q, k):
    """The two tokens' values [2, B, H, DIM]."""
    if dtype == "f32":
        return torch.stack([torch.zeros(q.shape), torch.ones(q.shape)]).to(TORCH[dtype])
    w = weights(q.double().numpy(), k.double().numpy())
    low = np.where(w <= 1, bf16(w), 1.0)                           # the larger of the two weights is 1, the other as with 8 bits
    one = np.where(w <= 1, 1.0, bf16(1 / w))
    both = np.stack([-low, one])[..., None] * np.ones(DIM)
    return torch.from_numpy(both).to(TORCH[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("room", [32, 8192])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_all_promised_bits_enter(dtype, cache, room):
    """In one launch, and in tables that are split."""
    page, per = 16, room // 16
    cfg, attn = M.KvCfg.make(B, page, H, DIM, dtype, cache), M.AttnCfg.make(B, H, per)
    assert (M.moe_attn_workspace_bytes(cfg, attn) > 256) == (room > 32)
    q, k2 = inputs(dtype)
    arrays = filled(cfg, 0)
    table = torch.zeros((B, per), dtype=torch.int32)
    table[:, :1] = tables(3, B, 1, B)
    slots = (table[:, 0] * page)[:, None] + torch.arange(2)
    k = torch.stack([torch.zeros_like(k2), k2], 1)                 # [B, 2, H, DIM]
    put = lambda v: M.moe_kv_write(cfg, k.reshape(2 * B, H, DIM).cuda(), v.transpose(0, 1).reshape(2 * B, H, DIM).contiguous().cuda(),
                                   slots.reshape(-1).int().cuda(), *arrays)
    put(torch.zeros((2, B, H, DIM), dtype=TORCH[dtype]))
    stored = lambda t, s: f64(t)[table[:, 0].numpy()].transpose(0, 2, 1, 3)[:, :2] * (1 if s is None else f64(s)[table[:, 0].numpy()].transpose(0, 2, 1)[:, :2, :, None])
    k_stored = stored(arrays[0], arrays[2])[:, 1]                  # (in e4m3 a row of one value is its scale: not quite k2)
    put(values(dtype, q, torch.from_numpy(k_stored)))
    v_stored = stored(arrays[1], arrays[3]).swapaxes(0, 1)
    out, lse = torch.empty((B, H, DIM), dtype=TORCH[dtype], device="cuda"), torch.empty((B, H), device="cuda")
    ws = torch.empty(M.moe_attn_workspace_bytes(cfg, attn), dtype=torch.uint8, device="cuda")

    def run(n):
        M.moe_attn_decode(cfg, attn, q.cuda(), *arrays, table.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"), out, lse, ws)
        torch.cuda.synchronize()
        return f64(out), f64(lse)

    got, got_lse = run(2)
    M.moe_kv_write(cfg, k2.cuda(), k2.cuda(), slots[:, 0].int().contiguous().cuda(), *arrays)       # the second token alone, where the first was
    check(dtype, f64(q), k_stored, v_stored, got, got_lse, run(1)[1])


@pytest.mark.parametrize("dtype,parts_q,parts_w", [("f32", 3, 3), ("f32", 2, 3), ("f32", 3, 2), ("bf16", 1, 2), ("bf16", 1, 1)])
def test_a_part_fewer_would_be_seen(dtype, parts_q, parts_w):
    """What the kernel does, in numpy: as it is the check passes, with a part fewer it does not."""
    q, k = (t.double().numpy() for t in inputs(dtype))
    k = bf16(k)
    v = values(dtype, torch.from_numpy(q), torch.from_numpy(k)).double().numpy()
    logit = SCALE * (held(q, parts_q)[..., COLUMN] * k[..., COLUMN])
    top = np.maximum(logit, 0.0)
    w = np.stack([np.exp(-top), np.exp(logit - top)])
    out = (held(w, parts_w)[..., None] * v).sum(0) / w.sum(0)[..., None]
    if dtype == "bf16":
        out = bf16(out)
    made = lambda: check(dtype, q, k, v, out, top + np.log(w.sum(0)), logit)
    if (parts_q, parts_w) in ((3, 3), (1, 2)):
        made()
    else:
        with pytest.raises(AssertionError, match="out|one token"):
            made()
