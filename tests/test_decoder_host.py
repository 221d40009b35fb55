"""Host-only checks of the operators around the expert layer: the oracle against itself and torch's conversions, workspace sizes, and
every refusal of the library and of the binding, before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D


def test_oracle_e4m3_is_the_nearest_value():
    """Against torch's conversion on every e4m3 value, every midpoint between neighbours and random values."""
    every = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()      # 0 .. 448
    mid = (every[1:] + every[:-1]) / 2
    rng = np.random.default_rng(0)
    r = np.concatenate([every, -every, mid, -mid, rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 0.01])
    want = torch.from_numpy(r).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(D.e4m3(r.astype(np.float32)), want)


def test_oracle_attention_by_sums():
    """The oracle against its definition written out token by token in exact order, and two halves joined by their lse."""
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal(16), rng.standard_normal((23, 16)), rng.standard_normal((23, 16))
    out, lse, p = D.attention(q, k, v, 0.3)
    weights = [np.exp(0.3 * sum(q[i] * k[t, i] for i in range(16))) for t in range(23)]
    total = sum(weights)
    assert abs(lse - np.log(total)) < 1e-12 and abs(p.sum() - 1) < 1e-12
    assert np.allclose(out, sum(w * v[t] for t, w in enumerate(weights)) / total, atol=1e-12)
    (o1, l1, _), (o2, l2, _) = D.attention(q, k[:9], v[:9], 0.3), D.attention(q, k[9:], v[9:], 0.3)
    assert np.allclose(out, o1 * np.exp(l1 - lse) + o2 * np.exp(l2 - lse), atol=1e-12)
    out, lse, _ = D.attention(q, k[:0], v[:0], 0.3)
    assert (out == 0).all() and lse == -np.inf


KV = dict(pages=8, page_size=16, heads=2, head_dim=64)


def test_workspace_grows_with_what_is_split():
    kv = M.KvCfg.make(**KV)
    size = lambda **kw: M.moe_attn_workspace_bytes(kv, M.AttnCfg.make(**{**dict(B=3, q_heads=32, table_pages=1000), **kw}))
    assert all(size(**kw) % 256 == 0 and size(**kw) >= 256 for kw in (dict(), dict(B=0), dict(B=4096, table_pages=1), dict(window=1)))
    assert size(table_pages=1) <= size(table_pages=100) <= size()                 # short sequences are not split
    assert size(q_heads=2) < size() < size(q_heads=1024)
    parts = min(3 * 2 * 125, 256)                                                 # blocks that each may leave two parts of a head's group
    assert size() >= 2 * parts * 16 * (64 + 2) * 4


@pytest.mark.parametrize("kw,frag", [
    (dict(T=-1, d=64), "T must be"), (dict(T=1 << 22, d=64), "T must be"), (dict(T=1, d=0), "d must be"), (dict(T=1, d=12), "d must be"),
    (dict(T=1, d=32776), "d must be"), (dict(T=1, d=64, q_group=16), "q_group must be"), (dict(T=1, d=96, q_group=64), "q_group must divide"),
    (dict(T=1, d=64, eps=0.0), "eps"), (dict(T=1, d=64, eps=float("nan")), "eps"), (dict(T=1, d=64, eps=float("inf")), "eps"),
    (dict(T=1, d=64, dtype=2), "dtype"),
])
def test_norm_refuses_a_bad_description(kw, frag):
    L = M.lib()
    assert L.moe_add_norm(C.addressof(M.NormCfg.make(**kw)), *[None] * 8) == -1
    assert frag.encode() in L.moe_last_error()


@pytest.mark.parametrize("kw,frag", [
    (dict(page_size=8), "page_size"), (dict(page_size=24), "page_size"), (dict(page_size=1 << 17), "page_size"), (dict(pages=0), "pages"),
    (dict(pages=1 << 27), "pages"), (dict(heads=0), "heads"), (dict(heads=1025), "heads"), (dict(head_dim=0), "head_dim"),
    (dict(head_dim=72), "head_dim"), (dict(head_dim=272), "head_dim"), (dict(dtype=2), "dtype"), (dict(cache_dtype=3), "cache_dtype"),
    (dict(cache_dtype="f32"), "fp32 cache"),
])
def test_cache_refuses_a_bad_description(kw, frag):
    L = M.lib()
    kv = M.KvCfg.make(**{**KV, **kw})
    attn = M.AttnCfg.make(1, max(1, kv.heads), 1)
    n = C.c_size_t(0)
    for rc in (L.moe_kv_write(C.addressof(kv), 1, None, 0, None, 0, *[None] * 6),
               L.moe_kv_read(C.addressof(kv), 1, *[None] * 6, 0, None, 0, None),
               L.moe_attn_workspace_bytes(C.addressof(kv), C.addressof(attn), C.byref(n)),
               L.moe_attn_decode(C.addressof(kv), C.addressof(attn), None, 0, *[None] * 10)):
        assert rc in (-1, -2)
        assert frag.encode() in L.moe_last_error()


@pytest.mark.parametrize("kw,frag", [
    (dict(B=-1), "B must"), (dict(B=4097), "B must"), (dict(q_heads=3), "q_heads"), (dict(q_heads=0), "q_heads"),
    (dict(q_heads=1026), "q_heads"), (dict(table_pages=0), "table_pages"), (dict(table_pages=(1 << 20) + 1), "table_pages"),
    (dict(window=-1), "window"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
])
def test_attention_refuses_a_bad_description(kw, frag):
    L = M.lib()
    kv, attn = M.KvCfg.make(**KV), M.AttnCfg.make(**{**dict(B=1, q_heads=4, table_pages=4), **kw})
    n = C.c_size_t(0)
    assert L.moe_attn_workspace_bytes(C.addressof(kv), C.addressof(attn), C.byref(n)) == -1
    assert frag.encode() in L.moe_last_error()


def test_null_misaligned_and_contradicting_arguments_are_refused():
    L = M.lib()
    buf = C.create_string_buffer(4096)
    al = (C.addressof(buf) + 255) & ~255
    norm, kv, e4 = M.NormCfg.make(2, 64), M.KvCfg.make(**KV), M.KvCfg.make(**KV, cache_dtype="e4m3")
    attn = M.AttnCfg.make(2, 4, 4)
    N, K, E, A = (C.addressof(c) for c in (norm, kv, e4, attn))

    def refused(rc, frag, code=-1):
        assert rc == code, L.moe_last_error()
        assert frag.encode() in L.moe_last_error()

    refused(L.moe_add_norm(None, *[al] * 8), "cfg is NULL")
    refused(L.moe_add_norm(N, al, al, None, al, al, None, None, None), "weight is NULL")
    refused(L.moe_add_norm(N, None, al, al, al, al, None, None, None), "x is NULL")
    refused(L.moe_add_norm(N, al, al, al, al, None, None, None, None), "both NULL")
    refused(L.moe_add_norm(N, al, al, al, al, al, al, None, None), "go together")
    refused(L.moe_add_norm(N, al, al, al, al, al, None, al, None), "go together")
    for at in range(6):
        args = [al, al, al, al, al, al, al]
        args[at] = al + 4
        refused(L.moe_add_norm(N, *args, None), "aligned")

    refused(L.moe_kv_write(None, 1, al, 128, al, 128, al, al, al, None, None, None), "cfg is NULL")
    refused(L.moe_kv_write(K, -1, al, 128, al, 128, al, al, al, None, None, None), "n must be")
    refused(L.moe_kv_write(K, 1, None, 128, al, 128, al, al, al, None, None, None), "k is NULL")
    refused(L.moe_kv_write(K, 1, al, 128, None, 128, al, al, al, None, None, None), "v is NULL")
    refused(L.moe_kv_write(K, 1, al, 127, al, 128, al, al, al, None, None, None), "stride of k")
    refused(L.moe_kv_write(K, 1, al, 128, al, 132, al, al, al, None, None, None), "stride of v")
    refused(L.moe_kv_write(K, 1, al, 128, al, 1 << 31, al, al, al, None, None, None), "stride of v")
    refused(L.moe_kv_write(K, 1, al, 128, al, 128, None, al, al, None, None, None), "slots is NULL")
    refused(L.moe_kv_write(K, 1, al, 128, al, 128, al, None, al, None, None, None), "k_pages is NULL")
    refused(L.moe_kv_write(K, 1, al, 128, al, 128, al, al, al + 2, None, None, None), "v_pages must be")
    refused(L.moe_kv_write(K, 1, al, 128, al, 128, al, al, al, al, None, None), "scales are for")
    refused(L.moe_kv_write(E, 1, al, 128, al, 128, al, al, al, al, None, None), "v_scales is NULL")
    refused(L.moe_kv_read(E, 1, al, al, None, al, al, al, 128, al, 128, None), "k_scales is NULL")
    refused(L.moe_kv_read(K, 1, al, al, None, None, al, al, 120, al, 128, None), "stride of k")
    refused(L.moe_kv_read(K, 1, al, al, None, None, None, al, 128, al, 128, None), "slots is NULL")
    assert L.moe_kv_write(K, 0, None, 0, None, 0, None, al, al, None, None, None) == 0
    assert L.moe_kv_read(K, 0, al, al, None, None, None, None, 0, None, 0, None) == 0
    assert L.moe_add_norm(C.addressof(M.NormCfg.make(0, 64)), None, None, al, None, al, None, None, None) == 0

    good = [al, 256, al, al, None, None, al, al, al, al, al]                     # q, stride, pages, scales, table, lens, out, lse, ws
    for at, frag in ((0, "q is NULL"), (2, "k_pages is NULL"), (3, "v_pages is NULL"), (6, "table is NULL"), (7, "lens is NULL"),
                     (8, "out is NULL"), (10, "ws is NULL")):
        args = list(good)
        args[at] = None
        refused(L.moe_attn_decode(K, A, *args, None), frag)
    refused(L.moe_attn_decode(K, None, *good, None), "attn is NULL")
    refused(L.moe_attn_decode(K, A, al, 248, *good[2:], None), "stride of q")
    refused(L.moe_attn_decode(E, A, *good, None), "k_scales is NULL")
    refused(L.moe_attn_decode(K, A, *good[:10], al + 16, None), "256-byte", code=-3)
    refused(L.moe_attn_decode(K, A, *good[:8], al + 8, *good[9:], None), "out must be")
    assert L.moe_attn_decode(K, C.addressof(M.AttnCfg.make(0, 4, 4)), None, 0, al, al, *[None] * 8) == 0
    assert L.moe_attn_workspace_bytes(K, A, None) == -1


def test_binding_refuses_tensors_of_another_size_type_or_layout():
    kv, norm = M.KvCfg.make(**KV), M.NormCfg.make(2, 64)
    b = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt)
    k, v, _, _ = kv.empty("cpu")
    slots = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(M.MoeError, match="x must be a contiguous"):
        M.moe_add_norm(norm, b(2, 32), None, b(64), None, b(2, 64))
    with pytest.raises(M.MoeError, match="weight must be a contiguous"):
        M.moe_add_norm(norm, None, None, b(64, dt=torch.float32), None, b(2, 64))
    with pytest.raises(M.MoeError, match="x must be in device memory"):
        M.moe_add_norm(norm, b(2, 64), None, b(64), None, b(2, 64))
    with pytest.raises(M.MoeError, match="k must be"):
        M.moe_kv_write(kv, b(3, 2, 32), b(3, 2, 64), slots, k, v)
    with pytest.raises(M.MoeError, match="contiguous rows"):
        M.moe_kv_write(kv, b(3, 64, 2).transpose(1, 2), b(3, 2, 64), slots, k, v)
    with pytest.raises(M.MoeError, match="k must be"):
        M.moe_kv_write(kv, b(2, 2, 64), b(3, 2, 64), slots, k, v)
    attn = M.AttnCfg.make(2, 4, 4)
    with pytest.raises(M.MoeError, match="q must be"):
        M.moe_attn_decode(kv, attn, b(2, 4, 32), k, v, None, None, slots, slots, None, None, None)
    with pytest.raises(M.MoeError, match="ws is smaller"):
        M.moe_attn_decode(kv, attn, None, k, v, None, None, slots, slots, None, None, b(16))


def test_no_rows_no_tokens_no_sequences_is_no_error():
    """Tensors without elements have no address: that is no missing argument."""
    L = M.lib()
    buf = C.create_string_buffer(64 * 2 + 16)
    weight = (C.addressof(buf) + 15) & ~15
    none = torch.empty((0, 64), dtype=torch.bfloat16).data_ptr()
    assert L.moe_add_norm(C.addressof(M.NormCfg.make(0, 64)), none, none, weight, none, none, None, None, None) == 0
    assert L.moe_add_norm(C.addressof(M.NormCfg.make(0, 64)), none, none, weight, none, None, none, none, None) == 0
