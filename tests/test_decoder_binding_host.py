"""What the binding does with arguments that its marshalling refuses: it says which one and why, and never calls the library.  On the CPU,
where no tensor is in device memory."""
import pytest
import torch

import paper_2106_10715_amd as M
from paper_2106_10715_amd import binding

KV = dict(pages=8, page_size=16, heads=2, head_dim=64)


def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_a_workspace_in_host_memory_is_refused():
    """Of any size, whatever else is given."""
    kv, attn = M.KvCfg.make(**KV), M.AttnCfg.make(2, 4, 4)
    n = M.moe_attn_workspace_bytes(kv, attn)
    for ws in (tensor(n, dtype=torch.uint8), tensor(n + 512, dtype=torch.uint8), tensor(n, dtype=torch.float32)):
        with pytest.raises(M.MoeError, match="ws must be in device memory"):
            M.moe_attn_decode(kv, attn, None, None, None, None, None, None, None, None, None, ws)
    with pytest.raises(M.MoeError, match="ws must be contiguous"):
        M.moe_attn_decode(kv, attn, None, None, None, None, None, None, None, None, None, tensor(n, 2, dtype=torch.uint8)[:, 0])
    with pytest.raises(M.MoeError, match="ws must be a tensor"):
        M.moe_attn_decode(kv, attn, None, None, None, None, None, None, None, None, None, n)


def test_no_slots_are_named():
    kv = M.KvCfg.make(**KV)
    k, v, _, _ = kv.empty("cpu")
    rows = tensor(3, 2, 64)
    with pytest.raises(M.MoeError, match="slots is NULL"):
        M.moe_kv_write(kv, rows, rows, None, k, v)
    with pytest.raises(M.MoeError, match="slots is NULL"):
        M.moe_kv_read(kv, k, v, None, None, None, rows, rows)


def test_descriptions_of_another_kind_and_things_that_are_no_tensors():
    kv, norm, attn = M.KvCfg.make(**KV), M.NormCfg.make(2, 64), M.AttnCfg.make(2, 4, 4)
    slots = tensor(3, dtype=torch.int32)
    for call, what in ((lambda: M.moe_add_norm(kv, None, None, None, None, None), "cfg must be a NormCfg"),
                       (lambda: M.moe_kv_write(norm, None, None, slots, None, None), "cfg must be a KvCfg"),
                       (lambda: M.moe_kv_read(attn, None, None, None, None, slots, None, None), "cfg must be a KvCfg"),
                       (lambda: M.moe_attn_decode(norm, attn, *[None] * 10), "cfg must be a KvCfg"),
                       (lambda: M.moe_attn_decode(kv, kv, *[None] * 10), "attn must be an AttnCfg"),
                       (lambda: M.moe_add_norm(norm, [1.0], None, None, None, None), "x must be a tensor"),
                       (lambda: M.moe_kv_write(kv, "k", None, slots, None, None), "k must be a tensor"),
                       (lambda: M.moe_kv_write(kv, None, None, 3, None, None), "slots must be a tensor"),
                       (lambda: M.moe_add_norm(M.NormCfg.make(2, 64, 7), None, None, None, None, None), "dtype"),
                       (lambda: M.moe_attn_decode(M.KvCfg.make(**KV, dtype=5), attn, *[None] * 10), "dtype")):
        with pytest.raises(M.MoeError, match=what):
            call()


def test_what_the_marshalling_refuses_is_never_passed_on(monkeypatch):
    """Even where the checks in Python find nothing to say."""
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: called.append(name) or 0

    M.lib()
    monkeypatch.setattr(binding, "_native", lambda *args, **kw: False)
    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(binding, "_stream", lambda stream: 0)
    kv, norm, attn = M.KvCfg.make(**KV), M.NormCfg.make(2, 64), M.AttnCfg.make(2, 4, 4)
    anything = torch.empty(0, dtype=torch.int32)
    monkeypatch.setattr(binding, "_array", lambda *args: None)
    monkeypatch.setattr(binding, "_head_rows", lambda *args: (None, 0))
    for call in (lambda: M.moe_add_norm(norm, None, None, None, None, None), lambda: M.moe_kv_write(kv, None, None, anything, None, None),
                 lambda: M.moe_kv_read(kv, None, None, None, None, anything, None, None), lambda: M.moe_attn_decode(kv, attn, *[None] * 10)):
        with pytest.raises(M.MoeError):
            call()
    assert called == []
