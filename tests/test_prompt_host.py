"""Host-only checks of rotary positions, prompts and scores by distance: the oracle against its definitions, frequencies, workspace sizes, and every refusal of
the library and of the binding, before anything is launched."""
import ctypes as C
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from paper_2106_10715_amd import binding

KV = dict(pages=8, page_size=16, heads=2, head_dim=64)


def test_oracle_masked_attention_by_sums():
    """Row by row, key by key, from the formula."""
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 8)), rng.standard_normal((11, 8)), rng.standard_normal((11, 8))
    bias = rng.standard_normal(4 + 2 + 1)
    place, first, end = [6, 7, 8, 9, 10], [0, 3, 9, 2, 0], [7, 8, 9, 20, 0]
    out, lse, _, p = D.masked_attention(q, k, v, 0.4, place, first, end, window=5, cap=1.5, slope=0.25, bias=bias, back=4, ahead=2)
    for i in range(5):
        weights = {}
        for t in range(11):
            if max(first[i], place[i] - 4) <= t < end[i]:
                d = place[i] - t
                x = 1.5 * math.tanh(0.4 * sum(q[i] * k[t]) / 1.5) - 0.25 * abs(d) + bias[min(max(d, -2), 4) + 2]
                weights[t] = math.exp(x)
        total = sum(weights.values())
        if not weights:
            assert (out[i] == 0).all() and lse[i] == -math.inf
            continue
        assert np.allclose(out[i], sum(w * v[t] for t, w in weights.items()) / total, atol=1e-12) and abs(lse[i] - math.log(total)) < 1e-12
    assert sorted(np.nonzero(p.sum(1) == 0)[0]) == [2, 4]


def test_oracle_rotary_by_rotation_matrices():
    rng = np.random.default_rng(4)
    x, freqs = rng.standard_normal((3, 2, 10)), D.frequencies(6)
    for neighbours in (False, True):
        got = D.rotary(x, [0, 5, -7], freqs, 6, neighbours, 1.1)
        for n, p in enumerate((0, 5, -7)):
            for i in range(3):
                a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + 3)
                c, s = math.cos(p * freqs[i]), math.sin(p * freqs[i])
                want = 1.1 * x[n][:, [a, b]] @ np.array([[c, s], [-s, c]])
                assert np.allclose(got[n][:, [a, b]], want, atol=1e-14)
        assert np.array_equal(got[..., 6:], x[..., 6:])


@pytest.mark.parametrize("rot", [2, 4, 32, 96, 128, 256])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_frequencies(rot, scaling):
    for base, factor, original, slow, fast in ((10000.0, 8.0, 4096, 1.0, 32.0), (500000.0, 1.5, 8192, 1.0, 4.0), (1e6, 40.0, 1, 0.0, 2.5)):
        cfg = M.RopeCfg.make(1, 1, 256, rot, scaling=scaling, base=base, factor=factor, original=original, slow=slow, fast=fast)
        got = M.moe_rope_frequencies(cfg)
        want = D.frequencies(rot, base, scaling, factor, original, slow, fast)
        assert got.dtype == torch.float64 and got.shape == (rot // 2,)
        assert np.abs(got.numpy() / want - 1).max() < 2.0 ** -46                 # a power of a power: its exponent's rounding times log base
        if scaling == "parts":
            plain = D.frequencies(rot, base)
            assert (got.numpy() <= plain * (1 + 1e-12)).all() and (got.numpy() >= plain / factor * (1 - 1e-12)).all()
    assert M.moe_rope_frequencies(M.RopeCfg.make(1, 1, 16, 2, scaling="base", factor=4.0)).tolist() == [1.0]


@pytest.mark.parametrize("kw,frag", [
    (dict(q_heads=-1), "q_heads"), (dict(q_heads=1025), "q_heads"), (dict(k_heads=1025), "k_heads"), (dict(head_dim=24), "head_dim"), (dict(head_dim=272), "head_dim"),
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=7), "rot_dim"), (dict(rot_dim=66), "rot_dim"), (dict(pairs=2), "pairs"), (dict(dtype=2), "dtype"),
    (dict(amplitude=float("nan")), "amplitude"), (dict(amplitude=float("inf")), "amplitude")])
def test_rope_refuses_a_bad_description(kw, frag):
    L = M.lib()
    cfg = M.RopeCfg.make(**{**dict(q_heads=2, k_heads=1, head_dim=64), **kw})
    for rc in (L.moe_rope(C.addressof(cfg), 1, *[None] * 3, 0, None, 0, None, 0, None, 0, None), L.moe_rope_frequencies(C.addressof(cfg), None)):
        assert rc == -1 and frag.encode() in L.moe_last_error()


@pytest.mark.parametrize("kw,frag", [
    (dict(base=0.0), "base"), (dict(base=float("inf")), "base"), (dict(scaling=4), "scaling"), (dict(scaling=-1), "scaling"), (dict(scaling="linear", factor=0.0), "factor"),
    (dict(scaling="base", factor=float("nan")), "factor"), (dict(scaling="parts", original=0), "parts need"), (dict(scaling="parts", original=9, slow=-1.0), "parts need"),
    (dict(scaling="parts", original=9, slow=2.0, fast=2.0), "parts need"), (dict(scaling="parts", original=9, fast=float("inf")), "parts need")])
def test_frequencies_refuse_a_bad_description(kw, frag):
    with pytest.raises(M.MoeError, match=frag):
        M.moe_rope_frequencies(M.RopeCfg.make(2, 1, 64, **kw))


def test_rope_refuses_null_misaligned_and_contradicting_arguments():
    L = M.lib()
    buf = C.create_string_buffer(4096)
    al = (C.addressof(buf) + 255) & ~255
    cfgs = [M.RopeCfg.make(2, 1, 64), M.RopeCfg.make(2, 0, 64), M.RopeCfg.make(0, 1, 64)]
    R, no_k, no_q = (C.addressof(c) for c in cfgs)

    def refused(rc, frag):
        assert rc == -1, L.moe_last_error()
        assert frag.encode() in L.moe_last_error()

    good = [al, al, al, 128, al + 512, 128, al, 64, al + 512, 64, None]                     # positions, freqs, q, stride, q_out, stride, k, ...
    refused(L.moe_rope(None, 1, *good), "cfg is NULL")
    refused(L.moe_rope(R, -1, *good), "n must be")
    refused(L.moe_rope(R, (1 << 24) + 1, *good), "n must be")
    for at, frag in ((0, "positions is NULL"), (1, "freqs is NULL"), (2, "q is NULL"), (4, "q_out is NULL"), (6, "k is NULL"), (8, "k_out is NULL")):
        args = list(good)
        args[at] = None
        refused(L.moe_rope(R, 1, *args), frag)
    for at, value, frag in ((2, al + 8, "q must be"), (8, al + 2, "k_out must be"), (3, 120, "stride of q "), (5, 132, "stride of q_out"), (9, 1 << 31, "stride of k_out")):
        args = list(good)
        args[at] = value
        refused(L.moe_rope(R, 1, *args), frag)
    args = list(good)
    args[4], args[5] = al, 136
    refused(L.moe_rope(R, 1, *args), "keep its stride")
    refused(L.moe_rope(no_k, 1, *good), "k has no heads")
    refused(L.moe_rope(no_q, 1, *good), "q has no heads")
    assert L.moe_rope(R, 0, None, al, *[None, 0] * 4, None) == 0
    assert L.moe_rope(R, 1, al, al, *[None, 0] * 4, None) == 0                              # neither side


@pytest.mark.parametrize("kw,frag", [
    (dict(tokens=-1), "tokens must"), (dict(tokens=1 << 22), "tokens must"), (dict(tokens=1 << 21, q_heads=256), "tokens * q_heads"), (dict(B=-1), "B must"), (dict(B=4097), "B must"), (dict(q_heads=3), "q_heads"),
    (dict(q_heads=1026), "q_heads"), (dict(table_pages=0), "table_pages"), (dict(table_pages=(1 << 20) + 1), "table_pages"), (dict(window=-1), "window"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale")])
def test_prompts_refuse_a_bad_description(kw, frag):
    L = M.lib()
    kv, prompt = M.KvCfg.make(**KV), M.PromptCfg.make(**{**dict(tokens=3, B=1, q_heads=4, table_pages=4), **kw})
    n = C.c_size_t(0)
    for rc in (L.moe_attn_prompt_workspace_bytes(C.addressof(kv), C.addressof(prompt), C.byref(n)),
               L.moe_attn_prompt(C.addressof(kv), C.addressof(prompt), None, None, 0, *[None] * 15)):
        assert rc == -1 and frag.encode() in L.moe_last_error()


@pytest.mark.parametrize("kw,frag", [
    (dict(cap=-1.0), "cap"), (dict(cap=float("nan")), "cap"), (dict(cap=float("inf")), "cap"), (dict(cap=1e-38), "cap"), (dict(cap=1e38), "cap"), (dict(back=-1), "back"),
    (dict(back=65536), "back"), (dict(ahead=-1), "ahead"), (dict(ahead=65536), "ahead")])
def test_scores_refuse_a_bad_description(kw, frag):
    L = M.lib()
    kv, prompt, attn, scores = M.KvCfg.make(**KV), M.PromptCfg.make(3, 1, 4, 4), M.AttnCfg.make(1, 4, 4), M.ScoresCfg.make(**kw)
    for rc in (L.moe_attn_prompt(C.addressof(kv), C.addressof(prompt), C.addressof(scores), None, 0, *[None] * 15),
               L.moe_attn_decode_scored(C.addressof(kv), C.addressof(attn), C.addressof(scores), None, 0, *[None] * 12)):
        assert rc == -1 and frag.encode() in L.moe_last_error()


def test_attention_refuses_null_misaligned_and_contradicting_arguments():
    L = M.lib()
    buf = C.create_string_buffer(4096)
    al = (C.addressof(buf) + 255) & ~255
    kv, e4, prompt, attn, scores = M.KvCfg.make(**KV), M.KvCfg.make(**KV, cache_dtype="e4m3"), M.PromptCfg.make(3, 1, 4, 4), M.AttnCfg.make(2, 4, 4), M.ScoresCfg.make(cap=2.0)
    K, E, P, A, S = (C.addressof(c) for c in (kv, e4, prompt, attn, scores))

    def refused(rc, frag, code=-1):
        assert rc == code, L.moe_last_error()
        assert frag.encode() in L.moe_last_error()

    tiny = M.PromptCfg.make(3, 1, 4, 4, scale=2.0 ** -65)
    refused(L.moe_attn_prompt(K, C.addressof(tiny), None, al, 256, al, al, None, None, al, al, al, None, None, al, None, al, al, al, None), "scale must be 0 or at least 2^-64")
    # q, stride, pages, scales, table, lens, starts, first, end, slopes, bias, out, lse, ws, stream
    good = [al, 256, al, al, None, None, al, al, al, None, None, al, al, al, al, al, None]
    for at, frag in ((0, "q is NULL"), (2, "k_pages is NULL"), (3, "v_pages is NULL"), (6, "table is NULL"), (7, "lens is NULL"), (8, "starts is NULL"), (13, "out is NULL"),
                     (15, "ws is NULL")):
        args = list(good)
        args[at] = None
        refused(L.moe_attn_prompt(K, P, S, *args), frag)
    refused(L.moe_attn_prompt(None, P, S, *good), "cfg is NULL")
    refused(L.moe_attn_prompt(K, None, S, *good), "prompt is NULL")
    refused(L.moe_attn_prompt(K, P, None, *good), "a bias needs scores")
    refused(L.moe_attn_prompt(E, P, S, *good), "k_scales is NULL")
    refused(L.moe_attn_prompt(K, P, S, *good[:1], 248, *good[2:]), "stride of q")
    refused(L.moe_attn_prompt(K, P, S, *good[:15], al + 16, None), "256-byte", code=-3)
    refused(L.moe_attn_prompt(K, P, S, *good[:13], al + 8, *good[14:]), "out must be")
    for tokens, B in ((0, 1), (3, 0)):
        none = M.PromptCfg.make(tokens, B, 4, 4)
        assert L.moe_attn_prompt(K, C.addressof(none), None, None, 0, al, al, *[None] * 13) == 0
    assert L.moe_attn_prompt_workspace_bytes(K, P, None) == -1

    # q, stride, pages, scales, table, lens, slopes, bias, out, lse, ws, stream
    good = [al, 256, al, al, None, None, al, al, al, al, al, al, al, None]
    for at, frag in ((0, "q is NULL"), (2, "k_pages is NULL"), (6, "table is NULL"), (7, "lens is NULL"), (10, "out is NULL"), (12, "ws is NULL")):
        args = list(good)
        args[at] = None
        refused(L.moe_attn_decode_scored(K, A, S, *args), frag)
    refused(L.moe_attn_decode_scored(K, None, S, *good), "attn is NULL")
    refused(L.moe_attn_decode_scored(K, A, None, *good), "a bias needs scores")
    refused(L.moe_attn_decode_scored(K, A, S, *good[:12], al + 16, None), "256-byte", code=-3)
    none = M.AttnCfg.make(0, 4, 4)
    assert L.moe_attn_decode_scored(K, C.addressof(none), None, None, 0, al, al, *[None] * 10) == 0


def test_binding_names_what_it_refuses():
    """On the CPU no tensor is in device memory: what is wrong beside that is said first."""
    kv, prompt, attn, rope, scores = M.KvCfg.make(**KV), M.PromptCfg.make(3, 2, 4, 4), M.AttnCfg.make(2, 4, 4), M.RopeCfg.make(2, 1, 64), M.ScoresCfg.make(back=3, ahead=1)
    b = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt)
    i = lambda *shape: b(*shape, dt=torch.int32)
    call = lambda **kw: M.moe_attn_prompt(**{**dict(cfg=kv, prompt=prompt, scores=None, q=None, k_pages=None, v_pages=None, k_scales=None, v_scales=None, table=None, lens=None,
                                                    starts=None, first=None, end=None, slopes=None, bias=None, out=None, lse=None, ws=None), **kw})
    one = lambda **kw: M.moe_attn_decode_scored(**{**dict(cfg=kv, attn=attn, scores=None, q=None, k_pages=None, v_pages=None, k_scales=None, v_scales=None, table=None, lens=None,
                                                         slopes=None, bias=None, out=None, lse=None, ws=None), **kw})
    turn = lambda **kw: M.moe_rope(**{**dict(cfg=rope, positions=i(3), freqs=None, q=None, q_out=None), **kw})
    for f, kw, what in (
            (call, dict(cfg=rope, q=b(1)), "cfg must be a KvCfg"), (call, dict(prompt=attn, q=b(1)), "prompt must be a PromptCfg"), (call, dict(scores=kv, q=b(1)), "scores must be a ScoresCfg"),
            (call, dict(q=b(3, 4, 32)), "q must be"), (call, dict(q=b(2, 4, 64)), "q must be"), (call, dict(starts=i(2)), "starts must be a contiguous"), (call, dict(first=i(4)), "first must be"),
            (call, dict(end=b(3)), "end must be"), (call, dict(slopes=b(4)), "slopes must be"), (call, dict(scores=scores, bias=b(4, 4, dt=torch.float32)), "bias must be"),
            (call, dict(bias=b(4, 5, dt=torch.float32)), "bias must be"), (call, dict(lse=b(3, 4)), "lse must be"), (call, dict(out=b(3, 4, 64).transpose(0, 1)), "out must be"),
            (call, dict(ws=b(7, dt=torch.uint8)), "ws is smaller"), (call, dict(ws=b(1 << 20, dt=torch.uint8)), "ws must be in device memory"), (call, dict(lens=i(2)), "lens must be in device"),
            (call, dict(table="t"), "table must be a tensor"),
            (one, dict(cfg=attn, q=b(1)), "cfg must be a KvCfg"), (one, dict(attn=prompt, q=b(1)), "attn must be an AttnCfg"), (one, dict(slopes=b(3, dt=torch.float32)), "slopes must be"),
            (one, dict(scores=scores, bias=b(4, 5, dt=torch.float32)), "bias must be in device"), (one, dict(ws=b(1, dt=torch.uint8)), "ws is smaller"), (one, dict(out=b(2, 4, 32)), "out must be"),
            (turn, dict(cfg=kv, q=b(1)), "cfg must be a RopeCfg"), (turn, dict(positions=None), "positions is NULL"), (turn, dict(positions=b(3)), "positions must be a contiguous"),
            (turn, dict(freqs=b(32)), "freqs must be"), (turn, dict(freqs=b(31, dt=torch.float64)), "freqs must be"), (turn, dict(q=b(3, 2, 32)), "q must be"), (turn, dict(q_out=b(3, 1, 64)), "q_out must be"),
            (turn, dict(k=b(3, 1, 64).transpose(1, 2)), "k must be"), (turn, dict(k_out=b(3, 1, 64)), "k_out must be in device"), (turn, dict(freqs=b(32, dt=torch.float64)), "freqs must be in device")):
        with pytest.raises(M.MoeError, match=what):
            f(**kw)


def test_what_the_marshalling_refuses_is_never_passed_on(monkeypatch):
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: called.append(name) or 0

    M.lib()
    monkeypatch.setattr(binding, "_native", lambda *args, **kw: False)
    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(binding, "_array", lambda *args: None)
    monkeypatch.setattr(binding, "_head_rows", lambda *args: None)
    kv, prompt, attn, rope = M.KvCfg.make(**KV), M.PromptCfg.make(3, 2, 4, 4), M.AttnCfg.make(2, 4, 4), M.RopeCfg.make(2, 1, 64)
    for call in (lambda: M.moe_attn_prompt(kv, prompt, *[None] * 17), lambda: M.moe_attn_decode_scored(kv, attn, *[None] * 14),
                 lambda: M.moe_rope(rope, torch.empty(0, dtype=torch.int32), None, None, None)):
        with pytest.raises(M.MoeError, match="not as its description says"):
            call()
    assert called == []


@pytest.mark.parametrize("counts", [[0], [1], [7], [8], [0, 3, 9, 0, 17, 1], [2000] * 40, [70000, 1, 65536]])
@pytest.mark.parametrize("most", [1, 8, 1 << 16])
def test_the_example_takes_prompts_in_calls(counts, most):
    spec = importlib.util.spec_from_file_location("decode_example", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    if sum(counts) // most > 100:
        most = 8000
    calls = [list(c) for c in example.Decoder.in_calls(counts, most)]
    assert [sum(c) for c in zip(*calls)] == (counts if sum(counts) else [])
    assert all(sum(c) == most for c in calls[:-1]) and all(0 < sum(c) <= most for c in calls)
    done = [0] * len(counts)
    for c in calls:                                                # a sequence begins when the one before it is done
        done = [a + b for a, b in zip(done, c)]
        assert sum(0 < a < b for a, b in zip(done, counts)) <= 1
