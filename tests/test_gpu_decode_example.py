"""examples/decode.py, the operators used together: several steps of a small decoder against the fp64 oracle on the same weights.

Both experts are selected for every token (k = E), so that a rounded hidden state cannot flip a selection.  bf16 stores some eight
intermediate results per layer, each off by at most 2^-8 (2^-9 root-mean-square over 3 on the whole): 2 layers stay below 2e-2 of the
result's norm.  An 8-bit cache or projection moves values by up to 2^-4 where a rounded input falls to the other side of a border, a
sixteenth of them at most: 5e-2."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from oracle import moe_oracle as O

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_spec = importlib.util.spec_from_file_location("decode_example", os.path.join(ROOT, "examples", "decode.py"))
X = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(X)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def reference(dec, xs, eps=1e-6):
    """The same steps in 64 bits: hidden states [steps, batch, d]."""
    B, H, G, dim = dec.batch, dec.kv_heads, dec.heads // dec.kv_heads, dec.dim
    e4 = dec.caches[0][2] is not None
    past = [([], []) for _ in dec.weights]
    weights = [(f64(w.norm_attn), f64(w.qkv), f64(w.o), f64(w.norm_moe), f64(w.gate), [tuple(f64(m) for m in w.expert(e)) for e in range(dec.moe.E)])
               for w in dec.weights]
    if dec.qkv == "e4m3":
        weights = [(na, f64(w.qkv8) * f64(w.qkv8_scale), o, nm, g, ex) for (na, _, o, nm, g, ex), w in zip(weights, dec.weights)]
    out = []
    for x in xs:
        h, delta = np.zeros_like(x), x
        for (na, qkv, wo, nm, gate, experts), (keys, values) in zip(weights, past):
            h, y = D.add_norm(delta, h, na, eps)
            if dec.qkv == "e4m3":
                c = D.e4m3_scale(y)[:, None]
                y = D.e4m3(y / c) * c
            rows = (y @ qkv.T).reshape(B, -1, dim)
            q, k, v = rows[:, :dec.heads], rows[:, dec.heads:dec.heads + H], rows[:, dec.heads + H:]
            if e4:
                k, v = (D.e4m3(t / D.e4m3_scale(t)[..., None]) * D.e4m3_scale(t)[..., None] for t in (k, v))
            keys.append(k)
            values.append(v)
            K, V = np.stack(keys, 2), np.stack(values, 2)                       # [B, H, tokens, dim]
            o = np.stack([np.concatenate([D.attention(q[b, j], K[b, j // G], V[b, j // G], dim ** -0.5)[0] for j in range(dec.heads)]) for b in range(B)])
            h, y = D.add_norm(o @ wo.T, h, nm, eps)
            delta = O.layer_forward(y, gate, lambda e: experts[e], dec.moe.E, dec.moe.k, None, 1)[0]
        out.append(h + delta)
    return np.stack(out)


@pytest.mark.parametrize("cache,qkv,tol", [("bf16", "bf16", 2e-2), ("e4m3", "bf16", 5e-2), ("bf16", "e4m3", 5e-2)])
def test_a_decoder_of_two_layers_step_by_step(cache, qkv, tol):
    dec = X.Decoder(batch=3, layers=2, d=256, heads=4, kv_heads=2, dim=64, f=128, E=2, k=2, room=40, page=16, cache=cache, qkv=qkv)
    g = torch.Generator().manual_seed(5)
    xs = [torch.randn((3, 256), generator=g).to(torch.bfloat16) for _ in range(20)]       # past the first page
    got = [f64(dec.step(x.cuda())) for x in xs]
    want = reference(dec, [f64(x) for x in xs])
    for step, (a, b) in enumerate(zip(got, want)):
        err = np.linalg.norm(a - b) / np.linalg.norm(b)
        assert err <= tol, f"step {step}: {err:.3e}"
