"""examples/decode.py with prompts, rotary positions and capped or sloped scores: prompts taken in in pieces and tokens generated behind them, by a small decoder
against the fp64 oracle on the same weights.  Tolerances as in test_gpu_decode_example.py: 2 layers store some eight results of 16 bits each, 2e-2 of the
result's norm; an 8-bit cache or projection 5e-2."""
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


class Reference:
    """The same decoder in 64 bits, one sequence after the other."""

    def __init__(self, dec, rot, neighbours, cap, eps=1e-6):
        self.dec, self.rot, self.neighbours, self.cap, self.eps = dec, rot, neighbours, cap, eps
        self.slopes = np.zeros(dec.heads) if dec.slopes is None else f64(dec.slopes)
        self.freqs = D.frequencies(rot) if rot else None
        self.past = [[[] for _ in range(dec.batch)] for _ in dec.weights]
        self.weights = [(f64(w.norm_attn), f64(w.qkv8) * f64(w.qkv8_scale) if dec.qkv == "e4m3" else f64(w.qkv), f64(w.o), f64(w.norm_moe), f64(w.gate),
                         [tuple(f64(m) for m in w.expert(e)) for e in range(dec.moe.E)]) for w in dec.weights]

    def quantised(self, t):
        scale = D.e4m3_scale(t)[..., None]
        return D.e4m3(t / scale) * scale

    def run(self, b, x, first=None, end=None):
        dec = self.dec
        H, dim = dec.kv_heads, dec.dim
        h, delta = np.zeros_like(x), x
        for (na, qkv, wo, nm, gate, experts), past in zip(self.weights, self.past):
            h, y = D.add_norm(delta, h, na, self.eps)
            rows = ((self.quantised(y) if dec.qkv == "e4m3" else y) @ qkv.T).reshape(len(x), -1, dim)
            q, k, v = rows[:, :dec.heads], rows[:, dec.heads:dec.heads + H], rows[:, dec.heads + H:]
            done = 0 if not past[b] else len(past[b][0])
            at = np.arange(done, done + len(x))
            if self.rot:
                q, k = (D.rotary(t, at, self.freqs, self.rot, self.neighbours) for t in (q, k))
            if dec.caches[0][2] is not None:
                k, v = self.quantised(k), self.quantised(v)
            past[b] = [k, v] if not past[b] else [np.concatenate([past[b][0], k]), np.concatenate([past[b][1], v])]
            lo, hi = (0 * at if first is None else first), (at + 1 if end is None else end)
            o = np.concatenate([D.masked_attention(q[:, j], past[b][0][:, j // (dec.heads // H)], past[b][1][:, j // (dec.heads // H)], dim ** -0.5, at, lo, hi,
                                                   cap=self.cap, slope=self.slopes[j])[0] for j in range(dec.heads)], 1)
            h, y = D.add_norm(o @ wo.T, h, nm, self.eps)
            delta = O.layer_forward(y, gate, lambda e: experts[e], dec.moe.E, dec.moe.k, None, 1)[0]
        return h + delta


@pytest.mark.parametrize("cache,qkv,rotary,cap,slopes,tol", [
    ("bf16", "bf16", {}, 0.0, False, 2e-2), ("bf16", "bf16", dict(rot_dim=32, pairs="neighbours"), 5.0, False, 2e-2), ("bf16", "bf16", None, 0.0, True, 2e-2),
    ("e4m3", "bf16", {}, 5.0, True, 5e-2), ("bf16", "e4m3", {}, 0.0, False, 5e-2)])
def test_prompts_in_pieces_then_tokens(cache, qkv, rotary, cap, slopes, tol):
    dec = X.Decoder(batch=3, layers=2, d=256, heads=4, kv_heads=2, dim=64, f=128, E=2, k=2, room=200, page=16, cache=cache, qkv=qkv, rotary=rotary, cap=cap, slopes=slopes)
    ref = Reference(dec, 0 if rotary is None else rotary.get("rot_dim", 64), rotary is not None and rotary.get("pairs") == "neighbours", cap)
    g = torch.Generator().manual_seed(6)
    draw = lambda n: torch.randn((n, 256), generator=g).to(torch.bfloat16)

    def close(got, want, what):
        err = np.linalg.norm(got - want) / np.linalg.norm(want)
        assert err <= tol, f"{what}: {err:.3e}"

    for piece, counts in enumerate(([40, 0, 17], [1, 70, 33])):
        x = draw(sum(counts))
        got = f64(dec.prompt(x.cuda(), counts))
        at = np.cumsum([0] + counts)
        for b in range(3):
            if counts[b]:
                close(got[at[b]:at[b + 1]], ref.run(b, f64(x[at[b]:at[b + 1]])), f"piece {piece}, sequence {b}")
    for step in range(4):
        x = draw(3)
        got = f64(dec.step(x.cuda()))
        for b in range(3):
            close(got[b:b + 1], ref.run(b, f64(x[b:b + 1])), f"step {step}, sequence {b}")


def test_a_prompt_whose_prefix_sees_all_of_itself():
    """The prefix mask through all layers."""
    dec = X.Decoder(batch=1, layers=2, d=256, heads=4, kv_heads=4, dim=64, f=128, E=2, k=2, room=200, page=16, rotary={})
    ref = Reference(dec, 64, False, 0.0)
    x = torch.randn((90, 256), generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    end = np.maximum(np.arange(90) + 1, 50)
    got = f64(dec.prompt(x.cuda(), [90], None, torch.from_numpy(end).int().cuda()))
    want = ref.run(0, f64(x), end=end)
    assert np.linalg.norm(got - want) / np.linalg.norm(want) <= 2e-2
