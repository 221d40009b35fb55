"""examples/decode.py: a prompt taken in at once, in two calls, and by single tokens, on the same weights.  Each is within 2e-2 of the result's norm of its 64-bit form
(5e-2 with an 8-bit cache; test_gpu_prompt_example.py), so two of them, off by t of it each,
are within 2 t / (1 - t) of each other by the norm of either."""
import numpy as np
import pytest
import torch

from test_gpu_prompt_example import X, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,rotary,cap,slopes,t", [
    ("bf16", {}, 0.0, False, 2e-2), ("bf16", dict(rot_dim=32, pairs="neighbours"), 5.0, False, 2e-2), ("bf16", None, 0.0, True, 2e-2), ("e4m3", {}, 5.0, True, 5e-2)])
def test_a_prompt_at_once_and_by_single_tokens(cache, rotary, cap, slopes, t):
    lens, most = [70, 33], 70
    g = torch.Generator().manual_seed(8)
    x = [torch.randn((n, 256), generator=g).to(torch.bfloat16).cuda() for n in lens]
    decoder = lambda: X.Decoder(batch=2, layers=2, d=256, heads=4, kv_heads=2, dim=64, f=128, E=2, k=2, room=100, page=16, cache=cache, rotary=rotary, cap=cap, slopes=slopes)

    dec = decoder()
    whole = f64(dec.prompt(torch.cat(x), lens))
    whole = [whole[:lens[0]], whole[lens[0]:]]
    dec = decoder()
    a = f64(dec.prompt(torch.cat([x[0][:41], x[1][:1]]), [41, 1]))
    b = f64(dec.prompt(torch.cat([x[0][41:], x[1][1:]]), [29, 32]))
    pieces = [np.concatenate([a[:41], b[:29]]), np.concatenate([a[41:], b[29:]])]
    dec = decoder()
    steps = [f64(dec.step(torch.stack([x[i][min(at, lens[i] - 1)] for i in range(2)]))) for at in range(most)]    # (the shorter one's last token again past its end)
    single = [np.stack([s[i] for s in steps[:lens[i]]]) for i in range(2)]
    for i in range(2):
        for name, got in (("in two calls", pieces[i]), ("by single tokens", single[i])):
            err = np.linalg.norm(got - whole[i]) / np.linalg.norm(whole[i])
            assert err <= 2 * t / (1 - t), f"sequence {i}, {name}: {err:.3e}"
