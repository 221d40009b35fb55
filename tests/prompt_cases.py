"""What the tests of scores by distance, masks and prompts share: masks by name, scores' arrays, a call and its comparison with the oracle.

Tolerance, per element, of an attention row of n keys with weights p (they sum to 1), A = sum p |v| and logits l:
  the sum q . k in fp32 (dim + 8 roundings of at most sum |q k| scale), its scaling, the tanh (within 8 * 2^-24 of its value), the bias and the slope's
  product, each within 2^-23 of the largest term: a logit is off by
      off = 2^-24 ((dim + 8) scale max sum |q k| + 16 max |l| + 4 max |bias| + 4 max |slope distance| + 8 cap),
  (the last with bf16 activations and caps up to 64, where the tanh is 1 - 2 / (e + 1), e = exp 2z: its exponent and e are off by 2^-23 of e each, what
  changes the quotient by at most 2^-23, which is off by 2^-23 itself, and the difference by 2^-24: 5 * 2^-24 in all, of the cap)
  which changes numerator and total by as much relatively each; their sums over runs, lanes, waves and parts by (n / 16 + 64) 2^-24 each;
  weights and output are rounded to bf16 where the activations are (2^-8 each, of A and of the result)."""
import math

import numpy as np
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from test_gpu_decoder import HALF, f64, normal, within

MASKS = ["causal", "prefix", "documents", "both", "all", "odd"]


def mask(kind, past, new, seed=0):
    """(first, end) of each of the `new` last tokens of past + new; None where the call's default is meant."""
    total, at = past + new, np.arange(past, past + new)
    if kind == "causal":
        return None, None
    if kind == "prefix":
        return None, np.maximum(at + 1, total // 2)
    if kind == "all":
        return None, np.full(new, total)
    if kind == "odd":                                             # any stretch, empty ones and ends outside of the sequence among them
        rng = np.random.default_rng(1000 * seed + total)
        first = rng.integers(-5, total + 3, new)
        return first, first + rng.integers(-3, total + 2, new)
    ends = np.cumsum(1 + (np.arange(total + 1) * 37 + 11 * seed) % 61)
    doc = np.searchsorted(ends, at, side="right")
    first = np.concatenate([[0], ends])[doc]
    return first, (np.minimum(ends[doc], total) if kind == "both" else None)


def spans(kind, news):
    """(first, end) [tokens] over sequences (past, new), the defaults written out, and which of the two are arrays of the call."""
    first, end, given = [], [], (False, False)
    for b, (past, new) in enumerate(news):
        f, e = mask(kind, past, new, b)
        given = (given[0] or f is not None, given[1] or e is not None)
        first.append(np.zeros(new, np.int64) if f is None else f)
        end.append(np.arange(past, past + new) + 1 if e is None else e)
    return np.concatenate(first), np.concatenate(end), given


class Scores:
    """Scores of `heads` query heads by name: plain, cap, slopes, table (a bias for near distances), each (all of it)."""

    def __init__(self, kind, heads, seed=0, back=21, ahead=9, cap=3.0):
        self.cap = cap if kind in ("cap", "each") else 0.0
        self.slopes = torch.exp2(-8.0 * torch.arange(1, heads + 1) / heads).cuda() if kind in ("slopes", "each") else None
        self.back, self.ahead = (back, ahead) if kind in ("table", "each") else (0, 0)
        self.bias = normal(900 + seed, (heads, back + ahead + 1), "f32", 2.0) if kind in ("table", "each") else None
        self.cfg = None if kind in ("plain", "slopes") else M.ScoresCfg.make(self.cap, self.back, self.ahead)

    def of(self, head):
        return dict(cap=float(np.float32(self.cap)), slope=0.0 if self.slopes is None else float(self.slopes[head]), bias=None if self.bias is None else f64(self.bias[head]),
                    back=self.back, ahead=self.ahead)

    def largest(self, head, distance):
        """The largest bias, and the largest a slope makes of this distance."""
        return (0.0 if self.bias is None else float(self.bias[head].abs().max())) + (0.0 if self.slopes is None else float(self.slopes[head]) * distance)


def check_rows(out, lse, q, k, v, scale, dtype, place, first, end, window, scores, head, what):
    """Rows of one query head of one sequence against the oracle."""
    if len(q) == 0:
        return
    ref, ref_lse, logits, p = D.masked_attention(q, k, v, scale, place, first, end, window, **scores.of(head))
    n = len(k)
    qk = (np.abs(q) @ np.abs(k).T).max(axis=1, initial=0.0) if n else np.zeros(len(q))
    off = 2 ** -24 * ((q.shape[1] + 8) * scale * qk + 16 * np.abs(logits).max(axis=1, initial=0.0) + 4 * scores.largest(head, n)
                    + (8 * scores.cap if dtype == "bf16" and scores.cap <= 64 else 0.0))
    sums = (n / 16 + 64) * 2 ** -24
    none = ref_lse == -np.inf
    assert (out[none] == 0).all() and (lse[none] == -np.inf).all(), f"{what}: rows without keys"
    weights = 2 ** -8 if dtype == "bf16" else 0.0
    tol = HALF[dtype] * np.abs(ref) + (weights + 2 * off[:, None] + 2 * sums) * (p @ np.abs(v)) * (1 + HALF[dtype])
    within(out, ref, tol, what)
    some = ~none
    if some.any():
        within(lse[some], ref_lse[some], off[some] + sums + 2 ** -22 * np.abs(ref_lse[some]) + 2 ** -22, f"lse, {what}")


def run_prompt(cfg, arrays, q, table, lens, starts, first=None, end=None, window=0, scale=0.0, scores=None, want_lse=True, stream=None):
    n, heads, dim = q.shape
    scores = scores or Scores("plain", heads)
    B = len(lens)
    prompt = M.PromptCfg.make(n, B, heads, table.shape[1], scale=scale, window=window)
    need = M.moe_attn_prompt_workspace_bytes(cfg, prompt)
    ws = torch.full((need + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((n, heads, dim), 7, dtype=q.dtype, device="cuda")
    lse = torch.full((n, heads), 7, dtype=torch.float32, device="cuda") if want_lse else None
    ints = lambda v: None if v is None else torch.as_tensor(np.asarray(v), dtype=torch.int32).cuda()
    M.moe_attn_prompt(cfg, prompt, scores.cfg, q, *arrays, table, ints(lens), ints(starts), ints(first), ints(end), scores.slopes, scores.bias, out, lse,
                      ws, stream=stream)
    torch.cuda.synchronize()
    assert (ws[need:] == 0xff).all(), "written past the workspace"
    return out, lse


def run_and_check(cfg, arrays, q, table, news, kind="causal", window=0, scale=0.0, scores=None, only=None, heads_only=None):
    """A call over sequences (past, new), all of it (or the sequences `only`, the heads `heads_only`) against the oracle."""
    n, heads, dim = q.shape
    dt = {0: "f32", 1: "bf16"}[cfg.dtype]
    scores = scores or Scores("plain", heads)
    lens, starts = [p + m for p, m in news], np.concatenate([[0], np.cumsum([m for _, m in news])])
    first, end, given = spans(kind, news)
    out, lse = run_prompt(cfg, arrays, q, table, lens, starts, first if given[0] else None, end if given[1] else None, window, scale, scores)
    o, l, qs = f64(out), f64(lse), f64(q)
    group, c, tab = heads // cfg.heads, scale or 1 / math.sqrt(dim), table.cpu().numpy()
    pages, scales = [f64(t) for t in arrays[:2]], [None if t is None else f64(t) for t in arrays[2:]]
    for b, (past, new) in enumerate(news):
        if only is not None and b not in only or new == 0:
            continue
        k, v = (D.paged_rows(t, s, tab[b], 0, past + new) for t, s in zip(pages, scales))
        rows = slice(starts[b], starts[b + 1])
        f, e = np.clip(first[rows], 0, None), np.clip(end[rows], None, past + new)
        for h in range(heads) if heads_only is None else heads_only:
            check_rows(o[rows, h], l[rows, h], qs[rows, h], k[h // group], v[h // group], c, dt, np.arange(past, past + new), f, e, window, scores, h,
                       f"sequence {b}, head {h}")
    return out, lse
