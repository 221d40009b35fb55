"""Prompts whose keys are cut into parts that a second launch joins, with keys, values and queries that are not finite: a row is what it is where nothing is cut.
The tolerance is derived in prompt_cases.py."""
import math

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from prompt_cases import Scores, check_rows, run_prompt
from test_gpu_decoder import TYPES, cache_of, f64, normal, run_attention, tables

pytestmark = pytest.mark.gpu

TOKENS, PAGE, NEW, HEADS, GROUP = 9003, 64, 3, 2, 2
SHAPES = [(dtype, cache, dim) for dtype, cache in TYPES for dim in (64, 128, 256)]


def make(dtype, cache, dim, tokens=TOKENS, room=TOKENS):
    """A sequence whose last NEW tokens are new, in a table for `room` tokens; queries without zeros and of one sign."""
    cfg = M.KvCfg.make(-(-room // PAGE) + 2, PAGE, HEADS, dim, dtype, cache)
    table = tables(71, 1, -(-room // PAGE), cfg.pages)
    return cfg, cache_of(72, cfg, table, [tokens]), normal(73, (NEW, HEADS * GROUP, dim), dtype).abs() + 2 ** -6, table.cuda()


def is_cut(cfg, table, tokens=NEW, B=1):
    return M.moe_attn_prompt_workspace_bytes(cfg, M.PromptCfg.make(tokens, B, HEADS * GROUP, table.shape[1])) > 256


def plant(cfg, arrays, table, side, head, tokens, column, value):
    """`value` in a column (a slice: in all of them) of these tokens' keys (side 0) or values; 8 bits: NaN or -1, the scale -value then."""
    bad = [None if t is None else t.clone() for t in arrays]
    at = torch.as_tensor(tokens)
    index, at = table[0].cpu()[at // PAGE].long().cuda(), (at % PAGE).cuda()
    if cfg.cache_dtype != 2:
        bad[side][index, head, at, column] = value
    elif math.isnan(value):
        bad[side].view(torch.uint8)[index, head, at, column] = 0x7f
    else:
        bad[side].view(torch.uint8)[index, head, at] = 0xb8
        bad[2 + side][index, head, at] = -value
    return bad


def same(got, want, rows, heads):
    """The rows and heads not named keep every bit."""
    other = torch.ones(want[1].shape, dtype=torch.bool, device="cuda")
    for r in rows:
        other[r, heads] = False
    return torch.equal(got[0][other], want[0][other]) and torch.equal(got[1][other], want[1][other])


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
def test_a_query_that_is_nan(dtype, cache, dim):
    """All of its row's logits are NaN in every part, and so is the row; in a call that is cut and in one that is not."""
    for tokens in (TOKENS, 200):
        cfg, arrays, q, table = make(dtype, cache, dim, tokens, tokens)
        assert is_cut(cfg, table) == (tokens == TOKENS)
        want = run_prompt(cfg, arrays, q, table, [tokens], [0, NEW])
        assert all(torch.isfinite(t).all() for t in want)
        q[1, 2, 5] = math.nan
        got = run_prompt(cfg, arrays, q, table, [tokens], [0, NEW])
        assert torch.isnan(got[0][1, 2]).all() and torch.isnan(got[1][1, 2]) and same(got, want, [1], [2]), f"{tokens} tokens"


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
@pytest.mark.parametrize("name,tokens", [("one key", [4000]), ("the first half", range(4608)), ("the second half", range(4400, TOKENS)), ("all", range(TOKENS))])
def test_keys_that_are_nan(name, tokens, dtype, cache, dim):
    """In one part's keys, in all keys of some parts, in all parts: the rows that see them are NaN, whatever the other parts hold.  A row that does not see them keeps every bit."""
    cfg, arrays, q, table = make(dtype, cache, dim)
    assert is_cut(cfg, table)
    first = [0, max(tokens) + 1 if max(tokens) < TOKENS - NEW else 0, 0]
    want = run_prompt(cfg, arrays, q, table, [TOKENS], [0, NEW], first)
    bad = plant(cfg, arrays, table, 0, 1, list(tokens), slice(None), math.nan)
    got = run_prompt(cfg, bad, q, table, [TOKENS], [0, NEW], first)
    rows = [r for r in range(NEW) if first[r] <= min(tokens)]
    assert torch.isnan(got[0][rows][:, 2:]).all() and torch.isnan(got[1][rows][:, 2:]).all() and same(got, want, rows, slice(2, 4))


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
def test_a_whole_part_of_keys_that_are_nan(dtype, cache, dim):
    """NaN in the first keys up to every tile's end within the first eighth, so in all of the first part and nowhere else once."""
    cfg, arrays, q, table = make(dtype, cache, dim)
    want = run_prompt(cfg, arrays, q, table, [TOKENS], [0, NEW])
    for end in range(32, TOKENS // 8, 32):
        got = run_prompt(cfg, plant(cfg, arrays, table, 0, 1, list(range(end)), slice(None), math.nan), q, table, [TOKENS], [0, NEW])
        assert torch.isnan(got[0][:, 2:]).all() and torch.isnan(got[1][:, 2:]).all() and same(got, want, range(NEW), slice(2, 4)), f"{end} keys"


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
def test_parts_whose_logits_are_minus_infinity_weigh_nothing(dtype, cache, dim):
    """The first half's keys have logits of -infinity: what is left is the attention of the others; with all of them a row is as one without keys."""
    cfg, arrays, q, table = make(dtype, cache, dim)
    for tokens in (4608, TOKENS):
        bad = plant(cfg, arrays, table, 0, 1, list(range(tokens)), 3, -math.inf)
        want = run_prompt(cfg, arrays, q, table, [TOKENS], [0, NEW])
        out, lse = run_prompt(cfg, bad, q, table, [TOKENS], [0, NEW])
        assert same((out, lse), want, range(NEW), slice(2, 4))
        if tokens == TOKENS:
            assert (out[:, 2:] == 0).all() and (lse[:, 2:] == -math.inf).all()
            continue
        k, v = (D.paged_rows(f64(t), None if s is None else f64(s), table.cpu().numpy()[0], tokens, TOKENS)[1] for t, s in zip(arrays[:2], arrays[2:]))
        at, none = np.arange(TOKENS - NEW, TOKENS) - tokens, np.zeros(NEW, np.int64)
        for h in (2, 3):
            check_rows(f64(out[:, h]), f64(lse[:, h]), f64(q[:, h]), k, v, 1 / math.sqrt(dim), dtype, at, none, at + 1, 0, Scores("plain", 4), h, f"head {h}")


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
def test_values_that_are_not_finite(dtype, cache, dim):
    """A value's column in one part: that column of the rows that see it, and nothing else."""
    cfg, arrays, q, table = make(dtype, cache, dim)
    first = [0, 5000, 0]
    want = run_prompt(cfg, arrays, q, table, [TOKENS], [0, NEW], first)
    for value in (math.nan,) if cache == "e4m3" else (math.nan, math.inf, -math.inf):
        got, lse = run_prompt(cfg, plant(cfg, arrays, table, 1, 1, [1234], 7, value), q, table, [TOKENS], [0, NEW], first)
        column = got[[0, 2], 2:, 7].float()
        assert torch.isnan(column).all() if math.isnan(value) else (column == value).all()
        got[[0, 2], 2:, 7] = want[0][[0, 2], 2:, 7]
        assert torch.equal(got, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dtype,cache,dim", SHAPES)
def test_parts_without_keys(dtype, cache, dim):
    """A sequence much shorter than its table, of whose parts most have no keys; rows whose mask leaves nothing, next to one that sees some, and to NaN; no tokens at all."""
    n = 300
    cfg, arrays, q, table = make(dtype, cache, dim, n, 16000)
    assert is_cut(cfg, table)
    k, v = (D.paged_rows(f64(t), None if s is None else f64(s), table.cpu().numpy()[0], 0, n) for t, s in zip(arrays[:2], arrays[2:]))
    at = np.arange(n - NEW, n)
    for first, end in ((np.zeros(NEW, np.int64), at + 1), (np.array([0, n, 20]), np.array([10, n, 5])), (np.array([n, n, n]), np.array([n, n, n]))):
        out, lse = run_prompt(cfg, arrays, q, table, [n], [0, NEW], first, end)
        for h in range(HEADS * GROUP):
            check_rows(f64(out[:, h]), f64(lse[:, h]), f64(q[:, h]), k[h // GROUP], v[h // GROUP], 1 / math.sqrt(dim), dtype, at, first, end, 0, Scores("plain", 4), h, f"head {h}")
    q[0, 3, 0] = math.nan
    out, lse = run_prompt(cfg, arrays, q, table, [n], [0, NEW], [0, n, 20], [10, n, 5])
    assert torch.isnan(out[0, 3]).all() and torch.isnan(lse[0, 3]) and torch.isfinite(out[0, :3]).all() and (out[1:] == 0).all() and (lse[1:] == -math.inf).all()
    out, lse = run_prompt(cfg, arrays, q, table, [0], [0, NEW])
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_single_tokens_with_nan(dtype, cache):
    """moe_attn_decode and moe_attn_decode_scored over sequences that are split."""
    from test_gpu_scored import run_scored
    cfg, arrays, q, table = make(dtype, cache, 128)
    q = q[:1]
    for call in (lambda a, x: run_attention(cfg, a, x, table, [TOKENS]), lambda a, x: run_scored(cfg, a, x, table, [TOKENS], Scores("each", HEADS * GROUP))):
        want = call(arrays, q)
        bad = q.clone()
        bad[0, 2, 5] = math.nan
        got = call(arrays, bad)
        assert torch.isnan(got[0][0, 2]).all() and torch.isnan(got[1][0, 2]) and same(got, want, [0], [2])
        for tokens in (range(4608), range(4400, TOKENS)):
            got = call(plant(cfg, arrays, table, 0, 1, list(tokens), slice(None), math.nan), q)
            assert torch.isnan(got[0][0, 2:]).all() and torch.isnan(got[1][0, 2:]).all() and same(got, want, [0], slice(2, 4))
