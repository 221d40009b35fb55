"""moe_attn_prompt on the GPU against the fp64 oracle on the same stored inputs; the tolerance is derived in prompt_cases.py."""
import math

import numpy as np
import pytest
import torch

import paper_2106_10715_amd as M
from oracle import decoder_oracle as D
from prompt_cases import MASKS, Scores, check_rows, run_and_check, run_prompt, spans
from test_gpu_decoder import TYPES, cache_of, f64, normal, run_attention, tables

pytestmark = pytest.mark.gpu

KINDS = ["plain", "cap", "slopes", "table", "each"]
# (past, new): edges of runs of 16, of tiles of 32 to 256 rows and 64 keys; nothing new, nothing at all
NEWS = [(0, 1), (0, 2), (0, 0), (15, 1), (0, 16), (0, 17), (3, 30), (50, 0), (0, 33), (64, 63), (0, 65), (100, 31), (0, 129), (70, 130), (0, 260)]


def make(news, heads, dim, page, dtype, cache, seed=20):
    per = max(1, max(-(-(p + n) // page) for p, n in news))
    cfg = M.KvCfg.make(len(news) * per + 3, page, heads, dim, dtype, cache)
    table = tables(seed, len(news), per, cfg.pages)
    arrays = cache_of(seed, cfg, table, [p + n for p, n in news])              # NaN wherever no token lies
    for b, (p, n) in enumerate(news):                                          # pages past a sequence's end: not even numbers of pages
        table[b, -(-(p + n) // page):] = 2 ** 31 - 1
    return cfg, arrays, table.cuda()


def queries(seed, n, heads, dim, dtype, std=2.0):
    """Stretches of wider rows."""
    return normal(seed, (n, heads * dim + 24), dtype, std)[:, 8:8 + heads * dim].view(n, heads, dim)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,window,kind,score", [
    (4, 1, 64, 16, 0, "causal", "plain"), (2, 3, 128, 32, 0, "prefix", "table"), (1, 8, 16, 64, 0, "documents", "slopes"), (3, 5, 80, 16, 100, "causal", "each"),
    (2, 16, 48, 512, 1, "all", "plain"), (1, 17, 128, 16, 33, "both", "cap"), (2, 2, 256, 16, 0, "odd", "plain"), (1, 40, 144, 128, 130, "causal", "slopes"),
    (1, 4, 160, 16, 0, "prefix", "each"), (5, 1, 96, 32, 0, "odd", "cap"), (2, 1, 224, 64, 7, "documents", "table")])
def test_prompts_at_the_edges_of_tiles_pages_and_masks(heads, group, dim, page, window, kind, score, dtype, cache):
    cfg, arrays, table = make(NEWS, heads, dim, page, dtype, cache)
    q = queries(22, sum(n for _, n in NEWS), heads * group, dim, dtype)
    run_and_check(cfg, arrays, q, table, NEWS, kind, window, scores=Scores(score, heads * group))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", KINDS)
@pytest.mark.parametrize("kind", MASKS)
def test_every_mask_with_every_score(kind, score, dtype):
    news = [(0, 150), (37, 41), (0, 3)]
    cfg, arrays, table = make(news, 2, 64, 16, dtype, dtype)
    q = queries(23, sum(n for _, n in news), 4, 64, dtype)
    for window in (0, 25):
        run_and_check(cfg, arrays, q, table, news, kind, window, scores=Scores(score, 4))


@pytest.mark.parametrize("back,ahead", [(0, 0), (1, 0), (0, 1), (127, 127), (5, 300), (1000, 3), (65535, 65535)])
def test_biases_of_all_widths(back, ahead):
    news = [(300, 200), (0, 77)]
    cfg, arrays, table = make(news, 1, 64, 32, "bf16", "bf16")
    q = queries(24, 277, 3, 64, "bf16")
    for kind in ("prefix", "causal", "all"):
        run_and_check(cfg, arrays, q, table, news, kind, scores=Scores("table", 3, back=back, ahead=ahead))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("B,past,new,heads,group,dim,page", [
    (1, 9000, 1, 1, 8, 128, 64), (1, 5000, 17, 2, 4, 64, 16), (3, 3001, 5, 1, 71, 80, 32), (2, 4000, 33, 4, 1, 256, 128), (1, 20000, 3, 1, 1, 64, 256), (5, 1200, 40, 2, 2, 112, 16)])
def test_a_few_tokens_after_long_sequences(B, past, new, heads, group, dim, page, dtype, cache):
    news = [(past - 37 * b, new - b % 2) for b in range(B)]
    cfg, arrays, table = make(news, heads, dim, page, dtype, cache, seed=26)
    q = queries(25, sum(n for _, n in news), heads * group, dim, dtype)
    few = sorted({0, heads * group // 2, heads * group - 1})
    a = run_and_check(cfg, arrays, q, table, news, scores=Scores("slopes", heads * group), heads_only=few)
    b = run_and_check(cfg, arrays, q, table, news, scores=Scores("slopes", heads * group), heads_only=[0])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), "two runs differ"
    run_and_check(cfg, arrays, q, table, news, "prefix", window=1000, scores=Scores("each", heads * group), heads_only=few)


@pytest.mark.parametrize("dtype,cache,dim", [("bf16", "bf16", 128), ("bf16", "e4m3", 64), ("bf16", "bf16", 256), ("f32", "f32", 64), ("f32", "e4m3", 128)])
def test_long_prompts(dtype, cache, dim):
    news = [(0, 2100), (0, 0), (500, 700), (0, 1301)]
    cfg, arrays, table = make(news, 2, dim, 64, dtype, cache, seed=28)
    q = queries(27, sum(n for _, n in news), 8, dim, dtype)
    a = run_and_check(cfg, arrays, q, table, news, heads_only=[0, 5])
    b = run_and_check(cfg, arrays, q, table, news, heads_only=[7])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), "two runs differ"
    run_and_check(cfg, arrays, q, table, news, "both", heads_only=[2], scores=Scores("cap", 8))
    run_and_check(cfg, arrays, q, table, news, "prefix", heads_only=[3], scores=Scores("table", 8, back=127, ahead=127))


@pytest.mark.parametrize("kind,window", [("causal", 0), ("prefix", 0), ("documents", 0), ("odd", 0), ("causal", 300)])
@pytest.mark.parametrize("dim,cache", [(128, "bf16"), (112, "e4m3")])
def test_prompts_long_enough_for_blocks_in_turns(dim, cache, kind, window):
    """Rows enough for blocks of eight waves, of which one half weighs while the other multiplies; all that a mask hides stays without effect."""
    news = [(100, 2100)]
    cfg, arrays, table = make(news, 16, dim, 64, "bf16", cache, seed=48)
    q = queries(49, 2100, 64, dim, "bf16")
    a = run_and_check(cfg, arrays, q, table, news, kind, window, heads_only=[0, 37, 63])
    b = run_and_check(cfg, arrays, q, table, news, kind, window, heads_only=[5])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), "two runs differ"
    bad = [None if t is None else t.clone() for t in arrays]
    first, end, given = spans(kind, news)
    at, token = np.arange(100, 2200), 1500
    lo = np.maximum(np.maximum(first, 0), at - window + 1) if window else np.maximum(first, 0)
    sees = torch.from_numpy((lo <= token) & (token < end)).cuda()
    place = (table[0, token // 64].long(), 9, token % 64, 5)
    bad[1].view(torch.uint8).view(*bad[1].shape, -1)[place] = 0x7f if cache == "e4m3" else torch.tensor([0x80, 0x7f], dtype=torch.uint8, device="cuda")
    got, got_lse = run_prompt(cfg, bad, q, table, [2200], [0, 2100], first if given[0] else None, end if given[1] else None, window)
    assert torch.equal(got_lse, a[1]) and torch.equal(got[~sees], a[0][~sees]) and not torch.isfinite(got[sees][:, 36:40, 5].float()).any()
    got[:, 36:40, 5] = a[0][:, 36:40, 5]
    assert torch.equal(got, a[0])


@pytest.mark.parametrize("kind,window", [("causal", 0), ("both", 0), ("causal", 1700)])
@pytest.mark.parametrize("dim,cache", [(128, "e4m3"), (80, "bf16")])
def test_prompts_after_long_ones_in_turns(dim, cache, kind, window):
    """Rows of several sequences, one without new tokens, after thousands of cached ones, in blocks of eight waves."""
    news = [(5000, 1200), (4100, 0), (4097, 700), (7001, 333)]
    cfg, arrays, table = make(news, 16, dim, 64, "bf16", cache, seed=58)
    q = queries(59, 2233, 64, dim, "bf16")
    a = run_and_check(cfg, arrays, q, table, news, kind, window, heads_only=[1, 62])
    b = run_and_check(cfg, arrays, q, table, news, kind, window, heads_only=[30])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), "two runs differ"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    """4096 of them, 0 to 5 new tokens each; and one among many that is longer than all others together."""
    for news, heads in (([((b * 31) % 40, b % 6) for b in range(4096)], 1), ([(0, 1 if b != 200 else 900) for b in range(300)], 2)):
        page = 16
        cfg = M.KvCfg.make(sum(-(-(p + n) // page) for p, n in news) + 1, page, heads, 64, dtype)
        per = max(-(-(p + n) // page) for p, n in news)
        table, at = torch.zeros((len(news), per), dtype=torch.int32), 0
        for b, (p, n) in enumerate(news):
            used = -(-(p + n) // page)
            table[b, :used] = torch.arange(at, at + used)
            at += used
        arrays = cache_of(30, cfg, table, [p + n for p, n in news])
        q = queries(29, sum(n for _, n in news), 2 * heads, 64, dtype)
        run_and_check(cfg, arrays, q, table.cuda(), news, only=[0, 1, 2, 3, 199, 200, 201, len(news) - 1])


def test_rows_of_no_sequence_are_left_as_they_were():
    """Rows before the first sequence and behind the last; starts outside of the rows are taken as within them."""
    news = [(5, 20), (0, 0), (0, 37)]
    for dtype in ("bf16", "f32"):
        cfg, arrays, table = make(news, 2, 64, 16, dtype, dtype)
        q = queries(31, 100, 4, 64, dtype)
        lens, starts = [25, 0, 37], [11, 31, 31, 68]
        out, lse = run_prompt(cfg, arrays, q, table, lens, starts)
        assert (out[:11] == 7).all() and (out[68:] == 7).all() and (lse[:11] == 7).all() and (lse[68:] == 7).all()
        want, want_lse = run_and_check(cfg, arrays, q[11:68], table, news)
        assert torch.equal(out[11:68], want) and torch.equal(lse[11:68], want_lse)
        # the last sequence's end past the rows: its new tokens are those up to the last row
        out2, _ = run_prompt(cfg, arrays, q[:68], table, lens, [11, 31, 31, 10 ** 9])
        assert torch.equal(out2[11:], want)
        out3, _ = run_prompt(cfg, arrays, q, table, lens, starts, want_lse=False)
        assert torch.equal(out3[11:68], want)


def test_lengths_and_pages_outside_of_their_ranges():
    """A length past the table is the table's, one below zero none; more new tokens than the sequence has: the first of them see nothing."""
    cfg, arrays, table = make([(0, 48), (0, 48)], 1, 64, 16, "bf16", "bf16")
    q = queries(32, 40, 2, 64, "bf16")
    want, want_lse = run_prompt(cfg, arrays, q, table, [48, 0], [0, 20, 40])
    got, got_lse = run_prompt(cfg, arrays, q, table, [10 ** 9, -7], [0, 20, 40])
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)
    assert (got[20:] == 0).all() and (got_lse[20:] == -math.inf).all()
    got, got_lse = run_prompt(cfg, arrays, q, table, [5, 48], [0, 20, 40])
    assert (got[:15] == 0).all() and (got_lse[:15] == -math.inf).all()
    assert torch.isfinite(got.float()).all() and torch.isfinite(got_lse[15:]).all()
    every = dict(end=np.full(40, 48))                                          # a window of all there is hides nothing, of tokens before the first either
    a, b = (run_prompt(cfg, arrays, q, table, [5, 48], [0, 20, 40], window=w, **every) for w in (0, 2 ** 31 - 1))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.isfinite(a[1]).all()
    table[0, 1] = cfg.pages + 5                                                # the nearest page that exists
    far = torch.clone(table)
    far[0, 1] = cfg.pages - 1
    a, b = run_prompt(cfg, arrays, q, table, [16, 48], [0, 20, 40]), run_prompt(cfg, arrays, q, far, [16, 48], [0, 20, 40])
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("dim,n", [(64, 40), (64, 300), (128, 200), (256, 150)])
def test_what_a_mask_hides_has_no_effect_and_what_it_shows_has_its_own(dim, n, dtype, cache):
    """NaN and infinities in keys and values that some rows of a tile see and others do not: the others keep every bit."""
    news = [(0, n)]
    cfg, arrays, table = make(news, 2, dim, 16, dtype, cache, seed=33)
    q = queries(34, n, 4, dim, dtype)
    tab = table.cpu()
    plant = [(0, 7, 3, math.nan), (1, 20, dim - 1, math.nan), (1, 30, 0, math.inf), (1, 33, 1, -math.inf), (1, n - 2, 5, math.inf), (0, n - 1, 2, math.nan)]
    if cache == "e4m3":
        plant = [p for p in plant if math.isnan(p[3])]
    for kind, window in (("causal", 0), ("causal", 10), ("documents", 0)):
        first, end, given = spans(kind, news)
        args = (table, [n], [0, n], first if given[0] else None, None, window)
        want, want_lse = run_prompt(cfg, arrays, q, *args)
        for side, token, column, value in plant:
            bad = [None if t is None else t.clone() for t in arrays]
            place = (tab[0, token // 16].long(), 1, token % 16, column)
            if cache == "e4m3":
                bad[side].view(torch.uint8)[place] = 0x7f
            else:
                bad[side][place] = value
            got, got_lse = run_prompt(cfg, bad, q, *args)
            at = np.arange(n)
            lo = np.maximum(first, at - window + 1) if window else first
            sees = torch.from_numpy((lo <= token) & (token < end)).cuda()
            what = f"{kind}, window {window}, {'KV'[side]}[{token}, {column}] = {value}"
            assert torch.equal(got[:, :2], want[:, :2]) and torch.equal(got_lse[:, :2], want_lse[:, :2]), what + ": the other key head"
            assert torch.equal(got[~sees, 2:], want[~sees, 2:]) and torch.equal(got_lse[~sees, 2:], want_lse[~sees, 2:]), what + ": rows that do not see it"
            if side == 0:
                assert torch.isnan(got[sees, 2:]).all(), what
            else:
                col = got[sees, 2:, column].float()
                assert torch.isnan(col).all() if math.isnan(value) else (col == value).all(), what
                keep = [c for c in range(dim) if c != column]
                assert torch.equal(got[sees, 2:][..., keep], want[sees, 2:][..., keep]) and torch.equal(got_lse, want_lse), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_that_are_not_finite_where_no_row_looks(dtype):
    """An 8-bit cache's scales of hidden tokens: NaN; of one that some rows see: theirs alone."""
    n = 90
    cfg, arrays, table = make([(0, n)], 1, 64, 16, dtype, "e4m3", seed=35)
    q = queries(36, n, 2, 64, dtype)
    want, _ = run_prompt(cfg, arrays, q, table, [n], [0, n])
    for side in (2, 3):
        bad = [t.clone() for t in arrays]
        bad[side][table[0, 50 // 16].long(), 0, 50 % 16] = math.nan
        got, _ = run_prompt(cfg, bad, q, table, [n], [0, n])
        assert torch.equal(got[:50], want[:50]) and torch.isnan(got[50:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_minus_infinity_and_growing_ones(dtype):
    """Keys whose logit is -infinity weigh nothing, rows that see no other are as rows without keys; a maximum that rises with every key, and one that never does."""
    n, dim = 200, 64
    cfg, arrays, table = make([(0, n)], 1, dim, 16, dtype, dtype, seed=37)
    q = queries(38, n, 2, dim, dtype).abs() + 2 ** -10
    at = torch.arange(n)
    tab = table.cpu()
    arrays[0][tab[0][at // 16].long(), 0, at % 16, 0] = torch.where(at < 60, -math.inf, 0.0).to(arrays[0].dtype).cuda()
    out, lse = run_prompt(cfg, arrays, q, table, [n], [0, n])
    assert (out[:60] == 0).all() and (lse[:60] == -math.inf).all()
    k, v = (D.paged_rows(f64(t), None, tab[0].numpy(), 60, n)[0] for t in arrays[:2])
    for h in range(2):
        check_rows(f64(out[60:, h]), f64(lse[60:, h]), f64(q[60:, h]), k, v, 1 / math.sqrt(dim), dtype, at[60:] - 60, 0 * at[60:], at[60:] - 59, 0,
                   Scores("plain", 2), h, f"head {h}")
    for slope in (0.5, -0.5, 40.0, -40.0):
        cfg, arrays, table = make([(0, n)], 1, dim, 16, dtype, dtype, seed=39)
        arrays[0][table.cpu()[0][at // 16].long(), 0, at % 16, 0] = (slope * at.float()).to(arrays[0].dtype).cuda()
        q = torch.zeros((n, 2, dim), dtype=arrays[0].dtype, device="cuda")
        q[:, :, 0] = 8.0
        run_and_check(cfg, arrays, q, table, [(0, n)])
        run_and_check(cfg, arrays, q, table, [(0, n)], "all", scores=Scores("cap", 2, cap=50.0))


def test_one_new_token_is_the_single_token_call():
    """Both calls on the same cache: within twice a rounding of each other."""
    lens = [1, 17, 64, 300, 1000]
    news = [(n - 1, 1) for n in lens]
    for dtype, cache, tol in (("bf16", "bf16", 2 ** -6), ("bf16", "e4m3", 2 ** -6), ("f32", "f32", 2 ** -17)):
        cfg, arrays, table = make(news, 2, 128, 16, dtype, cache, seed=41)
        q = queries(42, len(lens), 8, 128, dtype)
        out, lse = run_prompt(cfg, arrays, q, table, lens, range(6))
        want, want_lse = run_attention(cfg, arrays, q, table, lens)
        assert (out.float() - want.float()).abs().max() <= tol and (lse - want_lse).abs().max() <= 2 ** -16


def test_offsets_past_32_bits():
    """Rows of q far apart, and pages at the far end of a pool of over 2^32 bytes a side."""
    pages, page, heads, dim, n = 33100, 64, 8, 128, 150
    cfg = M.KvCfg.make(pages, page, heads, dim)
    arrays = cfg.empty()
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32)
    at = torch.arange(n)
    slots = (table[0][at // page] * page + at % page).int().cuda()
    k, v = normal(43, (n, heads, dim), "bf16"), normal(44, (n, heads, dim), "bf16")
    M.moe_kv_write(cfg, k, v, slots, *arrays)
    wide = torch.empty((n, 1 << 24), dtype=torch.bfloat16, device="cuda")
    assert wide.numel() > 2 ** 31
    q = wide[:, -2 * heads * dim:].view(n, 2 * heads, dim)
    q.copy_(normal(45, (n, 2 * heads, dim), "bf16", 2.0))
    far, _ = run_prompt(cfg, arrays, q, table.cuda(), [n], [0, n])
    small = M.KvCfg.make(3, page, heads, dim)
    near = small.empty()
    M.moe_kv_write(small, k, v, at.int().cuda(), *near)
    want, _ = run_prompt(small, near, q.contiguous(), torch.arange(3, dtype=torch.int32, device="cuda")[None], [n], [0, n])
    assert torch.equal(far, want)


def test_empty_calls():
    cfg = M.KvCfg.make(2, 16, 1, 64)
    arrays = cfg.empty()
    none, ints = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    for tokens, B in ((0, 2), (0, 0), (3, 0)):
        prompt = M.PromptCfg.make(tokens, B, 2, 2)
        ws = torch.empty(M.moe_attn_prompt_workspace_bytes(cfg, prompt), dtype=torch.uint8, device="cuda")
        q = torch.zeros((tokens, 2, 64), dtype=torch.bfloat16, device="cuda")
        out = torch.full_like(q, 7)
        M.moe_attn_prompt(cfg, prompt, None, q, *arrays, ints[:2 * B].view(B, 2), ints[:B], ints[:B + 1], None, None, None, None, out, None, ws)
        torch.cuda.synchronize()
        assert (out == 7).all()
    prompt = M.PromptCfg.make(2, 3, 2, 2)                                      # sequences without new tokens
    ws = torch.empty(M.moe_attn_prompt_workspace_bytes(cfg, prompt), dtype=torch.uint8, device="cuda")
    out = torch.full((2, 2, 64), 7, dtype=torch.bfloat16, device="cuda")
    M.moe_attn_prompt(cfg, prompt, None, torch.zeros_like(out), *arrays, ints[:6].view(3, 2), ints[:3], ints[:4], None, None, None, None, out, None, ws)
    torch.cuda.synchronize()
    assert (out == 7).all() and none.numel() == 0


@pytest.mark.parametrize("past", [0, 6000])
def test_on_another_stream_and_in_graphs_that_share_a_workspace(past):
    """Two captured calls over one workspace, replayed in turn and on new inputs, against eager calls on another stream."""
    news = [(past, 40), (past // 2, 9), (0, 100)]
    heads, group, dim = 2, 4, 64
    cfg, arrays, table = make(news, heads, dim, 64, "bf16", "e4m3", seed=46)
    n = sum(m for _, m in news)
    prompt = M.PromptCfg.make(n, 3, heads * group, table.shape[1])
    ws = torch.empty(M.moe_attn_prompt_workspace_bytes(cfg, prompt), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([p + m for p, m in news], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 40, 49, 149], dtype=torch.int32, device="cuda")
    scores = [Scores("plain", 8), Scores("each", 8)]
    q = [queries(47 + i, n, 8, dim, "bf16").contiguous() for i in range(2)]
    out = [torch.empty_like(t) for t in q]

    def call(i, stream=None):
        M.moe_attn_prompt(cfg, prompt, scores[i].cfg, q[i], *arrays, table, lens, starts, None, None, scores[i].slopes, scores[i].bias, out[i], None, ws,
                          stream=stream)

    for i in range(2):
        call(i)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    side = torch.cuda.Stream()
    for step in range(4):
        for i in range(2):
            q[i].copy_(queries(50 + 2 * step + i, n, 8, dim, "bf16"))
        graphs[step % 2].replay()
        graphs[1 - step % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for i in range(2):
            out[i].fill_(3)
        torch.cuda.synchronize()
        for i in range(2):
            call(i, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
