"""Attention with a window and sinks, and of drafted trees, against binary64 attention over the values that the rows see."""
import math
import random

import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, check_attention, filled_cache
from serving_util import attention_where, mask_words, seen_in_tree, seen_with_sinks, tree_masks
from util import Guarded

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def drop_unseen_pages(bt, seen):
    """Entries of pages that no row sees name no page."""
    row = 0
    for b, (n, c) in enumerate(zip(bt.lens, bt.counts)):
        pages = {j // bt.P for r in range(row, row + c) for j in seen[r]}
        for i in range(-(-n // bt.P)):
            if i not in pages:
                bt.table_host[b, i] = -7
        row += c
    bt.table = torch.from_numpy(bt.table_host).cuda()


def run(call, seen, bt, Hq, H, D, q_type=F16, o_type=F16, seed=0, q_scale=1.0, scale=None, drop=True):
    """call(Q, cache, ws, out, lse, scale); seen: positions per row."""
    cache = filled_cache(bt, H, D, seed=seed + 5)
    if drop:
        drop_unseen_pages(bt, seen)
    Q = (q_scale * torch.randn(bt.rows, Hq, D, generator=torch.Generator().manual_seed(seed + 9))).to(q_type).cuda()
    ws = Guarded((w4a8.kv_attention_workspace_bytes(bt.rows, len(bt.lens), Hq, H, D),), torch.uint8)
    w4a8.workspace_init(ws.t)
    out, lse = Guarded((bt.rows, Hq, D), o_type), Guarded((bt.rows, Hq), torch.float32)
    out.t.fill_(7.0)
    lse.t.fill_(7.0)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    call(Q, cache, ws.t, out.t, lse.t, scale)
    w4a8.check_status(ws.t)
    O = out.t.clone()
    for g, what in ((out, "O"), (lse, "lse"), (ws, "workspace")):
        g.check(what)
    o, want_lse, allow = attention_where(Q, cache, bt, H, scale, seen + [[]] * (bt.rows - bt.used))
    n = bt.used
    check_attention(O[:n], o[:n], allow[:n], o_type)
    got_lse = lse.t[:n].cpu().double()
    finite = torch.isfinite(want_lse[:n])
    assert torch.equal(finite, torch.isfinite(got_lse))
    qsum = Q[:n].cpu().double().abs().sum(-1)
    off = (D / 16 + 4) * 2.0 ** -23 * 30 * qsum * 2.0 * scale + 2.0 ** -19 * (1 + want_lse[:n].abs())
    assert bool(((got_lse - want_lse[:n]).abs()[finite] <= off[finite]).all())
    assert bool((O[n:] == 7.0).all()) and bool((lse.t[n:] == 7.0).all())      # padding rows
    call(Q, cache, ws.t, out.t, lse.t, scale)
    assert torch.equal(out.t, O)                                               # the same bits again
    return O


def sinks(lens, rows, P, Hq, H, D, window, few, causal=True, pad=0, **kw):
    bt = Batch(lens, rows, P, pad)
    seen = [s for n, c in zip(bt.lens, bt.counts) for s in (seen_with_sinks(n, c, i, causal, window, few) for i in range(c))]
    return run(lambda Q, cache, ws, out, lse, scale: w4a8.kv_attention_sinks(Q, cache, bt.table, bt.kv_lens, H, ws, window, few, cu_rows=bt.cu, scale=scale,
                                                                             causal=causal, out=out, lse=lse), seen, bt, Hq, H, D, **kw)


def tree(lens, rows, P, Hq, H, D, masks, window=0, few=0, words=None, pad=0, **kw):
    bt = Batch(lens, rows, P, pad)
    words = words or max(1, -(-max(rows) // 32))
    seen = [seen_in_tree(n, c, i, masks[bt.start[b] + i], window, few) for b, (n, c) in enumerate(zip(bt.lens, bt.counts)) for i in range(c)]
    bits = mask_words(list(masks) + [(1 << 32 * words) - 1] * pad, words).cuda()
    kw.setdefault("drop", all(n >= c for n, c in zip(lens, rows)))
    return run(lambda Q, cache, ws, out, lse, scale: w4a8.kv_attention_tree(Q, cache, bt.table, bt.kv_lens, H, ws, bits, cu_rows=bt.cu, scale=scale,
                                                                            window=window, sinks=few, out=out, lse=lse), seen, bt, Hq, H, D, **kw)


def random_tree(n, seed):
    rng = random.Random(seed)
    return tree_masks([-1 if j == 0 else rng.randint(max(-1, j - 6), j - 1) for j in range(n)])


LENS = [1, 0, 15, 33, 64, 65, 200, 331]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [1, 16, 31, 64, 100])
@pytest.mark.parametrize("few", [1, 4, 16, 33, 70])
def test_single_rows(D, window, few):
    sinks(LENS, None, 16, 4, 2, D, window, few)


@pytest.mark.parametrize("Hq,H", [(1, 1), (5, 1), (8, 2), (16, 1), (12, 3)])
@pytest.mark.parametrize("P", [16, 64, 1024])
def test_head_layouts_and_pages(Hq, H, P):
    sinks([700, 3, 129], None, P, Hq, H, 128, 100, 4, q_type=BF16, o_type=BF16)


@pytest.mark.parametrize("rows", [[2, 1, 0, 5], [17, 3, 1, 33], [64, 64, 64, 64], [130, 0, 40, 100]])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,few", [(21, 4), (64, 40), (1, 130), (500, 3), (0, 5)])
def test_several_rows(rows, causal, window, few):
    sinks([230, 3, 140, 164], rows, 32, 6, 2, 64, window, few, causal=causal, pad=2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,few", [(128, 4), (300, 64), (300, 65), (64, 1), (190, 200)])
def test_chunks_of_a_prompt(D, window, few):
    sinks([700, 513], [300, 129], 64, 4, 1, D, window, few)


def test_sinks_equal_plain_attention_without_a_window():
    bt = Batch([300, 70], [40, 3], 32)
    cache = filled_cache(bt, 2, 64)
    Q = torch.randn(bt.rows, 8, 64, dtype=F16, device="cuda")
    ws = w4a8.new_kv_workspace(bt.rows, 2, 8, 2, 64)
    want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, 2, ws, cu_rows=bt.cu)
    assert torch.equal(want, w4a8.kv_attention_sinks(Q, cache, bt.table, bt.kv_lens, 2, ws, 0, 4, cu_rows=bt.cu))
    want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, 2, ws, cu_rows=bt.cu, window=33)
    assert torch.equal(want, w4a8.kv_attention_sinks(Q, cache, bt.table, bt.kv_lens, 2, ws, 33, 0, cu_rows=bt.cu))


def test_long_sequences_are_shared_by_many_workgroups():
    sinks([9000, 20000], None, 64, 8, 1, 128, 7001, 37)
    sinks([5000], [90], 128, 4, 2, 128, 3001, 5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(4, 4), (8, 2), (16, 1)])
@pytest.mark.parametrize("n", [1, 5, 16, 40])
def test_trees(D, Hq, H, n):
    lens, rows = [n, n + 1, n + 31, n + 200], [n, n, max(1, n // 2), n]
    masks = [m for k, c in enumerate(rows) for m in random_tree(c, 7 * n + k)]
    tree(lens, rows, 16, Hq, H, D, masks, q_type=BF16)


@pytest.mark.parametrize("base", [0, 1, 31, 32, 33, 63, 64, 200])
@pytest.mark.parametrize("n", [70, 129])
def test_wide_trees(base, n):
    masks = random_tree(n, base) + random_tree(33, base + 1)
    tree([base + n, base + 33], [n, 33], 32, 4, 1, 128, masks, pad=3)


@pytest.mark.parametrize("rows", [[3, 2], [40, 70]])
def test_any_mask(rows):
    """Rows that see nothing drafted, bits of rows behind the last, rows that see later ones, more words than needed, no tokens in front."""
    rng = random.Random(3)
    n = sum(rows)
    masks = [rng.choice([0, (1 << 128) - 1, rng.getrandbits(128), 1 << 127, 1 << r % rows[0]]) for r in range(n)]
    tree([rows[0], rows[1] + 45], rows, 16, 8, 2, 64, masks, words=4, drop=False)
    tree([rows[0] + 100, rows[1]], rows, 16, 2, 2, 128, [0] * n, words=4, drop=False)


def test_rows_in_front_of_the_sequence():
    masks = random_tree(6, 1) + random_tree(50, 2)
    tree([4, 30], [6, 50], 16, 4, 2, 64, masks)


@pytest.mark.parametrize("rows", [[4, 9, 1], [60, 33, 70]])
@pytest.mark.parametrize("window,few", [(1, 0), (20, 0), (20, 4), (64, 33), (400, 7)])
def test_trees_with_a_window(rows, window, few):
    masks = [m for k, c in enumerate(rows) for m in random_tree(c, 11 * k)]
    tree([300, 45, 130], rows, 16, 4, 2, 128, masks, window=window, few=few)
    masks[1] = 0
    tree([300, 45, 130], rows, 16, 4, 2, 64, masks, window=window, few=few, drop=False)


@pytest.mark.parametrize("window,few", [(0, 0), (33, 4)])
def test_a_chain_sees_what_causal_rows_see(window, few):
    """(Within a window, a drafted row sees all of its own path: the chain is shorter than the window.)  The two calls share their work
    differently, so each is held to binary64."""
    for c in (5, 33, 64):
        if window and c > window:
            continue
        masks = [(2 << i) - 1 for i in range(c)] * 2
        for n in (200, c):
            for i in range(c):
                assert seen_in_tree(n, c, i, masks[i], window, few) == seen_with_sinks(n, c, i, True, window, few)
        tree([200, c], [c, c], 16, 8, 2, 128, masks, window=window, few=few)


def test_too_many_rows_for_the_mask_are_reported():
    for c in (40, 100):
        bt = Batch([c + 9], [c], 16)
        cache = filled_cache(bt, 1, 64)
        Q = torch.randn(c, 2, 64, dtype=F16, device="cuda")
        ws = w4a8.new_kv_workspace(c, 1, 2, 1, 64)
        bits = torch.full((c, 1), -1, dtype=torch.int32, device="cuda")
        w4a8.kv_attention_tree(Q, cache, bt.table, bt.kv_lens, 1, ws, bits, cu_rows=bt.cu)
        assert w4a8.poll_status(ws) == 9


@pytest.mark.parametrize("rows", [1, 70])
def test_pages_between_sinks_and_window_may_hold_anything(rows):
    """Their words are infinities and NaN patterns; so are those of the slots behind the end."""
    n, window, few, P, H, D = 300, 90, 5, 16, 2, 128
    bt = Batch([n], [rows], P)
    cache = filled_cache(bt, H, D)
    Q = torch.randn(rows, 4, D, dtype=F16, device="cuda")
    ws = w4a8.new_kv_workspace(rows, 1, 4, H, D)
    want = w4a8.kv_attention_sinks(Q, cache, bt.table, bt.kv_lens, H, ws, window, few, cu_rows=bt.cu)
    blocks = cache.view(bt.num_pages, H, 16 * (D + 8))
    words = blocks[..., 16 * D:].contiguous().view(torch.int32)
    first = max(0, n - rows + 1 - window)
    for i in range(-(-n // P)):
        gone = [s for s in range(P) if few <= i * P + s < first or i * P + s >= n]
        page = int(bt.table_host[0, i])
        for s in gone:
            words[page, :, s], words[page, :, 16 + s] = 0x7f80000f, -1
    blocks[..., 16 * D:] = words.view(torch.uint8).view(bt.num_pages, H, 128)
    got = w4a8.kv_attention_sinks(Q, cache, bt.table, bt.kv_lens, H, ws, window, few, cu_rows=bt.cu)
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [None, [40, 33]])
def test_queries_that_are_slices_and_one_row_per_sequence(rows):
    """Q as a slice of a wider projection output; without cu_rows a tree has one node per sequence, its mask any."""
    bt = Batch([300, 170], rows, 16)
    cache = filled_cache(bt, 2, 64)
    wide = torch.randn(bt.rows, 12, 64, dtype=BF16, device="cuda")
    Q, ws = wide[:, 2:10], w4a8.new_kv_workspace(bt.rows, 2, 8, 2, 64)
    bits = mask_words([1, 0] if rows is None else [m for c in rows for m in random_tree(c, c)], 2).cuda()
    for call in (lambda q: w4a8.kv_attention_sinks(q, cache, bt.table, bt.kv_lens, 2, ws, 70, 5, cu_rows=bt.cu),
                 lambda q: w4a8.kv_attention_tree(q, cache, bt.table, bt.kv_lens, 2, ws, bits, cu_rows=bt.cu)):
        assert torch.equal(call(Q), call(Q.contiguous()))
    if rows is None:
        seen = [seen_in_tree(n, 1, 0, m, 0, 0) for n, m in zip(bt.lens, (1, 0))]
        o, _, allow = attention_where(Q.contiguous(), cache, bt, 2, 0.125, seen)
        check_attention(w4a8.kv_attention_tree(Q, cache, bt.table, bt.kv_lens, 2, ws, bits), o, allow, F16)
    w4a8.check_status(ws)


def test_large_scores_and_far_tokens():
    """Weights that differ by thousands of powers of two: a sink far above the window's tokens, and far below them."""
    for few in (1, 4):
        for rows in (None, [70, 70]):
            sinks([400, 90 if rows else 33], rows, 16, 4, 2, 64, 50, few, q_scale=60.0, scale=4.0)


def test_items_alike_go_one_to_a_workgroup():
    """Row tiles of one length, as many as workgroups and a little fewer, a few more (the many-row form); single rows likewise."""
    for heads in (37, 36, 38):                 # 4 tiles of 64 tokens each
        sinks([600], [256], 64, 4 * heads, heads, 64, 100, 4)
    sinks([400] * 24, None, 16, 16, 16, 64, 100, 4)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pages", [0, 900])
def test_the_width_of_the_page_table(D, pages):
    """Pages that no sequence reaches yet: the tiles of rows may differ, the result does not."""
    def widen(bt):
        more = torch.full((len(bt.lens), pages), -7, dtype=torch.int32, device="cuda")
        return torch.cat([bt.table, more], 1)

    lens, rows, P, Hq, H = [130, 5, 77, 300], [5, 3, 0, 7], 16, 16, 4
    bt = Batch(lens, rows, P, 0)
    seen = [seen_with_sinks(n, c, i, True, 40, 3) for n, c in zip(lens, rows) for i in range(c)]
    run(lambda Q, cache, ws, out, lse, scale: w4a8.kv_attention_sinks(Q, cache, widen(bt), bt.kv_lens, H, ws, 40, 3, cu_rows=bt.cu, scale=scale, out=out, lse=lse),
        seen, bt, Hq, H, D)
    bt = Batch(lens, rows, P, 0)
    seen = [seen_with_sinks(n, c, i, True, 5000, 3) for n, c in zip(lens, rows) for i in range(c)]
    run(lambda Q, cache, ws, out, lse, scale: w4a8.kv_attention_sinks(Q, cache, widen(bt), bt.kv_lens, H, ws, 5000, 3, cu_rows=bt.cu, scale=scale, out=out, lse=lse),
        seen, bt, Hq, H, D)
    bt = Batch(lens, rows, P, 0)
    masks = [m for b, n in enumerate(rows) for m in random_tree(n, b)]
    seen = [seen_in_tree(n, c, i, masks[bt.start[b] + i], 0, 0) for b, (n, c) in enumerate(zip(lens, rows)) for i in range(c)]
    bits = mask_words(masks, 1).cuda()
    run(lambda Q, cache, ws, out, lse, scale: w4a8.kv_attention_tree(Q, cache, widen(bt), bt.kv_lens, H, ws, bits, cu_rows=bt.cu, scale=scale, out=out, lse=lse),
        seen, bt, Hq, H, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,few", [(1, 1), (20, 4), (33, 20), (64, 0)])
def test_a_few_rows_of_many_sequences(D, window, few):
    lens, rows = [90, 17, 64, 33, 5, 70, 32, 81, 48, 16, 0, 77], [7, 8, 5, 6, 5, 8, 3, 7, 8, 4, 0, 1]
    sinks(lens, rows, 16, 24, 12, D, window, few)
    masks = [m for b, n in enumerate(rows) for m in random_tree(n, b)]
    tree(lens, rows, 16, 24, 12, D, masks, window, few)
