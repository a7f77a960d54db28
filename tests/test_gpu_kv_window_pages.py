"""Attention with a window over a cache whose pages behind the window were given back: table entries in front of
the oldest visible token name no page, and nothing reads them."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, attention_reference, check_attention, filled_cache, vectors

pytestmark = pytest.mark.gpu


def released(bt, window):
    """The page table without the pages that lie wholly in front of every row's window."""
    table = bt.table_host.copy()
    for b, (n, c) in enumerate(zip(bt.lens, bt.counts)):
        oldest = max(0, n - c + 1 - window)
        table[b, :oldest // bt.P] = -7
    return torch.from_numpy(table).cuda()


# first visible tokens of the oldest rows: 20, 50 and 116 (32- and 64-token groups begin at 0, 32, 64, 96), 1, 0
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_entries_in_front_of_the_window_are_not_read(P, D, rows):
    window, H, Hq = 100, 2, 8
    lens = [first + window - 1 + rows for first in (20, 50, 116, 1)] + [rows + 7]
    bt = Batch(lens, None if rows == 1 else [rows] * len(lens), P)
    cache = filled_cache(bt, H, D)
    Q = vectors((bt.rows, Hq, D), 3, torch.float16).cuda()
    ws = w4a8.new_kv_workspace(bt.rows, len(lens), Hq, H, D)
    whole = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, window=window)
    w4a8.check_status(ws)
    table = released(bt, window)
    assert int((table != bt.table).sum()) >= (3 if P == 16 else 2 if P == 32 else 1)
    got = w4a8.kv_attention(Q, cache, table, bt.kv_lens, H, ws, cu_rows=bt.cu, window=window)
    w4a8.check_status(ws)
    o, _, allow = attention_reference(Q, cache, bt, H, D ** -0.5, True, window)
    check_attention(got, o, allow, torch.float16)
    assert torch.equal(got, whole)
