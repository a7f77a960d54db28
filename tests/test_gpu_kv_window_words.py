"""Slots in front of the window that were never written: whatever their words are, no row that does not see them
changes."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, filled_cache, vectors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_words_in_front_of_the_window_are_not_seen(rows, D):
    window, H, Hq, P = 100, 2, 8, 64
    first = (20, 50, 127)                                  # the oldest visible token of each sequence
    lens = [f + window - 1 + rows for f in first]
    bt = Batch(lens, None if rows == 1 else [rows] * 3, P)
    cache = filled_cache(bt, H, D)
    Q = vectors((bt.rows, Hq, D), 3, torch.float16).cuda()
    ws = w4a8.new_kv_workspace(bt.rows, 3, Hq, H, D)
    lse = torch.empty(bt.rows, Hq, device="cuda")
    want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, window=window, lse=lse)
    want_lse = lse.clone()
    raw = cache.view(bt.num_pages, H, P // 16, 16 * (D + 8))
    hidden = torch.zeros(bt.num_pages, P, dtype=torch.bool)
    for b, f in enumerate(first):
        for j in range(f):
            hidden[bt.table_host[b, j // P], j % P] = True
    words = raw[..., 16 * D:].contiguous().view(torch.int32).view(bt.num_pages, H, P // 16, 2, 16)
    where = hidden.view(bt.num_pages, 1, P // 16, 1, 16).cuda().expand_as(words)
    for bits in (0, 0x00000010, 0x7F800000, 0x7FFFFFFF, -1, -2 ** 31):       # zero, subnormal, infinity, NaN, negative
        words[where] = bits
        raw[..., 16 * D:] = words.view(torch.uint8).reshape(bt.num_pages, H, P // 16, 128)
        got = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, window=window, lse=lse)
        w4a8.check_status(ws)
        assert torch.equal(got, want) and torch.equal(lse, want_lse), hex(bits)
