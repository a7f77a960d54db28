"""Scores far below zero, within binary32: a row that sees keys is never taken for one that sees none."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, decode_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 96])
@pytest.mark.parametrize("scale", [1e26, 3e32])
def test_scores_far_below_zero(rows, scale):
    """All scores are below -1e30 and none is within a tenth of the largest: the output is that token's value."""
    H, D, P, n, best = 1, 64, 64, 300, 37
    bt = Batch([n], [rows], P)
    K = torch.zeros(n, 1, D)
    K[:, 0, 0] = 104.0
    K[best, 0, 0] = 13.0
    V = torch.randn(n, 1, D, generator=torch.Generator().manual_seed(0))
    cache = w4a8.new_kv_cache(bt.num_pages, P, H, D).fill_(0)
    ws = w4a8.new_kv_workspace(rows, 1, 1, H, D)
    w4a8.kv_append(K.half().cuda(), V.half().cuda(), cache, bt.table, bt.kv_lens, ws,
                   cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    Q = torch.zeros(rows, 1, D)
    Q[:, 0, 0] = -1024.0
    lse = torch.empty(rows, 1, device="cuda")
    O = w4a8.kv_attention(Q.half().cuda(), cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, scale=scale, causal=False, lse=lse)
    w4a8.check_status(ws)
    _, value, _, _ = decode_pages(cache, H, D, P)
    want = value[int(bt.table_host[0, best // P]), 0, best % P]
    # the value at weight 1: the offsets' binary32 sums and the output's rounding
    assert bool(((O.cpu().double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -14).all())
    top = -1024.0 * 13.0 * scale
    assert bool(((lse.cpu().double() - top).abs() <= 2.0 ** -18 * abs(top)).all())
