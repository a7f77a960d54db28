"""Calls that follow each other without a host synchronisation, each reading what the one before wrote: the same
slots appended, read and attended to over and over with other data (launches overlap at their ends)."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, vectors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("lens,rows", [([300] * 16, [1] * 16), ([300] * 16, [40] * 16), ([2000, 900], [700, 900])])
def test_append_read_attend_in_turn(lens, rows, captured):
    H, D, P, Hq, turns = 4, 128, 32, 8, 24
    bt = Batch(lens, rows, P)
    n = bt.rows
    data = [(vectors((n, H, D), 3 * k, torch.float16).cuda(), vectors((n, H, D), 3 * k + 1, torch.float16).cuda(),
             vectors((n, Hq, D), 3 * k + 2, torch.float16).cuda()) for k in range(4)]
    cache = w4a8.new_kv_cache(bt.num_pages, P, H, D).fill_(0)
    ws = w4a8.new_kv_workspace(n, len(lens), Hq, H, D)

    def step(k, out=None):
        K, V, Q = data[k % 4]
        out = out or (None, None, None)
        w4a8.kv_append(K, V, cache, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
        k, v = w4a8.kv_read(cache, bt.table, bt.kv_lens, n, H, D, ws, cu_rows=bt.cu, out=out[:2] if out[0] is not None else None)
        return k, v, w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, out=out[2])

    want = []
    for k in range(4):                                     # one at a time
        got = []
        for t in step(k):
            torch.cuda.synchronize()
            got.append(t.clone())
        want.append(got)
    if captured:
        outs = [tuple(torch.empty_like(t) for t in want[0]) for _ in range(turns)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for k in range(turns):
                step(k, outs[k])
        for _ in range(3):
            graph.replay()
    else:
        outs = [step(k) for k in range(turns)]
    w4a8.check_status(ws)
    for k, got in enumerate(outs):
        for a, b in zip(got, want[k % 4]):
            assert torch.equal(a, b), k


def test_length_and_table_change_between_calls():
    """Lengths, table and queries written by kernels right in front of the call that reads them."""
    H, D, P, Hq, batch = 2, 128, 32, 8, 6
    bt = Batch([500] * batch, None, P)
    g = torch.Generator().manual_seed(0)
    cache = w4a8.new_kv_cache(bt.num_pages, P, H, D)
    whole = torch.arange(bt.num_pages, dtype=torch.int32, device="cuda").view(1, -1)
    ws = w4a8.new_kv_workspace(batch, batch, Hq, H, D)
    n = bt.num_pages * P
    w4a8.kv_append(vectors((n, H, D), 1, torch.float16).cuda(), vectors((n, H, D), 2, torch.float16).cuda(), cache, whole,
                   torch.tensor([n], dtype=torch.int32, device="cuda"), ws, cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    states = [(torch.randint(1, 501, (batch,), generator=g).int().cuda(), bt.table[torch.randperm(batch, generator=g).cuda()].contiguous(),
               vectors((batch, Hq, D), 9 + k, torch.float16).cuda()) for k in range(8)]
    want = []
    for lens, table, Q in states:
        want.append(w4a8.kv_attention(Q, cache, table, lens, H, ws))
        torch.cuda.synchronize()
    lens, table, Q = (torch.empty_like(t) for t in states[0])
    got = []
    for k in range(64):
        for to, t in zip((lens, table, Q), states[k % 8]):
            to.copy_(t)
        got.append(w4a8.kv_attention(Q, cache, table, lens, H, ws))
    w4a8.check_status(ws)
    for k, o in enumerate(got):
        assert torch.equal(o, want[k % 8]), k
