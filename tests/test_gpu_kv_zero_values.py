"""Tokens whose value vector is zero but whose score is high (a sink): the others keep their precision."""
import math

import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, attention_reference, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 96])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits,size", [(10, 2.0 ** -10), (20, 2.0 ** -14), (6, 100.0), (-12, 1.0)])
def test_a_sink_of_zero_value(rows, D, bits, size):
    """One token scores `bits` bits above (below) the others and has the value zero; the others' values are of size `size`."""
    H, P, n = 1, 64, 2000
    g = torch.Generator().manual_seed(1)
    bt = Batch([n], [rows], P)
    K = torch.zeros(n, 1, D)
    K[:, 0, 1] = 0.5 * torch.randn(n, generator=g)
    K[7, 0] = 0
    K[7, 0, 0] = 1.0
    V = size * (torch.randn(n, 1, D, generator=g) + 0.5)
    V[7] = 0
    cache = w4a8.new_kv_cache(bt.num_pages, P, H, D).fill_(0)
    ws = w4a8.new_kv_workspace(rows, 1, 1, H, D)
    w4a8.kv_append(K.bfloat16().cuda(), V.bfloat16().cuda(), cache, bt.table, bt.kv_lens, ws,
                   cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    k, v = w4a8.kv_read(cache, bt.table, bt.kv_lens, n, H, D, ws, cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    assert bool((v[7] == 0).all()) and bool(v[8].any())
    Q = torch.zeros(rows, 1, D)
    Q[:, 0, 0] = bits * math.log(2.0)
    Q[:, 0, 1] = 1.0
    Q = Q.bfloat16().cuda()
    lse = torch.empty(rows, 1, device="cuda")
    O = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, scale=1.0, dtype=torch.bfloat16, lse=lse)
    w4a8.check_status(ws)
    # what a zero vector may add to the error is nothing: its step does not count in the allowance
    plain = cache.clone()
    page, slot = int(bt.table_host[0, 0]), 7
    plain[page, 16 * D + 64:16 * D + 128].view(torch.int32)[slot] = 0
    o, want_lse, allow = attention_reference(Q, plain, bt, H, 1.0)
    check_attention(O, o, allow, torch.bfloat16)
    assert bool(((lse.cpu().double() - want_lse).abs() <= 2.0 ** -12).all())
