"""Value vectors with the smallest steps that the cache keeps, tens of thousands of them in a sequence: the softmax's
denominator, which carries 1 / step, stays inside binary32."""
import math

import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, attention_reference, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows", [(1200, 1), (300, 66)])
@pytest.mark.parametrize("low", [-100, 80])
def test_denominator_of_many_small_steps(batch, rows, low):
    """Every sequence has the same pages: 256 tokens, then n - 256 that score ten and a half bits higher.  The values
    are 13 steps of 2^low up or down, so output and denominator are those of the two groups."""
    H, D, P, n = 1, 64, 1024, 65536
    one = Batch([n], [1], P)
    K = torch.zeros(n, 1, D)
    K[256:, 0, 0] = 13 / 8
    V = torch.full((n, 1, D), 13.0)
    V[::2] = -13.0
    V[256:512] = 13.0
    V = V * 2.0 ** low
    cache = w4a8.new_kv_cache(one.num_pages, P, H, D).fill_(0)
    ws = w4a8.new_kv_workspace(batch * rows, batch, 1, H, D)
    w4a8.kv_append(K.bfloat16().cuda(), V.bfloat16().cuda(), cache, one.table, one.kv_lens, ws,
                   cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    q = torch.zeros(1, 1, D)
    q[..., 0] = 10.5 * math.log(2.0) * 8 / 13
    q = q.half()
    o, want_lse, allow = attention_reference(q, cache, one, H, 1.0, causal=False)
    Q = q.expand(batch * rows, 1, D).contiguous().cuda()
    lse = torch.empty(batch * rows, 1, device="cuda")
    cu = torch.arange(0, batch * rows + 1, rows, dtype=torch.int32, device="cuda")
    O = w4a8.kv_attention(Q, cache, one.table.expand(batch, -1).contiguous(), one.kv_lens.expand(batch).contiguous(), H, ws,
                          cu_rows=cu, scale=1.0, causal=False, dtype=torch.bfloat16, lse=lse)
    w4a8.check_status(ws)
    check_attention(O, o.expand_as(O), allow.expand_as(O), torch.bfloat16)
    assert bool(((lse.cpu().double() - want_lse).abs() <= 2.0 ** -12).all())
