"""Elements that are NaN, and vectors with an infinity, in what is cached: the elements and vectors beside them are stored as without them."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,H,rows", [(64, 1, 5), (64, 8, 40), (128, 3, 300), (128, 8, 300)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rotary", [False, True])
def test_neighbours(D, H, rows, dtype, rotary):
    P, pages = 64, -(-rows // 64)
    g = torch.Generator().manual_seed(D + H)
    x = torch.randn(rows, H, D, generator=g).to(dtype)
    nan, inf = torch.rand(x.shape, generator=g) < 0.03, torch.rand(x.shape, generator=g) < 0.002
    inf &= torch.rand(rows, H, 1, generator=g) < 0.5
    clean = torch.where(nan, torch.zeros_like(x), x)           # (the range contains zero anyway)
    dirty = torch.where(inf, x.sign() * float("inf"), torch.where(nan, x * float("nan"), x))
    whole = ~inf.any(-1)                                       # vectors without an infinity
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, lens, cu = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1), i32([rows]), i32([0, rows])
    ws = w4a8.new_kv_workspace(rows, 1, H, H, D)
    got = []
    for v in (clean, dirty):
        cache = w4a8.new_kv_cache(pages, P, H, D).fill_(0)
        v = v.cuda()
        if rotary:                                             # (keys are turned, so the values only)
            w4a8.rope_kv_append(clean.cuda(), clean.cuda(), v, torch.arange(rows, dtype=torch.int32, device="cuda"), torch.full((8,), 0.1, device="cuda"), cache,
                                torch.arange(rows, device="cuda"), ws)
        else:
            w4a8.kv_append(v, v, cache, table, lens, ws, cu_rows=cu)
        got.append([t.cpu() for t in w4a8.kv_read(cache, table, lens, rows, H, D, ws, cu_rows=cu, dtype=dtype)])
    w4a8.check_status(ws)
    keep = (whole[..., None] & ~nan).expand(x.shape)
    for a, b in zip(*got):
        assert bool(torch.isfinite(a).all()) and torch.equal(a[keep], b[keep])
        assert bool(torch.isfinite(b[whole]).all())
    if rotary:
        assert torch.equal(got[0][0], got[1][0])
