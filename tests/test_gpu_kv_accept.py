"""Accepted paths: the cache's bytes against moves made one by one on the host."""
import random

import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, filled_cache
from util import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu


def bytes_of(s, D):
    """A slot's bytes in its block."""
    c = D // 16
    return ([s * (D // 2) + i for i in range(D // 2)] + [8 * D + ((s // 8 * 8 + g) * 8 + s % 8) * c + i for g in range(8) for i in range(c)]
            + [16 * D + w + 4 * s + i for w in (0, 64) for i in range(4)])


def moved(raw, bt, paths, D):
    """raw [pages, H, P / 16, block] with the moves done, in any order: from a copy of what was there."""
    old, P = raw.copy(), bt.P
    for b, (n, c, path) in enumerate(zip(bt.lens, bt.counts, paths)):
        for i, j in enumerate(path):
            to, at = n - c + i, n - c + j
            pt, pa = bt.table_host[b, to // P], bt.table_host[b, at // P]
            raw[pt, :, to % P // 16][:, bytes_of(to % 16, D)] = old[pa, :, at % P // 16][:, bytes_of(at % 16, D)]
    return raw


def run(hist, rows, paths, P, H, D, most=None, cu=True):
    bt = Batch([h + r for h, r in zip(hist, rows)], rows if cu else None, P)
    cache = Guarded((bt.num_pages, w4a8.kv_page_bytes(P, H, D)), torch.uint8)
    cache.t.copy_(filled_cache(bt, H, D))
    want = moved(cache.t.view(bt.num_pages, H, P // 16, 16 * (D + 8)).cpu().numpy().copy(), bt, paths, D)
    most = most or max(1, max(len(p) for p in paths))
    accepted = torch.full((len(rows), most), 10 ** 9, dtype=torch.int32)     # behind the path: anything
    for b, p in enumerate(paths):
        accepted[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    lens = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    ws, out = guarded_workspace(256), Guarded((len(rows),), torch.int32)
    got = w4a8.kv_accept(cache.t, bt.table, bt.kv_lens, accepted.cuda(), lens, H, D, ws.t, cu_rows=bt.cu, out=out.t)
    w4a8.check_status(ws.t)
    for g, what in ((cache, "cache"), (out, "lens"), (ws, "workspace")):
        g.check(what)
    assert got.tolist() == [h + len(p) for h, p in zip(hist, paths)]
    assert np.array_equal(cache.t.view(want.shape).cpu().numpy(), want)


def random_paths(rows, seed):
    rng = random.Random(seed)
    return [sorted(rng.sample(range(r), rng.randint(0, r))) for r in rows]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H", [1, 3, 8, 32])
@pytest.mark.parametrize("P", [16, 64])
def test_random_paths(D, H, P):
    rows = [1, 7, 16, 40, 3, 0, 64]
    run([0, 5, 15, 100, 16, 9, 31], rows, random_paths(rows, D + H), P, H, D)


def test_paths_that_overlap_themselves():
    """Every copy's destination is an earlier copy's source."""
    run([13], [40], [list(range(1, 40))], 16, 2, 128)
    run([13, 0], [40, 20], [list(range(20, 40)), list(range(20))], 32, 2, 64)
    run([3], [400], [list(range(0, 400, 2))], 16, 1, 64)      # more than are looked up at a time
    run([3], [400], [list(range(1, 400))], 16, 5, 128)


def test_nothing_or_all_accepted():
    run([5, 20], [6, 6], [[], [0, 1, 2, 3, 4, 5]], 16, 2, 64)
    run([5, 20], [1, 1], [[0], []], 16, 2, 64, most=3, cu=False)


def test_what_is_wrong_is_reported_and_moves_nothing():
    H, D, P = 2, 64, 16
    for change in (dict(lens=[4, 9]), dict(lens=[4, -1]), dict(path=[3, 2, 5]), dict(path=[0, 0, 1]), dict(path=[2, 4, 12]), dict(path=[-1, 1, 2]),
                   dict(kv=[200, 5]), dict(kv=[40, -3]), dict(kv=[40, 10 ** 6]), dict(cu=[0, 12, 5]), dict(cu=[0, 12, 10 ** 9])):
        bt = Batch([40, 30], [12, 12], P)
        cache = Guarded((bt.num_pages, w4a8.kv_page_bytes(P, H, D)), torch.uint8)
        cache.t.copy_(filled_cache(bt, H, D))
        ws = guarded_workspace(256)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        w4a8.kv_accept(cache.t, bt.table, i32(change.get("kv", [40, 30])), i32([[0, 1, 2, 3]] + [change.get("path", [0, 1, 2]) + [3]]), i32(change.get("lens", [3, 3])), H, D, ws.t,
                       cu_rows=i32(change.get("cu", [0, 12, 24])))
        assert w4a8.poll_status(ws.t) == 9, change
        cache.check("cache")
    bt = Batch([40], [12], P)                # a page outside the cache
    cache = filled_cache(bt, H, D)
    before = cache.clone()
    bad = bt.table.clone()
    bad[:] = bt.num_pages
    ws = guarded_workspace(256)
    w4a8.kv_accept(cache, bad, bt.kv_lens, i32([[3, 5]]), i32([2]), H, D, ws.t, cu_rows=bt.cu)
    assert w4a8.poll_status(ws.t) == 9 and torch.equal(cache, before)


def test_refusals_in_python():
    bt = Batch([40], [12], 16)
    cache, ws = filled_cache(bt, 2, 64), guarded_workspace(256).t
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    path, n = i32([[3, 5]]), i32([2])
    with pytest.raises(w4a8.W4A8Error):
        w4a8.kv_accept(cache, bt.table, bt.kv_lens, path, n, 2, 64, ws, cu_rows=bt.cu, out=bt.kv_lens)
    for bad in (lambda: w4a8.kv_accept(cache, bt.table, bt.kv_lens, path.long(), n, 2, 64, ws, cu_rows=bt.cu),
                lambda: w4a8.kv_accept(cache, bt.table, bt.kv_lens, path, n.cpu(), 2, 64, ws, cu_rows=bt.cu)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: w4a8.kv_accept(cache, bt.table, bt.kv_lens, path[0], n, 2, 64, ws, cu_rows=bt.cu),
                lambda: w4a8.kv_accept(cache, bt.table, bt.kv_lens, path, i32([2, 2]), 2, 64, ws, cu_rows=bt.cu),
                lambda: w4a8.kv_accept(cache, bt.table, bt.kv_lens, path, n, 3, 64, ws, cu_rows=bt.cu)):
        with pytest.raises(ValueError):
            bad()
