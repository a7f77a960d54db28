"""What accept leaves out and what it moves beside it: every byte of the cache and the lengths, for paths and lengths that are wrong."""
import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, filled_cache
from test_gpu_kv_accept import bytes_of
from util import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def kept_places(path, n):
    """(i, place) of a path that the contract moves: places among the n rows, above the one in front of them, not below their index."""
    return [(i, j) for i, j in enumerate(path) if i <= j < n and (i == 0 or j > path[i - 1])]


def accepted_image(raw, bt, paths, D):
    """raw [pages, H, P / 16, block] behind the call; the sources are taken from what was there before."""
    old, P = raw.copy(), bt.P
    for b, (n, c, path) in enumerate(zip(bt.lens, bt.counts, paths)):
        for i, j in kept_places(path, c):
            to, at = n - c + i, n - c + j
            pt, pa = bt.table_host[b, to // P], bt.table_host[b, at // P]
            raw[pt, :, to % P // 16][:, bytes_of(to % 16, D)] = old[pa, :, at % P // 16][:, bytes_of(at % 16, D)]
    return raw


def run(bt, paths, H, D, want_status, want_lens, lens=None, kv=None, cu=None, moved=None):
    """moved: the paths that count, [] for a sequence that keeps its slots.  want_lens: None where a length is not looked at."""
    P, most = bt.P, max(len(p) for p in paths)
    cache = Guarded((bt.num_pages, w4a8.kv_page_bytes(P, H, D)), torch.uint8)
    cache.t.copy_(filled_cache(bt, H, D))
    shape = (bt.num_pages, H, P // 16, 16 * (D + 8))
    want = accepted_image(cache.t.view(shape).cpu().numpy().copy(), bt, paths if moved is None else moved, D)
    ws, out = guarded_workspace(256), Guarded((len(paths),), torch.int32)
    w4a8.kv_accept(cache.t, bt.table, i32(bt.lens if kv is None else kv), i32([p + [0] * (most - len(p)) for p in paths]),
                   i32([len(p) for p in paths] if lens is None else lens), H, D, ws.t, cu_rows=i32(bt.start.tolist() if cu is None else cu), out=out.t)
    assert w4a8.poll_status(ws.t) == want_status
    for g in (cache, out, ws):
        g.check()
    assert all(got == n for got, n in zip(out.t.tolist(), want_lens) if n is not None)
    assert np.array_equal(cache.t.view(shape).cpu().numpy(), want)


GOOD = [0, 3, 4, 7]
BAD_PATHS = [[-1], [-2, -1], [0, -5, -3], [-3, -2, -1, 0, 1], [-2 ** 31, -2 ** 30, 5], [-100000, -90000, 2], [4, 0, 1, 2], [5, 2, 3, 4], [3, 2, 5], [0, 0, 1], [2, 4, 12],
             [2 ** 31 - 1, 2 ** 31 - 1, 4], [11, 12, 13], [1, 1, 1, 1, 1, 6, 5, 7], list(range(11, -1, -1)), [8] + list(range(11))]


@pytest.mark.parametrize("D,H,P", [(64, 2, 16), (128, 11, 64)])
def test_places_that_are_left_out(D, H, P):
    """Beside a healthy sequence in front and behind; rows that begin at position 0 and further on."""
    for base in (0, 3, 28):
        for path in BAD_PATHS:
            bt = Batch([40, base + 12, 17], [12, 12, 8], P)
            run(bt, [GOOD, path, GOOD], H, D, 9, [28 + 4, base + len(path), 9 + 4])


def test_more_places_than_are_looked_up_at_a_time():
    path = list(range(100, 240)) + [100, 101, -7, -6] + list(range(240, 300))
    for base in (0, 50):
        run(Batch([base + 300], [300], 16), [path], 1, 64, 9, [base + len(path)])


@pytest.mark.parametrize("change,after", [(dict(lens=[4, 9]), 18), (dict(lens=[4, -1]), 18), (dict(lens=[4, 13]), 18), (dict(kv=[40, -3]), None),
                                          (dict(kv=[40, 10 ** 6]), None), (dict(kv=[40, 5]), None), (dict(cu=[0, 12, 5]), None), (dict(cu=[0, 12, 10 ** 9]), None)])
def test_sequences_that_keep_their_slots(change, after):
    """Lengths or offsets out of range, more accepted rows than there are: the other sequence is served."""
    run(Batch([40, 30], [12, 12], 16), [GOOD, [0, 2, 5]], 2, 64, 9, [32, after], moved=[GOOD, []], **change)
