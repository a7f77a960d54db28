"""Steps that would take a number which is no page from the free list, or put one there: refused as a whole, wherever it stands; numbers
that do not change hands are not looked at."""
import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from test_gpu_kv_plan import KINDS, Case, refused, requests
from util import guarded_workspace

pytestmark = pytest.mark.gpu

NONE = [-1, -2 ** 31, 2 ** 31 - 1, None]         # None: the number of pages


def popped(c):
    """Numbers that the step takes from the list itself."""
    had = [-(-h // c.P) for h in c.held]
    has = [-(-(k + a) // c.P) for k, a in zip(c.kept, c.add)]
    return max(0, sum(max(0, n - h) for n, h in zip(has, had)) - sum(max(0, h - n) for n, h in zip(has, had)))


def surplus(c):
    """(sequence, page) of the entries that are given back."""
    return [(b, i) for b, (h, k, a) in enumerate(zip(c.held, c.kept, c.add)) for i in range(-(-(k + a) // c.P), -(-h // c.P))]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,hi,kinds", [(3, 60, ["prompt", "decode"]), (200, 90, KINDS), (1500, 120, ["prompt", "chunk", "decode", "draft"])])
def test_a_number_in_the_list(B, hi, kinds, in_place):
    c = Case(requests(B, hi, B, kinds), 16, seed=B)
    n = popped(c)
    assert n > 0
    for at, value in zip((0, n // 2, n - 1), NONE):
        was = c.free.copy()
        c.free[c.count - 1 - at] = c.pages if value is None else value
        refused(c, c.run(in_place=in_place), 9)
        c.free = was
    c.free[:c.count - n] = -1                      # below those that are taken
    c.check(c.run(in_place=in_place))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,hi,kinds", [(1, 400, ["ended"]), (40, 300, ["ended", "prompt"]), (700, 200, KINDS), (1500, 90, ["ended", "draft", "again"])])
def test_a_number_that_would_be_given_back(B, hi, kinds, in_place):
    c = Case(requests(B, hi, B, kinds), 16, seed=B)
    back = surplus(c)
    for at, value in zip((0, len(back) // 3, len(back) // 2, len(back) - 1), NONE):
        was = c.table.copy()
        c.table[back[at]] = c.pages if value is None else value
        refused(c, c.run(in_place=in_place), 9)
        c.table = was
    c.check(c.run(in_place=in_place))


def test_more_given_back_than_threads_look_at_once():
    c = Case([(9000, 0, 0), (40, 40, 7000), (12000, 11, 3)], 16, seed=1)
    back = surplus(c)
    for at in (0, 511, 512, len(back) - 1):
        was = c.table.copy()
        c.table[back[at]] = -1
        refused(c, c.run(), 9)
        c.table = was
    c.check(c.run())


def test_pages_taken_away_in_front_of_a_window():
    """Entries between the sinks and the window that name no page any more: a sequence goes on without them, and drafts are taken back;
    it ends with held 0, when the caller has given back the others."""
    c = Case([(300, 300, 30), (200, 190, 1), (64, 64, 1)], 16, seed=2)
    c.table[0, 1:10] = -1
    c.table[1, 1:5] = -1
    want = c.check(c.run())
    assert (want["table"][0, 1:10] == -1).all()
    ended = Case([(300, 0, 0), (200, 200, 1)], 16, seed=3)
    ended.table[0, 1:10] = -1
    refused(ended, ended.run(), 9)
    ended.held[0] = 0
    got = ended.check(ended.run())
    assert got["lens"].tolist() == [0, 201]


def test_the_step_behind_a_refused_one():
    """The same buffers: refused, mended, done."""
    c = Case(requests(300, 90, 4, KINDS), 32, seed=4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    held, count, ws = i32(c.held), i32([c.count]), guarded_workspace(512)
    table, free = torch.from_numpy(c.table).cuda(), torch.from_numpy(c.free).cuda()
    good = int(free[c.count - 1])
    free[c.count - 1] = c.pages
    for turn in range(3):
        out = w4a8.kv_plan(held, i32(c.kept), i32(c.add), table, free, count, c.P, c.rows, ws.t, out=(held, None, None, None, count))
        assert w4a8.poll_status(ws.t) == 9 and held.tolist() == c.held and count.tolist() == [c.count]
    free[c.count - 1] = good
    out = w4a8.kv_plan(held, i32(c.kept), i32(c.add), table, free, count, c.P, c.rows, ws.t, out=(held, None, None, None, count))
    c.status = w4a8.poll_status(ws.t)
    c.check({k: v.cpu().numpy() for k, v in dict(table=table, free=free, lens=out[0], cu=out[1], positions=out[2], slots=out[3], count=out[4]).items()})
    assert np.array_equal(ws.t[256:].cpu().numpy(), np.zeros(256, np.uint8))
