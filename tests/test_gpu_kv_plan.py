"""A step's plan on the device against one that is made page by page."""
import random

import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from serving_util import plan_reference
from util import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu


def requests(B, hi, seed, kinds):
    rng = random.Random(seed)
    got = []
    for _ in range(B):
        n, kind = rng.randint(1, hi), rng.choice(kinds)
        kept = max(0, n - rng.randint(0, 20))
        got.append({"decode": (n, n, 1), "prompt": (0, 0, n), "chunk": (n, n, rng.randint(0, hi)), "draft": (n, kept, rng.randint(0, 9)),
                    "ended": (n, 0, 0), "idle": (n, n, 0), "empty": (0, 0, 0), "again": (n, 0, rng.randint(1, hi))}[kind])
    return got


class Case:
    def __init__(self, req, P, spare_pages=3, spare_rows=5, seed=0, short=0):
        rng = np.random.default_rng(seed)
        self.P = P
        self.held, self.kept, self.add = (list(x) for x in zip(*req))
        had = [-(-h // P) for h in self.held]
        has = [-(-(k + a) // P) for k, a in zip(self.kept, self.add)]
        need = sum(max(0, n - h) for n, h in zip(has, had)) - sum(max(0, h - n) for n, h in zip(has, had))
        self.most = max(1, max(had + has)) + 1
        self.pages = max(1, sum(had) + max(0, need) + spare_pages)
        perm = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(req), self.most), -5, np.int32)
        at = 0
        for b, k in enumerate(had):
            self.table[b, :k] = perm[at:at + k]
            at += k
        self.free = np.full(self.pages, -9, np.int32)
        self.free[:self.pages - at] = perm[at:]
        self.count = self.pages - at - short
        self.rows = max(1, sum(self.add) + spare_rows)

    def run(self, held=True, in_place=False, rows=None, out=True):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        rows = rows or self.rows
        B = len(self.held)
        self.g = {k: Guarded(s, t) for k, s, t in (("table", self.table.shape, torch.int32), ("free", (self.pages,), torch.int32), ("lens", (B,), torch.int32),
                                                   ("cu", (B + 1,), torch.int32), ("positions", (rows,), torch.int32), ("slots", (rows,), torch.int64),
                                                   ("count", (1,), torch.int32))}
        t = {k: g.t for k, g in self.g.items()}
        t["table"].copy_(torch.from_numpy(self.table))
        t["free"].copy_(torch.from_numpy(self.free))
        self.ws = guarded_workspace(512)
        h, k, a, c = i32(self.held), i32(self.kept), i32(self.add), i32([self.count])
        if in_place:
            t["lens"], t["count"] = (h if held else k), c
        w4a8.kv_plan(h if held else None, k, a, t["table"], t["free"], c, self.P, rows, self.ws.t,
                     out=(t["lens"], t["cu"], t["positions"], t["slots"], t["count"]))
        self.status = w4a8.poll_status(self.ws.t)
        for name, g in self.g.items():
            g.check(name)
        self.ws.check("workspace")
        assert bool((self.ws.t[256:] == 0).all())
        return {k: v.cpu().numpy() for k, v in t.items()}

    def check(self, got, rows=None):
        want = plan_reference(self.held, self.kept, self.add, self.table, self.free, self.count, self.P, rows or self.rows)
        assert self.status == 0
        for k, v in want.items():
            assert np.array_equal(got[k], v), k
        return want


KINDS = ["decode", "prompt", "chunk", "draft", "ended", "idle", "empty", "again"]


@pytest.mark.parametrize("B", [1, 2, 31, 33, 511, 513, 1500])
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("in_place", [False, True])
def test_mixed_requests(B, P, in_place):
    c = Case(requests(B, 90, B, KINDS), P, seed=B)
    c.check(c.run(in_place=in_place))


@pytest.mark.parametrize("kinds", [["decode"], ["prompt"], ["ended"], ["idle", "empty"], ["ended", "prompt"], ["again"]])
def test_one_kind(kinds):
    for seed in range(3):
        c = Case(requests(40, 300, seed, kinds), 32, spare_pages=seed, spare_rows=seed, seed=seed)
        c.check(c.run(in_place=seed == 1))


def test_without_held_lengths():
    c = Case(requests(70, 200, 5, ["decode", "prompt", "chunk", "idle"]), 16)
    for in_place in (False, True):
        c.check(c.run(held=False, in_place=in_place))


@pytest.mark.parametrize("P", [16, 256, 1024])
def test_many_rows(P):
    c = Case(requests(37, 9000, 3, ["prompt", "draft", "ended"]), P, spare_rows=3001)
    c.check(c.run())


def test_the_largest_batch():
    c = Case(requests(8192, 3, 3, KINDS), 16)
    c.check(c.run(in_place=True))


def test_pages_given_back_are_taken_at_once():
    """No page is free: the new sequence lives on what the ended one gives back."""
    c = Case([(100, 0, 0), (0, 0, 100), (64, 10, 0), (0, 0, 33)], 16, spare_pages=0)
    assert c.count <= 0 + c.pages - 11
    c.check(c.run())


def refused(c, got, status):
    assert c.status == status
    B = len(c.held)
    assert not got["cu"].any() and (got["slots"] == -1).all() and not got["positions"].any()
    assert np.array_equal(got["lens"], c.held[:B]) and got["count"] == [c.count]
    assert np.array_equal(got["table"], c.table) and np.array_equal(got["free"], c.free)


@pytest.mark.parametrize("in_place", [False, True])
def test_too_few_pages(in_place):
    c = Case([(10, 10, 40), (30, 30, 1), (0, 0, 90)], 16, spare_pages=0, short=1)
    refused(c, c.run(in_place=in_place), 10)


def test_what_does_not_fit_is_refused_as_a_whole():
    base = [(10, 10, 40), (30, 30, 1), (70, 20, 9)]
    c = Case(base, 16)
    refused(c, c.run(rows=49), 9)
    c.check(c.run(rows=50), 50)
    for k, bad in ((0, (-1, -1, 4)), (1, (5, 6, 1)), (2, (7, 7, -1)), (1, (5, 5, 10 ** 6)), (0, (10 ** 6, 3, 1)), (2, (5, 5, 2 ** 31 - 1))):
        c = Case(base, 16)
        c.held[k], c.kept[k], c.add[k] = bad
        refused(c, c.run(rows=100), 9)
    for count in (-1, 10 ** 6):
        c = Case(base, 16)
        c.count = count
        refused(c, c.run(), 9)
    c = Case([(70, 0, 0)], 16)
    c.count = c.pages                      # more given back than the list has room for
    refused(c, c.run(), 9)


def test_a_bad_page_in_the_list_is_reported():
    c = Case([(0, 0, 40)], 16)
    c.free[:] = c.pages + 7
    got = c.run()
    assert c.status == 9 and (got["slots"] == -1).all()


def test_refusals_in_python():
    c = Case(requests(3, 20, 1, ["decode"]), 16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = guarded_workspace(512).t
    held, kept, add, table, free, count = i32(c.held), i32(c.kept), i32(c.add), torch.from_numpy(c.table).cuda(), torch.from_numpy(c.free).cuda(), i32([c.count])
    out = w4a8.kv_plan(held, kept, add, table, free, count, 16, 5, ws)
    assert [t.shape for t in out] == [(3,), (4,), (5,), (5,), (1,)] and out[3].dtype == torch.int64
    for bad in (lambda: w4a8.kv_plan(held, kept.long(), add, table, free, count, 16, 5, ws), lambda: w4a8.kv_plan(held, kept, add, table.cpu(), free, count, 16, 5, ws),
                lambda: w4a8.kv_plan(held, kept, add, table[:, ::2], free, count, 16, 5, ws), lambda: w4a8.kv_plan(held, kept, None, table, free, count, 16, 5, ws)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: w4a8.kv_plan(held, kept[:2], add, table, free, count, 16, 5, ws), lambda: w4a8.kv_plan(held, kept, add, table, free, kept, 16, 5, ws),
                lambda: w4a8.kv_plan(held, kept, add, table, free, count, 16, -5, ws)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(w4a8.W4A8Error):
        w4a8.kv_plan(held, kept, add, table, free, count, 17, 5, ws)
    with pytest.raises(w4a8.W4A8Error):
        w4a8.kv_plan(held, kept, add, table, free, count, 16, 5, ws, out=(kept, None, None, None, None))


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_outputs_off_the_16_byte_grid(shift):
    """Positions and slots that begin anywhere: the wide stores are left out."""
    c = Case(requests(20, 90, shift, KINDS), 16, spare_rows=3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = guarded_workspace(512)
    pos, slots = torch.full((c.rows + 8,), 77, dtype=torch.int32, device="cuda"), torch.full((c.rows + 8,), 77, dtype=torch.int64, device="cuda")
    table, free = torch.from_numpy(c.table).cuda(), torch.from_numpy(c.free).cuda()
    out = w4a8.kv_plan(i32(c.held), i32(c.kept), i32(c.add), table, free, i32([c.count]), 16, c.rows, ws.t,
                       out=(None, None, pos[shift:shift + c.rows], slots[shift:shift + c.rows], None))
    c.status = w4a8.poll_status(ws.t)
    c.check(dict(table=table.cpu().numpy(), free=free.cpu().numpy(), lens=out[0].cpu().numpy(), cu=out[1].cpu().numpy(),
                 positions=out[2].cpu().numpy(), slots=out[3].cpu().numpy(), count=out[4].cpu().numpy()))
    for t in (pos, slots):
        assert (t[:shift] == 77).all() and (t[shift + c.rows:] == 77).all()
