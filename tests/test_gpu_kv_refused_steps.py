"""A step whose plan is refused, between two that are not: the sequences keep what they kept, and the step behind it is the one that would
have followed at once."""
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, filled_cache, vectors
from test_gpu_serving_chain import F16, Engine, i32
from util import guarded_workspace

pytestmark = pytest.mark.gpu


class Loop:
    """Plan, rotation with the cache write, acceptance in place of the kept lengths; captured or not."""

    def __init__(self, captured):
        self.e = e = Engine(2, 16, 2, 4, 64, 12, 10, 40)
        self.paths, self.taken = i32([[1, 4, 6], [0, 5, 0]]), i32([0, 0])
        self.graph = None
        if captured:
            self.step()                        # (no rows)
            w4a8.check_status(e.ws)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.step()

    def step(self):
        e = self.e
        e.plan()
        w4a8.rope_kv_append(e.Q, e.K, e.V, e.positions, e.freq, e.cache, e.slots, e.ws, out=e.Q)
        w4a8.kv_accept(e.cache, e.table, e.held, self.paths, self.taken, e.H, e.D, e.ws, cu_rows=e.cu, out=e.kept, kept=e.kept)

    def run(self, add, taken, seed):
        e = self.e
        for k, t in enumerate((e.Q, e.K, e.V)):
            t.copy_(vectors(t.shape, seed + k, F16))
        e.add.copy_(i32(add))
        self.taken.copy_(i32(taken))
        self.graph.replay() if self.graph else self.step()
        return w4a8.poll_status(e.ws)

    def state(self):
        e = self.e
        return [t.clone() for t in (e.held, e.kept, e.table, e.free, e.count, e.cache)]


@pytest.mark.parametrize("captured", [False, True])
def test_a_refused_step_loses_nothing(captured):
    a, b = Loop(captured), Loop(captured)
    for loop in (a, b):
        assert loop.run([20, 10], [3, 2], 1) == 0
        assert loop.e.kept.tolist() == [3, 2] and loop.e.held.tolist() == [20, 10]
    before = a.state()
    for add, taken in (([150, 10], [3, 2]), ([150, 10], [0, 0]), ([41, 0], [1, 0]), ([-1, 4], [0, 2])):       # pages, then rows, then lengths that do not fit
        assert a.run(add, taken, 50) in (9, 10)
        assert all(torch.equal(x, y) for x, y in zip(a.state(), before))
    for loop in (a, b):
        assert loop.run([8, 9], [3, 2], 100) == 0
        assert loop.e.kept.tolist() == [6, 4] and loop.e.held.tolist() == [11, 11]
        assert loop.run([7, 0], [1, 0], 200) == 0                   # one without rows
        assert loop.e.kept.tolist() == [7, 4] and loop.e.held.tolist() == [13, 4]
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))


def test_kept_lengths_of_sequences_without_rows():
    """They are taken as they are, in place too; so are those of sequences that are out of range.  Without them the lengths are the call's."""
    bt = Batch([40, 30, 17], [12, 0, 5], 16)
    cache, ws = filled_cache(bt, 2, 64), guarded_workspace(256).t
    path, kept = i32([[0, 3], [0, 0], [1, 2]]), i32([101, 102, 103])
    call = lambda lens, **kw: w4a8.kv_accept(cache.clone(), bt.table, bt.kv_lens, path, i32(lens), 2, 64, ws, cu_rows=bt.cu, **kw)  # noqa: E731
    assert call([2, 0, 2]).tolist() == [30, 30, 14]
    assert call([2, 0, 2], kept=kept).tolist() == [30, 102, 14]
    w4a8.check_status(ws)
    assert call([2, 0, -1], kept=kept).tolist() == [30, 102, 103] and w4a8.poll_status(ws) == 9
    assert call([2, 1, 2], out=kept, kept=kept).tolist() == [30, 102, 14] and w4a8.poll_status(ws) == 9
    assert kept.tolist() == [30, 102, 14]
    with pytest.raises(TypeError):
        call([2, 0, 2], kept=kept.long())
    with pytest.raises(ValueError):
        call([2, 0, 2], kept=kept[:2])


@pytest.mark.parametrize("nodes", [4, 40])
def test_calls_behind_a_refused_plan_do_nothing(nodes):
    """With its row offsets: nothing is cached, read back, attended to or moved."""
    e = Engine(2, 16, 2, 4, 64, 12, 10, 2 * nodes)
    e.add.copy_(i32([nodes, 3]))
    e.plan()
    w4a8.check_status(e.ws)
    e.cache.random_(0, 200)
    before, held = e.cache.clone(), e.held.tolist()
    e.add.copy_(i32([150, 3]))
    e.plan()
    assert w4a8.poll_status(e.ws) == 9 and e.cu.tolist() == [0, 0, 0] and e.held.tolist() == held
    K, V, Q = (vectors((e.rows, h, 64), k, F16).cuda() for k, h in enumerate((2, 2, 4)))
    outs = [torch.full_like(Q, 9.0) for _ in range(4)]
    w4a8.kv_append(K, V, e.cache, e.table, e.held, e.ws, cu_rows=e.cu)
    w4a8.rope_kv_append(Q, K, V, e.positions, e.freq, e.cache, e.slots, e.ws, out=outs[0])
    w4a8.kv_attention(Q, e.cache, e.table, e.held, 2, e.ws, cu_rows=e.cu, out=outs[1])
    w4a8.kv_attention_sinks(Q, e.cache, e.table, e.held, 2, e.ws, 9, 2, cu_rows=e.cu, out=outs[2])
    w4a8.kv_attention_tree(Q, e.cache, e.table, e.held, 2, e.ws, torch.full((e.rows, 2), -1, dtype=torch.int32, device="cuda"), cu_rows=e.cu, out=outs[3])
    w4a8.kv_accept(e.cache, e.table, e.held, i32([[1, 2], [1, 2]]), i32([0, 0]), 2, 64, e.ws, cu_rows=e.cu)
    w4a8.check_status(e.ws)
    assert torch.equal(e.cache, before) and all(bool((o == 9.0).all()) for o in outs)
