"""The serving calls one after the other, as an engine uses them: captured once and replayed with other lengths, trees and paths, on side
streams, in caches beyond 32-bit offsets."""
import ctypes
import random

import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, check_attention, decode_pages, filled_cache, quantize_vectors, vectors
from serving_util import attention_where, mask_words, plan_reference, rotate_reference, seen_in_tree, seen_with_sinks, tree_masks
from util import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu

F16 = torch.float16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def frequencies(D):
    return torch.from_numpy((10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)).cuda()


class Engine:
    """Device state of a small engine: page table, free list, lengths; a step's buffers."""

    def __init__(self, B, P, H, Hq, D, max_pages, num_pages, rows, seed=0):
        self.B, self.P, self.H, self.Hq, self.D, self.rows = B, P, H, Hq, D, rows
        self.table = torch.full((B, max_pages), -3, dtype=torch.int32, device="cuda")
        self.free = torch.from_numpy(np.random.default_rng(seed).permutation(num_pages).astype(np.int32)).cuda()
        self.count = i32([num_pages])
        self.held, self.kept, self.add = i32([0] * B), i32([0] * B), i32([0] * B)
        self.cu, self.positions, self.slots = i32([0] * (B + 1)), i32([0] * rows), torch.zeros(rows, dtype=torch.int64, device="cuda")
        self.cache = w4a8.new_kv_cache(num_pages, P, H, D).fill_(0)
        self.ws = w4a8.new_kv_workspace(rows, B, Hq, H, D)
        self.freq = frequencies(D)
        self.Q, self.K, self.V = (torch.zeros(rows, h, D, dtype=F16, device="cuda") for h in (Hq, H, H))

    def plan(self):
        """In place: `held` becomes the lengths with this step's rows."""
        w4a8.kv_plan(self.held, self.kept, self.add, self.table, self.free, self.count, self.P, self.rows, self.ws,
                     out=(self.held, self.cu, self.positions, self.slots, self.count))

    def host_batch(self, lens, counts):
        bt = Batch.__new__(Batch)
        bt.lens, bt.counts, bt.P, bt.rows, bt.used = lens, counts, self.P, self.rows, sum(counts)
        bt.table_host = self.table.cpu().numpy()
        bt.num_pages = self.cache.shape[0]
        return bt

    def cached(self, b, pos):
        """Values of the keys and values at positions of a sequence, binary64 [len(pos), H, D] each."""
        K, V, _, _ = decode_pages(self.cache, self.H, self.D, self.P)
        table = self.table.cpu()
        pages = torch.tensor([int(table[b, p // self.P]) for p in pos])
        places = torch.tensor([p % self.P for p in pos])
        return K[pages, :, places], V[pages, :, places]


def as_quantized(x):
    lev, step, _ = quantize_vectors(x)
    return torch.from_numpy(lev * step.astype(np.float64))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("Hq,H,D,nodes", [(4, 2, 64, 6), (8, 1, 128, 20)])
def test_drafted_steps(Hq, H, D, nodes, captured):
    """Plan, rotation and cache write, attention of the trees, acceptance of a path; the next step's plan takes back what was not
    accepted.  Sequences grow at different speeds, one ends and another begins in its place."""
    B, P, most = 3, 16, 5
    e = Engine(B, P, H, Hq, D, 20, 40, B * nodes + 4)
    paths, taken = i32([[0] * most] * B), i32([0] * B)
    lens_after = i32([0] * B)
    words = -(-nodes // 32)
    masks, where = torch.zeros(e.rows, words, dtype=torch.int32, device="cuda"), i32([0] * e.rows)
    O = torch.zeros(e.rows, Hq, D, dtype=F16, device="cuda")

    def step():
        e.plan()
        w4a8.rope_kv_append(e.Q, e.K, e.V, where, e.freq, e.cache, e.slots, e.ws, out=e.Q)
        w4a8.kv_attention_tree(e.Q, e.cache, e.table, e.held, H, e.ws, masks, cu_rows=e.cu, out=O)
        w4a8.kv_accept(e.cache, e.table, e.held, paths, taken, H, D, e.ws, cu_rows=e.cu, out=lens_after)

    graph = None
    if captured:
        step()                             # (no rows: nothing is taken or written)
        w4a8.check_status(e.ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    rng = random.Random(nodes)
    known = [[] for _ in range(B)]         # the keys and values that each sequence should hold
    held = [0] * B
    for turn in range(7):
        if turn == 4:
            known[1] = []                  # the request ends, another takes its place
        kept = [len(k) for k in known]
        counts = [nodes, rng.randint(1, nodes), rng.randint(0, nodes)] if turn else [nodes] * 3
        trees = [tree_masks([-1 if j == 0 else rng.randint(max(0, j - 4), j - 1) for j in range(c)]) for c in counts]
        flat = [m for t in trees for m in t]
        rows = [(b, i) for b, c in enumerate(counts) for i in range(c)]
        depth = [kept[b] + bin(trees[b][i]).count("1") - 1 for b, i in rows]
        accepted = [sorted(rng.sample(range(c), rng.randint(min(1, c), min(c, most)))) for c in counts]
        want_plan = plan_reference(held, kept, counts, e.table.cpu().numpy(), e.free.cpu().numpy(), int(e.count[0]), P, e.rows)
        Q, K, V = (vectors(t.shape, 100 * turn + k, F16) for k, t in enumerate((e.Q, e.K, e.V)))
        for to, x in ((e.Q, Q), (e.K, K), (e.V, V)):
            to.copy_(x)
        e.kept.copy_(torch.tensor(kept, dtype=torch.int32))
        e.add.copy_(torch.tensor(counts, dtype=torch.int32))
        masks[:len(flat)] = mask_words(flat, words).cuda()
        where[:len(rows)] = i32(depth)
        taken.copy_(torch.tensor([len(p) for p in accepted], dtype=torch.int32))
        for b, p in enumerate(accepted):
            paths[b, :len(p)] = i32(p)
        O.fill_(9.0)
        graph.replay() if captured else step()
        w4a8.check_status(e.ws)
        # the plan
        assert np.array_equal(e.table.cpu().numpy(), want_plan["table"]) and np.array_equal(e.free.cpu().numpy(), want_plan["free"])
        assert e.count.tolist() == want_plan["count"].tolist() and e.held.tolist() == want_plan["lens"].tolist()
        assert np.array_equal(e.slots.cpu().numpy(), want_plan["slots"]) and e.cu.tolist() == want_plan["cu"].tolist()
        held = [k + c for k, c in zip(kept, counts)]
        # rotated queries, and what the rows put into the cache
        n, axis = len(rows), np.zeros(D // 2, np.int64)
        at = np.array(depth + [0] * (e.rows - n), np.int32)[None]
        turned = rotate_reference(Q.float().numpy(), at, axis, e.freq.cpu().numpy(), False)[:n]
        assert torch.equal(e.Q[:n].cpu(), torch.from_numpy(turned).half()) and torch.equal(e.Q[n:].cpu(), Q[n:])
        newK = as_quantized(rotate_reference(K.float().numpy(), at, axis, e.freq.cpu().numpy(), False)[:n])
        newV = as_quantized(V.float().numpy()[:n])
        # the accepted path's tokens lie behind those that were there
        first = [sum(counts[:b]) for b in range(B)]
        for b in range(B):
            known[b] = known[b] + [(newK[first[b] + j], newV[first[b] + j]) for j in accepted[b]]
            if known[b]:
                k, v = e.cached(b, list(range(len(known[b]))))
                assert torch.equal(k, torch.stack([x for x, _ in known[b]])) and torch.equal(v, torch.stack([x for _, x in known[b]]))
        assert lens_after.tolist() == [len(k) for k in known]
        # attention, over the cache as it was in front of the moves: the drafted slots that a move overwrote are put back
        bt = e.host_batch(held, counts)
        before = e.cache.clone()
        # (the rows' vectors again, unturned queries' place is theirs already)
        w4a8.rope_kv_append(e.Q.clone(), e.K, e.V, where, e.freq, before, e.slots, e.ws)
        seen = [seen_in_tree(held[b], counts[b], i, trees[b][i], 0, 0) for b, i in rows]
        o, _, allow = attention_where(e.Q, before, bt, H, D ** -0.5, seen + [[]] * (e.rows - n))
        check_attention(O[:n], o[:n], allow[:n], F16)
        assert bool((O[n:] == 9.0).all())
    w4a8.check_status(e.ws)


def test_long_chat_with_a_window():
    """Prompts, then single tokens, one captured step replayed: the plan's own positions and slots, window and sinks."""
    B, P, H, Hq, D, window, few = 2, 16, 2, 4, 64, 40, 3
    e = Engine(B, P, H, Hq, D, 12, 24, B)
    O = torch.zeros(B, Hq, D, dtype=F16, device="cuda")
    # prompts of 33 and 50 tokens, by calls of their own
    lens, rows = [33, 50], 83
    out = w4a8.kv_plan(None, e.kept, i32(lens), e.table, e.free, e.count, P, rows, e.ws, out=(e.held, None, None, None, e.count))
    K, V, Q = (vectors((rows, h, D), k, F16).cuda() for k, h in enumerate((H, H, Hq)))
    w4a8.rope_kv_append(Q, K, V, out[2], e.freq, e.cache, out[3], e.ws)
    e.kept.copy_(e.held)
    e.add.fill_(1)

    def step():
        e.plan()
        e.kept.copy_(e.held)
        w4a8.rope_kv_append(e.Q, e.K, e.V, e.positions, e.freq, e.cache, e.slots, e.ws, out=e.Q)
        w4a8.kv_attention_sinks(e.Q, e.cache, e.table, e.held, H, e.ws, window, few, out=O)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    state = [t.clone() for t in (e.held, e.kept, e.table, e.free, e.count)]
    with torch.cuda.graph(graph):
        step()
    for t, x in zip((e.held, e.kept, e.table, e.free, e.count), state):
        assert torch.equal(t, x)
    lens = [n + 1 for n in lens]
    for turn in range(60):
        for k, t in enumerate((e.Q, e.K, e.V)):
            t.copy_(vectors(t.shape, 1000 + 3 * turn + k, F16))
        graph.replay()
        lens = [n + 1 for n in lens]
        assert e.held.tolist() == lens and e.positions.tolist() == [n - 1 for n in lens]
        if turn % 13 == 0 or turn == 59:
            bt = e.host_batch(lens, [1, 1])
            seen = [seen_with_sinks(n, 1, 0, True, window, few) for n in lens]
            o, _, allow = attention_where(e.Q, e.cache, bt, H, D ** -0.5, seen)
            check_attention(O, o, allow, F16)
    w4a8.check_status(e.ws)
    assert int(e.count[0]) == 24 - sum(-(-n // P) for n in lens)


def test_two_streams_with_workspaces_of_their_own():
    """The same calls at the same time on two streams: results as one after the other."""
    H, Hq, D, P = 2, 8, 128, 16
    bt = Batch([300, 170], [40, 33], P)
    parents = [[-1] + [random.Random(j).randint(max(0, j - 5), j - 1) for j in range(1, c)] for c in bt.counts]
    bits = mask_words([m for p in parents for m in tree_masks(p)], 2).cuda()
    base = filled_cache(bt, H, D)
    slots = torch.tensor([int(bt.table_host[b, p // P]) * P + p % P for b, p in bt.positions()], device="cuda")
    pos = i32([p for _, p in bt.positions()])
    paths, taken = i32([[1, 5, 9], [0, 2, 30]]), i32([3, 2])

    def calls(k, cache, ws):
        Q, K, V = (vectors((bt.rows, h, D), 7 * k + j, F16).cuda() for j, h in enumerate((Hq, H, H)))
        q = w4a8.rope_kv_append(Q, K, V, pos, frequencies(D), cache, slots, ws)
        o = w4a8.kv_attention_tree(q, cache, bt.table, bt.kv_lens, H, ws, bits, cu_rows=bt.cu)
        p = w4a8.kv_attention_sinks(q, cache, bt.table, bt.kv_lens, H, ws, 50, 4, cu_rows=bt.cu)
        n = w4a8.kv_accept(cache, bt.table, bt.kv_lens, paths, taken, H, D, ws, cu_rows=bt.cu)
        return q, o, p, n, cache

    spaces = [w4a8.new_kv_workspace(bt.rows, 2, Hq, H, D) for _ in range(2)]
    want = [[t.clone() for t in calls(k, base.clone(), spaces[0])] for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(5):
        got = []
        caches = [base.clone() for _ in range(2)]
        torch.cuda.synchronize()
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append(calls(k, caches[k], spaces[k]))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))
    for ws in spaces:
        w4a8.check_status(ws)


def test_pages_beyond_32_bit_offsets():
    """The same pages at the far end of a cache of more than 4 GiB."""
    H, Hq, D, P = 8, 16, 128, 64
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough device memory")
    bt = Batch([200, 165], [40, 33], P)
    small = filled_cache(bt, H, D)
    big = w4a8.new_kv_cache((1 << 32) // small.shape[1] + 2 * bt.num_pages, P, H, D)
    shift = big.shape[0] - bt.num_pages
    big[shift:] = small
    ws = w4a8.new_kv_workspace(bt.rows, 2, Hq, H, D)
    slots = torch.tensor([int(bt.table_host[b, p // P]) * P + p % P for b, p in bt.positions()], device="cuda")
    Q, K, V = (vectors((bt.rows, h, D), k, F16).cuda() for k, h in enumerate((Hq, H, H)))
    pos = i32([p for _, p in bt.positions()])
    far = torch.where(bt.table < 0, bt.table, bt.table + shift)
    bits = mask_words([(2 << i) - 1 for c in bt.counts for i in range(c)], 2).cuda()
    results = []
    for cache, table, off in ((small, bt.table, 0), (big, far, shift)):
        q = w4a8.rope_kv_append(Q, K, V, pos, frequencies(D), cache, slots + off * P, ws)
        o = w4a8.kv_attention_tree(q, cache, table, bt.kv_lens, H, ws, bits, cu_rows=bt.cu)
        p = w4a8.kv_attention_sinks(q, cache, table, bt.kv_lens, H, ws, 77, 4, cu_rows=bt.cu)
        w4a8.kv_accept(cache, table, bt.kv_lens, i32([[3, 39], [32, 0]]), i32([2, 1]), H, D, ws, cu_rows=bt.cu)
        w4a8.check_status(ws)
        results.append((q, o, p, cache[off:off + bt.num_pages]))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    # and a plan whose slots pass 32 bits
    pages = (1 << 31) // 1024 + 5
    free = torch.arange(pages, dtype=torch.int32, device="cuda")
    table = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    out = w4a8.kv_plan(None, i32([0]), i32([2000]), table, free, i32([pages]), 1024, 2000, ws)
    w4a8.check_status(ws)
    assert out[3][0] == (pages - 1) * 1024 and out[3][1999] == (pages - 2) * 1024 + 975 and out[4].tolist() == [pages - 2]


def test_plan_without_positions_or_slots():
    """The C call's optional outputs."""
    P = ctypes.c_void_p
    ws = guarded_workspace(512)
    kept, add = i32([5, 0]), i32([20, 3])
    for with_positions, with_slots in ((False, False), (True, False), (False, True)):
        table, free, count, left = torch.full((2, 2), -1, dtype=torch.int32, device="cuda"), i32([7, 3, 1, 0, 0, 0, 0, 0]), i32([3]), i32([0])
        table[0, 0] = 5
        lens, cu, pos, slots = Guarded((2,), torch.int32), Guarded((3,), torch.int32), Guarded((23,), torch.int32), Guarded((23,), torch.int64)
        st = w4a8.lib.w4a8_kv_plan(None, P(kept.data_ptr()), P(add.data_ptr()), 2, P(table.data_ptr()), 2, 16, P(free.data_ptr()), 8, P(count.data_ptr()),
                                   P(left.data_ptr()), P(lens.t.data_ptr()), P(cu.t.data_ptr()), P(pos.t.data_ptr()) if with_positions else None,
                                   P(slots.t.data_ptr()) if with_slots else None, 23, P(ws.t.data_ptr()), ws.t.numel(),
                                   P(torch.cuda.current_stream().cuda_stream))
        assert st == 0
        w4a8.check_status(ws.t)
        for g in (lens, cu, pos, slots):
            g.check()
        assert lens.t.tolist() == [25, 3] and cu.t.tolist() == [0, 20, 23] and table.tolist() == [[5, 1], [3, -1]] and left.tolist() == [1]
        if with_positions:
            assert pos.t.tolist() == list(range(5, 25)) + [0, 1, 2]
        if with_slots:
            assert slots.t.tolist() == [5 * 16 + p for p in range(5, 16)] + [16 + p for p in range(9)] + [48, 49, 50]


def test_a_table_that_lost_a_page_is_reported():
    """The page into which a sequence's next row goes has no number: no slot, a report, the other rows as planned."""
    ws = guarded_workspace(512)
    table = i32([[-1, -1], [4, -1]])
    out = w4a8.kv_plan(None, i32([5, 5]), i32([1, 1]), table, i32([1, 2, 3, 0, 0]), i32([3]), 16, 2, ws.t)
    assert w4a8.poll_status(ws.t) == 9
    assert out[3].tolist() == [-1, 4 * 16 + 5] and out[2].tolist() == [5, 5]


def test_attention_refusals():
    H, D, P = 2, 64, 16
    bt = Batch([20, 5], None, P)
    cache = filled_cache(bt, H, D)
    ws = w4a8.new_kv_workspace(2, 2, 4, H, D)
    Q, bits = vectors((2, 4, D), 1, F16).cuda(), i32([[1], [1]])

    def sinks(q=Q, c=cache, table=bt.table, lens=bt.kv_lens, heads=H, space=ws, window=9, few=4, **kw):
        return w4a8.kv_attention_sinks(q, c, table, lens, heads, space, window, few, **kw)

    def tree(q=Q, c=cache, table=bt.table, lens=bt.kv_lens, heads=H, space=ws, mask=bits, **kw):
        return w4a8.kv_attention_tree(q, c, table, lens, heads, space, mask, **kw)

    for call in (sinks, tree):
        for error, kw in ((TypeError, dict(q=Q.float())), (TypeError, dict(q=Q.cpu())), (TypeError, dict(table=bt.table.long())), (ValueError, dict(lens=bt.kv_lens[:1])),
                          (ValueError, dict(heads=3)), (ValueError, dict(out=torch.empty(2, 4, 32, dtype=F16, device="cuda"))),
                          (TypeError, dict(out=torch.empty(2, 4, D, device="cuda"))), (ValueError, dict(lse=torch.empty(2, 2, device="cuda"))),
                          (w4a8.W4A8Error, dict(scale=0.0)), (w4a8.W4A8Error, dict(window=-1)), (w4a8.W4A8Error, dict(space=ws[:256])),
                          (w4a8.W4A8Error, dict(q=Q[:, :3].contiguous())), (ValueError, dict(cu_rows=i32([0, 2]))), (TypeError, dict(dtype=torch.float32))):
            with pytest.raises(error):
                call(**kw)
    for error, call in ((w4a8.W4A8Error, lambda: sinks(few=-1)), (TypeError, lambda: sinks(few=None)), (w4a8.W4A8Error, lambda: tree(sinks=-1)),
                        (TypeError, lambda: tree(mask=bits.long())), (TypeError, lambda: tree(mask=bits.cpu())), (ValueError, lambda: tree(mask=bits[:1])),
                        (ValueError, lambda: tree(mask=bits[0])), (w4a8.W4A8Error, lambda: tree(mask=bits[:, :0].contiguous()))):
        with pytest.raises(error):
            call()
    sinks(), tree()
    w4a8.check_status(ws)
    huge = 2 ** 31 - 1                     # the largest window and sinks: all of the sequence
    want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws)
    for window, few in ((huge, 4), (3, huge), (huge, huge)):
        assert torch.allclose(sinks(window=window, few=few).float(), want.float(), rtol=2 ** -9, atol=2 ** -9)


def test_bad_tables_are_reported():
    H, D, P = 2, 64, 16
    cache = w4a8.new_kv_cache(4, P, H, D).fill_(0)
    good = i32([[0], [1]])
    for rows in (2, 8, 100):                               # one row each, a few, many
        Q = vectors((rows, 4, D), 1, F16).cuda()
        bits = torch.full((rows, 4), -1, dtype=torch.int32, device="cuda")
        ws = w4a8.new_kv_workspace(rows, 2, 4, H, D)
        ok = None if rows == 2 else i32([0, rows // 2, rows])
        for table, lens, cu in ((i32([[4], [1]]), i32([3, 3]), ok), (i32([[0], [-1]]), i32([9, 9]), ok), (good, i32([3, 17]), ok), (good, i32([-1, 3]), ok),
                                (good, i32([3, 3]), i32([0, 1, rows + 1])), (good, i32([3, 3]), i32([0, -4, 2]))):
            w4a8.kv_attention_sinks(Q, cache, table, lens, H, ws, 200, 4, cu_rows=cu)
            assert w4a8.poll_status(ws) == 9, (rows, table, lens, cu)
            w4a8.kv_attention_tree(Q, cache, table, lens, H, ws, bits, cu_rows=cu)
            assert w4a8.poll_status(ws) == 9, (rows, table, lens, cu)
        w4a8.kv_attention_sinks(Q, cache, good, i32([9, 9]), H, ws, 5, 2, cu_rows=ok)
        w4a8.kv_attention_tree(Q, cache, good, i32([9, 9]), H, ws, bits, cu_rows=ok)
        w4a8.check_status(ws)
