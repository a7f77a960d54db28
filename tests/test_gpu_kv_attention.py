"""Attention over the paged dINT4 cache against binary64 attention over the values it holds."""
import math

import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, attention_reference, check_attention, filled_cache, vectors
from util import Guarded

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def run(lens, rows, P, Hq, H, D, q_type=F16, o_type=F16, causal=True, window=0, pad=0, seed=0, q_scale=1.0, v_scale=1.0,
        scale=None):
    bt = Batch(lens, rows, P, pad, seed=seed)
    cache = filled_cache(bt, H, D, seed=seed + 5, scale=v_scale)
    Q = (q_scale * torch.randn(bt.rows, Hq, D, generator=torch.Generator().manual_seed(seed + 9))).to(q_type).cuda()
    ws = Guarded((w4a8.kv_attention_workspace_bytes(bt.rows, len(lens), Hq, H, D),), torch.uint8)
    w4a8.workspace_init(ws.t)
    out, lse = Guarded((bt.rows, Hq, D), o_type), Guarded((bt.rows, Hq), torch.float32)
    out.t.fill_(7.0)
    lse.t.fill_(7.0)
    scale = 1.0 / math.sqrt(D) if scale is None else scale

    def call():
        w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws.t, cu_rows=bt.cu, scale=scale, causal=causal, window=window,
                          out=out.t, lse=lse.t)
        w4a8.check_status(ws.t)
        return out.t.clone()

    O = call()
    out.check("O")
    lse.check("lse")
    ws.check("workspace")
    o, want_lse, allow = attention_reference(Q, cache, bt, H, scale, causal, window)
    n = bt.used
    check_attention(O[:n], o[:n], allow[:n], o_type)
    got_lse = lse.t[:n].cpu().double()
    finite = torch.isfinite(want_lse[:n])
    assert torch.equal(finite, torch.isfinite(got_lse))
    # ln of the denominator: the scores' allowance again, and binary32
    qsum = Q[:n].cpu().double().abs().sum(-1)
    off = (D / 16 + 4) * 2.0 ** -23 * 30 * qsum * 2.0 * v_scale * scale + 2.0 ** -19 * (1 + want_lse[:n].abs())
    assert bool(((got_lse - want_lse[:n]).abs()[finite] <= off[finite]).all())
    assert bool((O[n:] == 7.0).all()) and bool((lse.t[n:] == 7.0).all())      # padding rows
    assert torch.equal(call(), O)                                              # the same bits again
    return O


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 4), (8, 2), (5, 1), (7, 1), (16, 2), (16, 1), (24, 1), (12, 3)])
def test_decode_head_layouts(D, Hq, H):
    run([1, 0, 15, 16, 17, 100, 33], None, 16, Hq, H, D)


@pytest.mark.parametrize("q_type", [F16, BF16])
@pytest.mark.parametrize("o_type", [F16, BF16])
def test_types(q_type, o_type):
    run([70, 3, 129], None, 32, 8, 2, 128, q_type, o_type)
    run([70, 3, 129], [4, 3, 9], 32, 8, 2, 64, q_type, o_type)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
def test_page_sizes(P):
    run([1000, 1, 64, 63, 65, 513], None, P, 8, 2, 128, BF16)


@pytest.mark.parametrize("rows", [[2, 1, 0, 5], [17, 3, 1, 33], [64, 64, 64, 64]])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 21])
def test_several_rows_per_sequence(rows, causal, window):
    run([130, 3, 40, 64], rows, 32, 6, 2, 64, causal=causal, window=window, pad=2)
    if window != 1:
        run([130, 3, 40, 64], rows, 32, 4, 1, 128, BF16, BF16, causal=causal, window=window)


def test_rows_that_see_nothing():
    """More rows than tokens: the rows in front of position 0 get zeros; an empty sequence too."""
    O = run([2, 0, 5], [6, 3, 1], 16, 4, 2, 64)
    assert bool((O[:4] == 0).all()) and bool((O[6:9] == 0).all()) and bool((O[4:6] != 0).any())
    for rows in ([6, 3, 1], [150, 3, 70]):                 # a window beyond any position hides nothing
        assert torch.equal(run([2, 0, 5], rows, 16, 4, 2, 64), run([2, 0, 5], rows, 16, 4, 2, 64, window=2 ** 31 - 1))


@pytest.mark.parametrize("window", [1, 7, 16, 100, 5000])
def test_window_decode(window):
    run([1, 40, 300, 129], None, 16, 8, 2, 128, window=window)


def test_long_sequence_and_split():
    run([40001], None, 64, 8, 2, 128, BF16, BF16)
    run([9000, 1, 33, 2500], [1, 1, 3, 2], 64, 4, 4, 64)


def test_many_sequences():
    rng = np.random.default_rng(3)
    run([int(v) for v in rng.integers(0, 90, 300)], None, 16, 4, 2, 64)


@pytest.mark.parametrize("q_scale", [1e-3, 30.0])
def test_flat_and_peaked_weights(q_scale):
    run([257, 1000], None, 64, 8, 2, 128, q_scale=q_scale)
    run([257, 100], [33, 100], 64, 8, 2, 128, q_scale=q_scale)


@pytest.mark.parametrize("v_scale", [2.0 ** -14, 200.0])
def test_small_and_large_cached_values(v_scale):
    run([257, 31], None, 64, 8, 2, 128, F16, BF16, v_scale=v_scale, scale=0.1 / v_scale)


def test_garbage_behind_the_sequence_is_not_seen():
    """Slots behind a sequence's end and unused pages hold words that are infinities and NaN."""
    H, D, P = 2, 128, 64
    for lens, rows in (([5, 70, 64, 17], None), ([5, 70, 64, 17], [5, 40, 2, 17])):
        bt = Batch(lens, rows, P)
        cache = filled_cache(bt, H, D)
        Q = torch.randn(bt.rows, 8, D, generator=torch.Generator().manual_seed(1)).to(F16).cuda()
        ws = w4a8.new_kv_workspace(bt.rows, 4, 8, H, D)
        want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu).clone()
        raw = cache.view(bt.num_pages, H, P // 16, 16 * (D + 8))
        seen = torch.zeros(bt.num_pages, P, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                seen[bt.table_host[b, j // P], j % P] = True
        words = raw[..., 16 * D:].contiguous().view(torch.int32).view(bt.num_pages, H, P // 16, 2, 16)
        hidden = (~seen).view(bt.num_pages, 1, P // 16, 1, 16).cuda().expand_as(words)
        for bits in (0x7F800000, 0x7FFFFFFF, -1):
            words[hidden] = bits
            raw[..., 16 * D:] = words.view(torch.uint8).reshape(bt.num_pages, H, P // 16, 128)
            got = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu)
            w4a8.check_status(ws)
            assert torch.equal(got, want)


def test_strided_queries_other_stream_and_graph():
    """Queries as a slice of a wider projection; on another stream; captured and replayed on new lengths."""
    H, D, P, Hq = 2, 128, 32, 8
    bt = Batch([200, 90, 31], None, P)
    cache = filled_cache(bt, H, D)
    wide = vectors((3, Hq + 2 * H, D), 4, F16).cuda()
    Q = wide[:, :Hq]
    ws = w4a8.new_kv_workspace(3, 3, Hq, H, D)
    want = w4a8.kv_attention(Q.contiguous(), cache, bt.table, bt.kv_lens, H, ws)
    assert torch.equal(w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    with torch.cuda.stream(side):
        w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, out=out)
    for lens in ([200, 90, 31], [1, 0, 17], [150, 90, 1]):
        bt.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        got = out.clone()
        bt.lens = lens
        o, _, allow = attention_reference(Q, cache, bt, H, 1 / math.sqrt(D))
        check_attention(got, o, allow, F16)
    w4a8.check_status(ws)


@pytest.mark.parametrize("lens,rows,P,Hq,H,D,window", [
    ([700, 300, 0, 64], [513, 300, 0, 1], 32, 10, 2, 128, 0),       # five heads share a key head: rows straddle row tiles
    ([700, 300, 9, 64], [90, 300, 9, 64], 16, 7, 1, 64, 100),
    ([300], [257], 64, 1, 1, 128, 0),                               # one head alone; a second row tile of one row
    ([129, 65, 63, 64, 1], [129, 65, 63, 64, 1], 128, 24, 1, 64, 0),
    ([2000, 10], [20, 10], 16, 16, 2, 128, 1900),
    ([20000], [24], 64, 8, 2, 128, 0),                              # every item is shared by many CTAs
])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows(lens, rows, P, Hq, H, D, window, causal):
    run(lens, rows, P, Hq, H, D, BF16, F16, causal=causal, window=window, pad=3)


def test_one_distant_token_against_many_light_ones():
    """One token holds most of the weight and thousands hold 2^-27 of it each: a reference that sat on the
    largest exponent would round those to binary16's zero."""
    H, D, P, n = 1, 64, 64, 6000
    for rows in (1, 96):
        bt = Batch([n], [rows], P)
        K = torch.zeros(n, 1, D)
        K[0, 0, 0] = 1.0
        V = torch.ones(n, 1, D)
        V[0] = -1.0
        cache = w4a8.new_kv_cache(bt.num_pages, P, H, D).fill_(0)
        ws = w4a8.new_kv_workspace(rows, 1, 1, H, D)
        w4a8.kv_append(K.half().cuda(), V.half().cuda(), cache, bt.table, bt.kv_lens, ws,
                       cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
        Q = torch.zeros(rows, 1, D)
        Q[:, 0, 0] = 27 * math.log(2.0)
        Q = Q.half().cuda()
        O = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, scale=1.0, dtype=BF16)
        w4a8.check_status(ws)
        o, _, allow = attention_reference(Q, cache, bt, H, 1.0)
        check_attention(O, o, allow, BF16)


@pytest.mark.parametrize("rows", [None, 100])
@pytest.mark.parametrize("extreme", ["large", "inf", "nan"])
def test_a_row_of_extreme_queries_leaves_the_others_alone(rows, extreme):
    """One query head of one row holds values 2^90 above the others', or ones that are not finite: the other
    rows and heads of its tile are what they are without it."""
    H, D, n = 2, 128, 300
    bt = Batch([n], None if rows is None else [rows], 64)
    cache = filled_cache(bt, H, D)
    Q = vectors((bt.rows, 8, D), 3, BF16)
    row, head = bt.rows // 2, 1
    Q[row, head] = {"large": Q[row, head] * 2.0 ** 90, "inf": math.inf, "nan": math.nan}[extreme]
    Q[row, 7] *= 2.0 ** -20                                # and a small one, apart from its tile without the large one
    Q = Q.cuda()
    ws = w4a8.new_kv_workspace(bt.rows, 1, 8, H, D)
    O = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, scale=0.1)
    w4a8.check_status(ws)
    Q[row, head] = 0
    o, _, allow = attention_reference(Q, cache, bt, H, 0.1)
    O[row, head] = 0
    o[row, head] = 0
    check_attention(O, o, allow, F16)


def _problem(lens, rows, P, Hq, H, D, seed):
    bt = Batch(lens, rows, P, seed=seed)
    cache = filled_cache(bt, H, D, seed=seed)
    Q = vectors((bt.rows, Hq, D), seed + 3, F16).cuda()
    return bt, cache, Q, H


def test_calls_of_different_forms_share_a_workspace():
    """Many-row and few-row calls in turn on one workspace, with other kernels' leavings on the chip between
    them: every call gives the bits that it gives alone on a fresh workspace."""
    problems = [_problem([3000], [100], 64, 8, 2, 128, 1), _problem([700, 1, 2500], None, 32, 16, 2, 128, 2),
                _problem([300, 40], [300, 40], 16, 6, 2, 64, 3), _problem([5000], None, 64, 8, 1, 64, 4),
                _problem([900, 900], [6, 7], 64, 8, 2, 128, 5)]
    size, want = 0, []
    for bt, cache, Q, H in problems:
        n = w4a8.kv_attention_workspace_bytes(bt.rows, len(bt.lens), Q.shape[1], H, Q.shape[2])
        size = max(size, n)
        want.append(w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, w4a8.new_kv_workspace(
            bt.rows, len(bt.lens), Q.shape[1], H, Q.shape[2]), cu_rows=bt.cu))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    w4a8.workspace_init(ws)
    noise = torch.randn(2048, 2048, device="cuda").half()
    order = [0, 1, 2, 3, 4, 1, 0, 4, 2, 0, 3, 1]
    got = []
    for k in order:
        bt, cache, Q, H = problems[k]
        got.append(w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu))
        if k % 2 == 0:
            noise = (noise @ noise).clamp(-1, 1)
    w4a8.check_status(ws)
    for k, o in zip(order, got):
        assert torch.equal(o, want[k]), k


def test_streams_and_graphs_with_workspaces_of_their_own():
    """Calls that overlap on two streams, and two captured graphs, each with its own workspace."""
    for lens, rows in (([4000, 100, 9], None), ([2000, 500], [200, 100])):
        bt, cache, Q, H = _problem(lens, rows, 64, 8, 2, 128, 11)
        spaces = [w4a8.new_kv_workspace(bt.rows, len(lens), 8, H, 128) for _ in range(2)]
        want = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, spaces[0], cu_rows=bt.cu)
        streams = [torch.cuda.Stream() for _ in range(2)]
        outs = [[torch.empty_like(want) for _ in range(6)] for _ in range(2)]
        torch.cuda.synchronize()
        for k in range(6):
            for st, ws, out in zip(streams, spaces, outs):
                with torch.cuda.stream(st):
                    w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, out=out[k])
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for out in outs for o in out)
        graphs, held = [], []
        for ws in spaces:
            graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
            with torch.cuda.graph(graph):
                w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, out=out)
            graphs.append(graph)
            held.append(out)
        for _ in range(3):
            for graph, st, out in zip(graphs, streams, held):
                with torch.cuda.stream(st):
                    out.zero_()
                    graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for out in held)
        for ws in spaces:
            w4a8.check_status(ws)


def test_captured_call_of_many_rows_follows_its_inputs():
    """Replays with other lengths, row counts and queries in the captured tensors."""
    bt, cache, Q, H = _problem([400, 300], [60, 40], 32, 8, 2, 128, 21)
    ws = w4a8.new_kv_workspace(bt.rows, 2, 8, H, 128)
    out = torch.zeros(bt.rows, 8, 128, dtype=F16, device="cuda")
    w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu, out=out)
    for k, (lens, counts) in enumerate([([400, 300], [60, 40]), ([100, 1], [99, 1]), ([33, 300], [0, 100]), ([0, 0], [50, 50]),
                                        ([400, 17], [1, 1])]):
        bt.lens, bt.counts = lens, counts
        bt.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        bt.cu.copy_(torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32))
        Q.copy_(vectors(Q.shape, 30 + k, F16))
        out.fill_(5.0)
        graph.replay()
        o, _, allow = attention_reference(Q, cache, bt, H, 128 ** -0.5)
        n = sum(counts)
        check_attention(out[:n].clone(), o[:n], allow[:n], F16)
        assert bool((out[n:] == 5.0).all())
    w4a8.check_status(ws)


def test_pages_beyond_32_bit_offsets():
    """The same pages at the far end of a cache of more than 4 GiB."""
    H, D, P = 8, 128, 64
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough device memory")
    for lens, rows in (([200, 65], None), ([200, 65], [100, 65])):
        bt = Batch(lens, rows, P)
        small = filled_cache(bt, H, D)
        big = w4a8.new_kv_cache((1 << 32) // small.shape[1] + 2 * bt.num_pages, P, H, D)
        shift = big.shape[0] - bt.num_pages
        big[shift:] = small
        Q = vectors((bt.rows, 16, D), 3, F16).cuda()
        ws = w4a8.new_kv_workspace(bt.rows, 2, 16, H, D)
        want = w4a8.kv_attention(Q, small, bt.table, bt.kv_lens, H, ws, cu_rows=bt.cu)
        got = w4a8.kv_attention(Q, big, torch.where(bt.table < 0, bt.table, bt.table + shift), bt.kv_lens, H, ws, cu_rows=bt.cu)
        w4a8.check_status(ws)
        assert torch.equal(got, want)


def test_refusals():
    H, D, P = 2, 64, 16
    bt = Batch([20, 5], None, P)
    cache = filled_cache(bt, H, D)
    ws = w4a8.new_kv_workspace(2, 2, 4, H, D)
    Q = vectors((2, 4, D), 1, F16).cuda()
    K = vectors((2, H, D), 1, F16).cuda()

    def attend(q=Q, c=cache, table=bt.table, lens=bt.kv_lens, heads=H, space=ws, **kw):
        return w4a8.kv_attention(q, c, table, lens, heads, space, **kw)

    for error, call in (
            (TypeError, lambda: attend(q=Q.float())), (TypeError, lambda: attend(q=Q.cpu())), (TypeError, lambda: attend(q=Q.view(2, -1))),
            (TypeError, lambda: attend(table=bt.table.long())), (TypeError, lambda: attend(lens=bt.kv_lens.long())),
            (TypeError, lambda: attend(c=cache.view(torch.int32))), (ValueError, lambda: attend(lens=bt.kv_lens[:1])),
            (ValueError, lambda: attend(heads=3)), (ValueError, lambda: attend(c=cache[:, :-8].contiguous())),
            (ValueError, lambda: attend(out=torch.empty(2, 4, 32, dtype=F16, device="cuda"))),
            (TypeError, lambda: attend(out=torch.empty(2, 4, D, device="cuda"))),
            (ValueError, lambda: attend(lse=torch.empty(2, 2, device="cuda"))), (w4a8.W4A8Error, lambda: attend(scale=0.0)),
            (w4a8.W4A8Error, lambda: attend(scale=float("nan"))), (w4a8.W4A8Error, lambda: attend(window=-1)),
            (w4a8.W4A8Error, lambda: attend(q=Q[:, :3].contiguous())), (w4a8.W4A8Error, lambda: attend(space=ws[:256])),
            (w4a8.W4A8Error, lambda: attend(q=torch.cat([Q, Q]))),
            (ValueError, lambda: attend(cu_rows=torch.zeros(2, dtype=torch.int32, device="cuda"))),
            (TypeError, lambda: w4a8.kv_append(K, K.bfloat16(), cache, bt.table, bt.kv_lens, ws)),
            (ValueError, lambda: w4a8.kv_append(K, K[:1], cache, bt.table, bt.kv_lens, ws)),
            (w4a8.W4A8Error, lambda: w4a8.kv_append(K[:1], K[:1], cache, bt.table, bt.kv_lens, ws)),
            (TypeError, lambda: w4a8.kv_read(cache, bt.table, bt.kv_lens, 2, H, D, ws, dtype=torch.float32))):
        with pytest.raises(error):
            call()
    attend()
    w4a8.check_status(ws)


def test_bad_tables_are_reported():
    H, D, P = 2, 64, 16
    cache = w4a8.new_kv_cache(4, P, H, D).fill_(0)
    ws = w4a8.new_kv_workspace(8, 2, 4, H, D)

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    good = i32(0, 1).view(2, 1)
    for rows in (2, 8, 100):                               # one row each, a few, many
        Q = vectors((rows, 4, D), 1, F16).cuda()
        ws = w4a8.new_kv_workspace(rows, 2, 4, H, D)
        ok = None if rows == 2 else i32(0, rows // 2, rows)
        for table, lens, cu in ((i32(4, 1).view(2, 1), i32(3, 3), ok), (i32(0, -1).view(2, 1), i32(9, 9), ok),
                                (good, i32(3, 17), ok), (good, i32(-1, 3), ok), (good, i32(3, 3), i32(0, 1, rows + 1)),
                                (good, i32(3, 3), i32(0, -4, 2))):
            w4a8.kv_attention(Q, cache, table, lens, H, ws, cu_rows=cu)
            assert w4a8.poll_status(ws) == 9, (rows, table, lens, cu)
        w4a8.kv_attention(Q, cache, good, i32(9, 9), H, ws, cu_rows=ok)
        w4a8.check_status(ws)


def test_decoder_step_through_the_public_calls():
    """qkv linear -> append -> attention -> quantizer -> output linear -> residual + norm + quantizer, three
    steps of two sequences, against the same step with dequantized tensors in binary64."""
    from paper_2311_05161_b200 import synth
    Hq, H, D, K, P = 4, 2, 64, 256, 16
    qkv_n = (Hq + 2 * H) * D
    g = torch.Generator().manual_seed(0)
    lay1, lay2 = synth.make_layer(K, qkv_n, 2, seed=1), synth.make_layer(Hq * D, K, 2, seed=2)
    p1, p2 = (w4a8.pack_weights(torch.from_numpy(l["W"]).cuda()) for l in (lay1, lay2))
    ws1, ws2 = w4a8.new_workspace(2, qkv_n, K), w4a8.new_workspace(2, K, Hq * D)
    ws = w4a8.new_kv_workspace(2, 2, Hq, H, D)
    bt = Batch([13, 20], None, P)
    cache = filled_cache(bt, H, D)
    stream = torch.randn(2, K, generator=g).cuda()
    weight = torch.ones(K, device="cuda")
    Xq, tok = w4a8.quantize_act(torch.randn(2, K, generator=g).half().cuda())
    for step in range(3):
        lens = [14 + step, 21 + step]
        bt.lens = lens
        bt.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        qkv = w4a8.linear(Xq, tok, p1, None, qkv_n, 0, ws1).view(2, Hq + 2 * H, D)
        w4a8.kv_append(qkv[:, Hq:Hq + H], qkv[:, Hq + H:], cache, bt.table, bt.kv_lens, ws)
        Q = qkv[:, :Hq]
        o = w4a8.kv_attention(Q, cache, bt.table, bt.kv_lens, H, ws)
        want, _, allow = attention_reference(Q, cache, bt, H, D ** -0.5)
        check_attention(o, want, allow, F16)
        Oq, otok = w4a8.quantize_act(o.view(2, Hq * D))
        y = w4a8.linear(Oq, otok, p2, None, K, 0, ws2)
        before = stream.clone()
        Xq, tok, stream = w4a8.add_norm_quantize_act(y, stream, weight, residual_out=stream)
        assert torch.equal(stream, before + y.float())
        x = stream.double()
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(1e-5)))
        # half a code, and the binary32 roundings of x and of its product with 127 / amax
        assert bool(((Xq.double() * tok.double()[:, None] - x).abs() <= (0.5 + 127 * 2.0 ** -21) * tok.double()[:, None]).all())
    for w in (ws, ws1, ws2):
        w4a8.check_status(w)
