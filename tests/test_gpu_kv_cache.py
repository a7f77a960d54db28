"""The paged dINT4 cache on the GPU: bytes written by kv_append and values given back by kv_read
against the definitions."""
import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import LARGEST, Batch, decode_pages, encode_block, quantize_vectors, vectors
from util import Guarded

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]


def new_ws(H, D):
    return w4a8.new_kv_workspace(1, 1, H, H, D)


def guarded_cache(bt, H, D):
    g = Guarded((bt.num_pages, w4a8.kv_page_bytes(bt.P, H, D)), torch.uint8)
    g.t.fill_(0x5A)
    return g


def expected(bt, H, D, K, V, before):
    """The cache bytes after the append, block by block."""
    want = before.cpu().numpy().copy().reshape(bt.num_pages, H, bt.P // 16, 16 * (D + 8))
    Kf, Vf = K.cpu().float().numpy(), V.cpu().float().numpy()
    for row, (b, pos) in enumerate(bt.positions()):
        if pos < 0:
            continue
        page, slot = bt.table_host[b, pos // bt.P], pos % bt.P
        s, c = slot % 16, D // 16
        for h in range(H):
            pad = np.zeros((16, D), np.float32)
            k, v = pad.copy(), pad.copy()
            k[s], v[s] = Kf[row, h], Vf[row, h]
            blk, to = encode_block(k, v), want[page, h, slot // 16]
            to[s * D // 2:(s + 1) * D // 2] = blk[s * D // 2:(s + 1) * D // 2]
            for g in range(8):
                at = 8 * D + ((s // 8 * 8 + g) * 8 + s % 8) * c
                to[at:at + c] = blk[at:at + c]
            for at in (16 * D + 4 * s, 16 * D + 64 + 4 * s):
                to[at:at + 4] = blk[at:at + 4]
    return want.reshape(bt.num_pages, -1)


CASES = [  # lens, rows, P, H, D, padding rows
    ([1], None, 16, 1, 64, 0),
    ([5, 16, 17, 33], None, 16, 3, 128, 0),
    ([40], [40], 32, 2, 128, 0),
    ([19, 0, 130, 64], [19, 0, 7, 64], 64, 5, 64, 3),
    ([3, 2], [5, 2], 16, 2, 128, 1),                  # two rows in front of position 0
    ([1024 + 7], [9], 1024, 1, 128, 0),
    ([7] * 70, [1, 0] * 35, 16, 1, 64, 5),            # more sequences than a warp has lanes
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_writes_the_defined_bytes_and_read_gives_them_back(case, dtype):
    lens, rows, P, H, D, pad = CASES[case]
    bt = Batch(lens, rows, P, pad, seed=case)
    K, V = vectors((bt.rows, H, D), 10 + case, dtype, 1.7).cuda(), vectors((bt.rows, H, D), 20 + case, dtype, 0.6).cuda()
    g, ws = guarded_cache(bt, H, D), new_ws(H, D)
    before = g.t.clone()
    w4a8.kv_append(K, V, g.t, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    w4a8.check_status(ws)
    g.check("cache")
    assert np.array_equal(g.t.cpu().numpy(), expected(bt, H, D, K, V, before))
    gk, gv = Guarded((bt.rows, H, D), dtype), Guarded((bt.rows, H, D), dtype)
    gk.t.fill_(7.0)
    gv.t.fill_(7.0)
    w4a8.kv_read(g.t, bt.table, bt.kv_lens, bt.rows, H, D, ws, cu_rows=bt.cu, out=(gk.t, gv.t))
    w4a8.check_status(ws)
    gk.check("K")
    gv.check("V")
    for got, x in ((gk.t, K), (gv.t, V)):
        lev, step, _ = quantize_vectors(x.cpu().float().numpy())
        want = torch.from_numpy(lev.astype(np.float32) * step).clamp(-LARGEST[dtype], LARGEST[dtype]).to(dtype)
        for row, (b, pos) in enumerate(bt.positions()):
            if pos < 0:
                want[row] = 0
        want[bt.used:] = 7.0                          # rows behind the last sequence are left alone
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantization_error_is_within_the_format(dtype):
    """An element is off by at most half a step, and inside (-3/4, 3/4) steps by a quarter; the range ends by the
    zero-point's rounding (half a step) more.  binary32 decisions: 2^-20 of a step."""
    D, H = 128, 4
    bt = Batch([48], [48], 16)
    x = vectors((48, H, D), 5, dtype).cuda()
    cache, ws = w4a8.new_kv_cache(bt.num_pages, 16, H, D), new_ws(H, D)
    w4a8.kv_append(x, x, cache, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    K, V, ks, vs = decode_pages(cache, H, D, 16)
    pages = torch.from_numpy(bt.table_host[0]).long()
    for got, step in ((K, ks), (V, vs)):
        got = got[pages].transpose(0, 1).reshape(H, -1, D).transpose(0, 1)
        step = step[pages].transpose(0, 1).reshape(H, -1).transpose(0, 1)[..., None]
        u, e = x.cpu().double() / step, (got - x.cpu().double()).abs() / step
        assert bool((e <= 1.0 + 2.0 ** -19).all())
        assert bool((e[u.abs() < 0.75] <= 0.25 + 2.0 ** -19).all())
        inner = (u > u.amin(-1, keepdim=True) + 0.51) & (u < u.amax(-1, keepdim=True) - 0.51)
        assert bool((e[inner] <= 0.5 + 2.0 ** -19).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_extreme_vectors(dtype):
    """Zeros, constants, one-sided, ties, the type's largest and smallest values."""
    D, H = 64, 1
    top, tiny = LARGEST[dtype], float(torch.finfo(dtype).tiny)
    rows = [torch.zeros(D), torch.full((D,), 3.0), torch.full((D,), -2.5), torch.linspace(0, 13, D), torch.linspace(-13, 0, D),
            torch.arange(D) % 27 * 0.25 - 3.25, torch.full((D,), top), torch.linspace(-1, 1, D) * top,
            torch.full((D,), tiny), torch.linspace(-tiny, tiny, D), -torch.zeros(D), (torch.arange(D) == 5) * 1e-3]
    x = torch.stack([r.float() for r in rows]).to(dtype).view(-1, H, D).cuda()
    n = x.shape[0]
    bt = Batch([n], [n], 16)
    cache, ws = w4a8.new_kv_cache(bt.num_pages, 16, H, D), new_ws(H, D)
    w4a8.kv_append(x, x, cache, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    K, V = w4a8.kv_read(cache, bt.table, bt.kv_lens, n, H, D, ws, cu_rows=bt.cu, dtype=dtype)
    lev, step, _ = quantize_vectors(x.cpu().float().numpy())
    with np.errstate(over="ignore"):
        want = torch.from_numpy(lev.astype(np.float32) * step).clamp(-top, top).to(dtype)
    assert torch.equal(K.cpu(), want) and torch.equal(V.cpu(), want)
    assert bool(torch.isfinite(K.float()).all())


@pytest.mark.parametrize("D", [64, 128])
def test_slices_of_a_fused_projection(D):
    H, bt = 3, Batch([33, 20], [6, 20], 32)
    wide = vectors((bt.rows, 4 * H + 1, D), 3, torch.float16).cuda()
    K, V = wide[:, H:2 * H], wide[:, 3 * H + 1:]
    a, b = w4a8.new_kv_cache(bt.num_pages, 32, H, D).fill_(0), w4a8.new_kv_cache(bt.num_pages, 32, H, D).fill_(0)
    ws = new_ws(H, D)
    w4a8.kv_append(K, V, a, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    w4a8.kv_append(K.contiguous(), V.contiguous(), b, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    w4a8.check_status(ws)
    assert torch.equal(a, b) and bool(a.any())


def test_bad_pages_lengths_and_offsets_are_reported():
    """Numbers the kernels check before they use them as an index."""
    H, D, P = 2, 64, 16
    K = vectors((2, H, D), 1, torch.float16).cuda()
    cache, ws = w4a8.new_kv_cache(4, P, H, D).fill_(0), new_ws(H, D)

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    good = i32(0, 1).view(2, 1)
    for table, lens, cu in ((i32(4, 1).view(2, 1), i32(3, 3), None), (i32(0, -1).view(2, 1), i32(3, 3), None),
                            (good, i32(3, 17), None), (good, i32(-1, 3), None),
                            (good, i32(3, 3), i32(0, 1, 5))):
        w4a8.kv_append(K, K, cache, table, lens, ws, cu_rows=cu)
        assert w4a8.poll_status(ws) == 9
        w4a8.kv_read(cache, table, lens, 2, H, D, ws, cu_rows=cu)
        assert w4a8.poll_status(ws) == 9
        assert w4a8.poll_status(ws) == 0             # cleared by the poll
    w4a8.kv_append(K, K, cache, good, i32(3, 3), ws)
    w4a8.check_status(ws)


def test_pages_beyond_32_bit_offsets():
    """A cache of more than 2^32 bytes: the last page's bytes and values."""
    H, D, P = 8, 128, 1024
    nbytes = w4a8.kv_page_bytes(P, H, D)
    pages = (1 << 32) // nbytes + 3
    cache = torch.empty((pages, nbytes), dtype=torch.uint8, device="cuda")
    ws = w4a8.new_kv_workspace(2, 2, H, H, D)
    table = torch.tensor([[pages - 1], [0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([P, 5], dtype=torch.int32, device="cuda")
    K, V = vectors((2, H, D), 1, torch.float16).cuda(), vectors((2, H, D), 2, torch.float16).cuda()
    w4a8.kv_append(K, V, cache, table, lens, ws)
    k, v = w4a8.kv_read(cache, table, lens, 2, H, D, ws)
    w4a8.check_status(ws)
    for got, x in ((k, K), (v, V)):
        lev, step, _ = quantize_vectors(x.cpu().float().numpy())
        assert torch.equal(got.cpu(), torch.from_numpy(lev.astype(np.float32) * step).to(torch.float16))
