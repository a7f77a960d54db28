"""Rotary positions with the cache write: the rotation's operations one by one, and the cache's bytes as kv_append's quantizer gives them."""
import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import encode_block, vectors
from serving_util import rotate_reference
from util import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def frequencies(rot, base=10000.0):
    return torch.from_numpy((base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)).cuda()


def rounded(x, dtype):
    """Rounded once, to the largest finite value beyond the range."""
    top = torch.finfo(dtype).max
    return torch.from_numpy(x).clamp(-top, top).to(dtype)


def cache_image(K, V, slots, pages, P, H, D):
    """The bytes of the written vectors, and which bytes they are: K, V numpy float32 [rows, H, D]."""
    want, there = np.zeros((pages, H, P // 16, 16 * (D + 8)), np.uint8), np.zeros((pages, H, P // 16, 16 * (D + 8)), bool)
    for r, slot in enumerate(slots):
        if not 0 <= slot < pages * P:
            continue
        page, place = slot // P, slot % P
        s, c = place % 16, D // 16
        for h in range(H):
            k16, v16 = np.zeros((16, D), np.float32), np.zeros((16, D), np.float32)
            k16[s], v16[s] = K[r, h], V[r, h]
            block = encode_block(k16, v16)
            at = list(range(s * (D // 2), (s + 1) * (D // 2))) + [16 * D + 4 * s + i for i in range(4)] + [16 * D + 64 + 4 * s + i for i in range(4)]
            at += [8 * D + ((s // 8 * 8 + g) * 8 + s % 8) * c + i for g in range(8) for i in range(c)]
            want[page, h, place // 16, at], there[page, h, place // 16, at] = block[at], True
    return want, there


def run(rows, Hq, H, D, rot, P=16, axes=1, interleaved=False, dtype=F16, fused=False, seed=0, far=5000, in_place=False, skip=(), scale=1.0):
    rng = np.random.default_rng(seed)
    top = torch.finfo(dtype).max
    wide = vectors((rows, Hq + 2 * H, D), seed, dtype, scale).clamp(-top, top).cuda()
    if fused:
        Q, K, V = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]
    else:
        Q, K, V = (x.contiguous() for x in (wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]))
    pages = -(-rows // P) + 2
    slots = rng.permutation(pages * P)[:rows].astype(np.int64)
    for r in skip:
        slots[r] = -1 - r
    positions = rng.integers(0, far, (axes, rows)).astype(np.int32)
    axis = rng.integers(0, axes, rot // 2).astype(np.int32)
    freq = frequencies(rot)
    cache = Guarded((pages, w4a8.kv_page_bytes(P, H, D)), torch.uint8)
    cache.t.fill_(0x3C)
    out = Guarded((rows, Hq, D), dtype)
    out.t.fill_(7.0)
    ws = guarded_workspace(256)
    x = wide.float().cpu().numpy()
    pos = torch.from_numpy(positions if axes > 1 else positions[0]).cuda()
    got = w4a8.rope_kv_append(Q, K, V, pos, freq, cache.t, torch.from_numpy(slots).cuda(), ws.t,
                              pair_axis=torch.from_numpy(axis).cuda() if axes > 1 else None, interleaved=interleaved, out=Q if in_place else out.t)
    w4a8.check_status(ws.t)
    for g, what in ((cache, "cache"), (out, "Q_out"), (ws, "workspace")):
        g.check(what)
    turned = rotate_reference(x[:, :Hq + H], positions, axis, freq.cpu().numpy(), interleaved)
    want = rounded(turned[:, :Hq], dtype)
    for r in range(rows):
        if r in skip:
            assert torch.equal(got[r].cpu().float(), torch.from_numpy(x[r, :Hq]) if in_place else torch.full((Hq, D), 7.0))
        else:
            assert torch.equal(got[r].cpu(), want[r]), f"queries of row {r}"
    if fused and in_place:                 # nothing else of the projection output changes
        assert torch.equal(wide[:, Hq:].float().cpu(), torch.from_numpy(x[:, Hq:]))
    want, there = cache_image(turned[:, Hq:], x[:, Hq + H:], slots, pages, P, H, D)
    raw = cache.t.view(*want.shape).cpu().numpy()
    assert np.array_equal(raw[there], want[there])
    assert (raw[~there] == 0x3C).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 1), (8, 2), (5, 5), (12, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_layouts(D, Hq, H, interleaved):
    run(7, Hq, H, D, D, interleaved=interleaved, fused=Hq == 8)


@pytest.mark.parametrize("D,rot", [(64, 16), (64, 32), (64, 48), (128, 16), (128, 80), (128, 96), (128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_partial_rotation(D, rot, interleaved):
    run(5, 3, 2, D, rot, interleaved=interleaved, dtype=BF16)


@pytest.mark.parametrize("axes", [1, 2, 3, 4, 16])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_axes_and_types(axes, dtype):
    run(20, 4, 2, 128, 128, P=32, axes=axes, dtype=dtype, fused=axes == 3)
    run(9, 4, 2, 64, 64, axes=axes, dtype=dtype, interleaved=True)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 300])
def test_rows(rows):
    run(rows, 2, 1, 128, 128, fused=True)
    run(rows, 4, 1, 64, 32)


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 29, 2 ** 31 - 1])
def test_far_positions(far):
    run(40, 2, 1, 128, 128, axes=2, far=far, seed=3)


def test_in_place_and_skipped_rows():
    run(19, 4, 2, 128, 128, in_place=True, fused=True, skip=(0, 7, 18))
    run(19, 4, 2, 64, 48, in_place=True, skip=(3,))
    run(5, 4, 2, 128, 64, skip=(0, 1, 2, 3, 4))


def test_largest_values():
    """Turned queries beyond binary16's range become its largest values."""
    run(6, 2, 2, 128, 128, dtype=F16, scale=20000.0)
    run(6, 2, 2, 64, 64, dtype=BF16, scale=2.0 ** 100)


def test_more_vectors_than_a_workgroup_takes():
    """Sizes at which a row's vectors are split over several workgroups in different ways."""
    run(700, 9, 1, 64, 64)
    run(2500, 2, 1, 128, 128, P=64)


def test_position_zero_is_the_cache_write_alone():
    K, V = vectors((40, 2, 64), 1, F16).cuda(), vectors((40, 2, 64), 2, F16).cuda()
    K[3], V[5] = 0, 0
    a, b = w4a8.new_kv_cache(3, 16, 2, 64), w4a8.new_kv_cache(3, 16, 2, 64)
    ws = w4a8.new_kv_workspace(1, 1, 2, 2, 64)
    a.zero_(), b.zero_()
    table, lens = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3), torch.tensor([40], dtype=torch.int32, device="cuda")
    w4a8.kv_append(K, V, a, table, lens, ws, cu_rows=torch.tensor([0, 40], dtype=torch.int32, device="cuda"))
    Q = w4a8.rope_kv_append(K, K, V, torch.zeros(40, dtype=torch.int32, device="cuda"), frequencies(64), b, torch.arange(40, device="cuda"), ws)
    assert torch.equal(a, b) and torch.equal(Q, K)


def test_bad_slots_and_axes_are_reported():
    ws = guarded_workspace(256)
    cache = Guarded((3, w4a8.kv_page_bytes(16, 1, 64)), torch.uint8)
    cache.t.fill_(0x3C)
    x = vectors((4, 1, 64), 1, F16).cuda()
    pos, freq = torch.arange(4, dtype=torch.int32, device="cuda"), frequencies(64)
    w4a8.rope_kv_append(x, x, x, pos, freq, cache.t, torch.tensor([48, 2 ** 40, 2 ** 62, -1], device="cuda"), ws.t)
    assert w4a8.poll_status(ws.t) == 9
    cache.check("cache")
    assert bool((cache.t == 0x3C).all())
    axis = torch.zeros(32, dtype=torch.int32, device="cuda")
    axis[5], axis[31] = -1, 3
    two = torch.stack([pos, pos + 9])
    got = w4a8.rope_kv_append(x, x, x, two, freq, cache.t, torch.arange(4, device="cuda"), ws.t, pair_axis=axis)
    assert w4a8.poll_status(ws.t) == 9
    assert torch.equal(got, w4a8.rope_kv_append(x, x, x, pos, freq, cache.t, torch.arange(4, device="cuda"), ws.t))


def test_refusals_in_python():
    ws, cache = guarded_workspace(256).t, w4a8.new_kv_cache(3, 16, 2, 64)
    Q, K = vectors((4, 4, 64), 1, F16).cuda(), vectors((4, 2, 64), 1, F16).cuda()
    pos, freq, slots = torch.arange(4, dtype=torch.int32, device="cuda"), frequencies(64), torch.arange(4, device="cuda")
    good = dict(Q=Q, K=K, V=K, positions=pos, inv_freq=freq, cache=cache, slots=slots, workspace=ws)
    w4a8.rope_kv_append(**good)
    for kw in (dict(K=K.bfloat16()), dict(slots=slots.int()), dict(positions=pos.long()), dict(inv_freq=freq.double()), dict(Q=Q.float()), dict(cache=cache.int()),
               dict(Q=Q.transpose(1, 2)), dict(out=Q.bfloat16()), dict(pair_axis=freq), dict(V=None), dict(workspace=ws.cpu())):
        with pytest.raises(TypeError):
            w4a8.rope_kv_append(**{**good, **kw})
    for kw in (dict(V=K[:, :1]), dict(slots=slots[:3]), dict(positions=pos[:3]), dict(K=K[:3]), dict(pair_axis=pos), dict(out=Q[:3]),
               dict(cache=w4a8.new_kv_cache(3, 16, 3, 64)), dict(inv_freq=freq.view(2, 16)), dict(positions=pos.view(1, 1, 4))):
        with pytest.raises(ValueError):
            w4a8.rope_kv_append(**{**good, **kw})
    for kw in (dict(inv_freq=frequencies(24)), dict(inv_freq=frequencies(80)), dict(positions=pos.repeat(17, 1)), dict(workspace=ws[:128])):
        with pytest.raises(w4a8.W4A8Error):
            w4a8.rope_kv_append(**{**good, **kw})
