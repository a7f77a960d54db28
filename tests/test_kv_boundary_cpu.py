"""Refusals and size queries of the cache, attention and residual-norm calls: no device needed."""
import ctypes

import pytest

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def w4a8():
    entry.build()
    import paper_2311_05161_b200 as mod
    return mod


P = ctypes.c_void_p
GOOD = 0x10000          # never dereferenced: validation fails first


def test_page_and_workspace_sizes(w4a8):
    assert w4a8.kv_page_bytes(64, 8, 128) == 8 * 64 * 136
    assert w4a8.kv_page_bytes(16, 1, 64) == 16 * 72
    for bad in ((0, 8, 128), (8, 8, 128), (48, 8, 128), (2048, 8, 128), (64, 0, 128), (64, 8, 96), (64, -1, 64), (-64, 8, 128)):
        assert w4a8.kv_page_bytes(*bad) == 0
    assert w4a8.kv_attention_workspace_bytes(1, 1, 8, 8, 128) >= 256
    for bad in ((0, 1, 8, 8, 128), (1, 0, 8, 8, 128), (1, 1, 8, 3, 128), (1, 1, 4, 8, 128), (1, 1, 8, 8, 80), (1 << 20, 1, 65535, 1, 64)):
        assert w4a8.kv_attention_workspace_bytes(*bad) == 0


def append_args(**kw):
    a = dict(K=P(GOOD), V=P(GOOD), dtype=0, ks=1024, vs=1024, cache=P(GOOD), pages=4, P=64, H=8, D=128, table=P(GOOD), mp=2,
             lens=P(GOOD), cu=P(GOOD), batch=2, rows=5, ws=P(GOOD), wsb=1 << 20, st=None)
    a.update(kw)
    return list(a.values())


def test_append_refusals(w4a8):
    f = w4a8.lib.w4a8_kv_append
    for k in ("K", "V", "cache", "table", "lens", "ws"):
        assert f(*append_args(**{k: None})) == 1, k
    for kw in (dict(dtype=2), dict(dtype=-1), dict(ks=1016), dict(ks=1028), dict(vs=0), dict(vs=-1024), dict(pages=0), dict(P=24),
               dict(H=0), dict(D=32), dict(mp=0), dict(batch=0), dict(rows=0), dict(cu=None), dict(mp=1 << 25),
               dict(rows=(1 << 31) - 1)):
        assert f(*append_args(**kw)) == 2, kw
    for kw in (dict(K=P(GOOD + 8)), dict(V=P(GOOD + 2)), dict(cache=P(GOOD + 8)), dict(table=P(GOOD + 2)), dict(lens=P(GOOD + 1)),
               dict(cu=P(GOOD + 2)), dict(ws=P(GOOD + 128))):
        assert f(*append_args(**kw)) == 3, kw
    assert f(*append_args(wsb=255)) == 4


def read_args(**kw):
    a = dict(cache=P(GOOD), pages=4, P=64, H=8, D=128, table=P(GOOD), mp=2, lens=P(GOOD), cu=P(GOOD), batch=2, rows=5, K=P(GOOD),
             V=P(GOOD), dtype=0, ws=P(GOOD), wsb=1 << 20, st=None)
    a.update(kw)
    return list(a.values())


def test_read_refusals(w4a8):
    f = w4a8.lib.w4a8_kv_read
    for k in ("K", "V", "cache", "table", "lens", "ws"):
        assert f(*read_args(**{k: None})) == 1, k
    for kw in (dict(dtype=2), dict(pages=-1), dict(P=0), dict(H=-1), dict(D=256), dict(mp=0), dict(batch=0), dict(rows=0), dict(cu=None)):
        assert f(*read_args(**kw)) == 2, kw
    for kw in (dict(K=P(GOOD + 8)), dict(V=P(GOOD + 2)), dict(cache=P(GOOD + 4)), dict(ws=P(GOOD + 128))):
        assert f(*read_args(**kw)) == 3, kw
    assert f(*read_args(wsb=0)) == 4


def attn_args(**kw):
    a = dict(Q=P(GOOD), qt=0, qs=4096, cache=P(GOOD), pages=4, P=64, H=8, D=128, table=P(GOOD), mp=2, lens=P(GOOD), cu=P(GOOD),
             batch=2, rows=5, Hq=32, scale=0.1, causal=1, window=0, O=P(GOOD), ot=0, lse=None, ws=P(GOOD), wsb=1 << 30, st=None)
    a.update(kw)
    return list(a.values())


def test_attention_refusals(w4a8):
    f = w4a8.lib.w4a8_kv_attention
    for k in ("Q", "O", "cache", "table", "lens", "ws"):
        assert f(*attn_args(**{k: None})) == 1, k
    for kw in (dict(qt=2), dict(ot=2), dict(qs=4088), dict(qs=4100), dict(Hq=30), dict(Hq=0), dict(Hq=4), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(rows=0), dict(batch=0), dict(cu=None),
               dict(D=96), dict(P=20)):
        assert f(*attn_args(**kw)) == 2, kw
    for kw in (dict(Q=P(GOOD + 8)), dict(O=P(GOOD + 2)), dict(lse=P(GOOD + 2)), dict(cache=P(GOOD + 8)), dict(ws=P(GOOD + 128))):
        assert f(*attn_args(**kw)) == 3, kw
    need = w4a8.kv_attention_workspace_bytes(5, 2, 32, 8, 128)
    assert f(*attn_args(wsb=need - 1)) == 4


def test_add_norm_refusals(w4a8):
    def args(**kw):
        a = dict(X=P(GOOD), xt=0, res=P(GOOD), rt=2, out=P(GOOD), w=P(GOOD), b=None, kind=0, eps=1e-5, M=4, K=256, Xq=P(GOOD), tok=P(GOOD),
                 st=None)
        a.update(kw)
        return list(a.values())

    f = w4a8.lib.w4a8_add_norm_quantize_act
    for k in ("X", "res", "out", "w", "Xq", "tok"):
        assert f(*args(**{k: None})) == 1, k
    for kw in (dict(xt=2), dict(xt=-1), dict(rt=3), dict(kind=2), dict(eps=0.0), dict(M=0), dict(K=200), dict(K=16512), dict(K=0)):
        assert f(*args(**kw)) == 2, kw
    for k in ("X", "res", "out", "w", "b", "Xq"):
        assert f(*args(**{k: P(GOOD + 8)})) == 3, k
    assert f(*args(tok=P(GOOD + 2))) == 3


def test_python_calls_refuse_before_they_touch_a_device(w4a8):
    """Tensors of the host, wrong types and numbers raise in the marshalling; nothing is launched."""
    import torch
    w = w4a8
    half, page = torch.zeros(1, 4, 64, dtype=torch.float16), torch.zeros(1, 16 * 72, dtype=torch.uint8)
    one = torch.ones(1, 1, dtype=torch.int32)
    for call in (lambda: w.kv_attention(half, page, one, one[0], 1, page), lambda: w.kv_append(half, half, page, one, one[0], page),
                 lambda: w.kv_read(page, one, one[0], 1, 1, 64, page), lambda: w.kv_attention(None, page, one, one[0], 1, page),
                 lambda: w.kv_attention(half, page, one, one[0], "1", page), lambda: w.add_norm_quantize_act(half, half, half),
                 lambda: w.add_norm_quantize_act(1, 2, 3)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        w.kv_read(page, one, one[0], 1, 2 ** 40, 64, page)
