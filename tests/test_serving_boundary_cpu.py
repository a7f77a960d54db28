"""Refusals of the serving calls around the cache: no device needed."""
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


def with_changes(base):
    def args(**kw):
        a = dict(base)
        assert set(kw) <= set(a)
        a.update(kw)
        return list(a.values())
    return args


plan_args = with_changes(dict(held=P(GOOD), lens=P(GOOD), add=P(GOOD), batch=3, table=P(GOOD), mp=4, P=64, free=P(GOOD), pages=9, count=P(GOOD), left=P(GOOD),
                              out=P(GOOD + 64), cu=P(GOOD), pos=P(GOOD), slots=P(GOOD), rows=7, ws=P(GOOD), wsb=512, st=None))


def test_plan_refusals(w4a8):
    f = w4a8.lib.w4a8_kv_plan
    for k in ("lens", "add", "table", "free", "count", "left", "out", "cu", "ws"):
        assert f(*plan_args(**{k: None})) == 1, k
    for kw in (dict(batch=0), dict(batch=8193), dict(mp=0), dict(mp=1 << 25), dict(P=8), dict(P=48), dict(P=2048), dict(pages=0), dict(rows=0), dict(rows=-1),
               dict(out=P(GOOD))):
        assert f(*plan_args(**kw)) == 2, kw
    for k in ("held", "lens", "add", "table", "free", "count", "left", "out", "cu", "pos"):
        assert f(*plan_args(**{k: P(GOOD + 2)})) == 3, k
    for kw in (dict(slots=P(GOOD + 4)), dict(ws=P(GOOD + 128))):
        assert f(*plan_args(**kw)) == 3, kw
    assert f(*plan_args(wsb=511)) == 4


rope_args = with_changes(dict(Q=P(GOOD), K=P(GOOD), V=P(GOOD), dtype=0, qs=4096, ks=1024, vs=1024, pos=P(GOOD), axes=3, axis=P(GOOD), freq=P(GOOD), rot=128, inter=0,
                              out=P(GOOD + 16), os=4096, cache=P(GOOD), pages=4, P=64, H=8, D=128, slots=P(GOOD), rows=5, Hq=32, ws=P(GOOD), wsb=256, st=None))


def test_rope_refusals(w4a8):
    f = w4a8.lib.w4a8_rope_kv_append
    for k in ("Q", "K", "V", "pos", "freq", "out", "cache", "slots", "ws"):
        assert f(*rope_args(**{k: None})) == 1, k
    for kw in (dict(dtype=2), dict(dtype=-1), dict(qs=4088), dict(qs=4100), dict(ks=1016), dict(vs=1028), dict(os=4088), dict(os=4100), dict(axes=0), dict(axes=17),
               dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(D=64), dict(D=96), dict(P=24), dict(H=0), dict(Hq=0), dict(Hq=65536), dict(pages=0),
               dict(rows=0), dict(rows=1 << 27), dict(out=P(GOOD), os=8192)):
        assert f(*rope_args(**kw)) == 2, kw
    for kw in (dict(Q=P(GOOD + 8)), dict(K=P(GOOD + 2)), dict(V=P(GOOD + 8)), dict(out=P(GOOD + 8)), dict(cache=P(GOOD + 8)), dict(pos=P(GOOD + 2)),
               dict(axis=P(GOOD + 1)), dict(freq=P(GOOD + 2)), dict(slots=P(GOOD + 4)), dict(ws=P(GOOD + 128))):
        assert f(*rope_args(**kw)) == 3, kw
    assert f(*rope_args(wsb=255)) == 4


attn = dict(Q=P(GOOD), qt=0, qs=4096, cache=P(GOOD), pages=4, P=64, H=8, D=128, table=P(GOOD), mp=2, lens=P(GOOD), cu=P(GOOD), batch=2, rows=5, Hq=32, scale=0.1)
end = dict(O=P(GOOD), ot=0, lse=None, ws=P(GOOD), wsb=1 << 30, st=None)
sinks_args = with_changes(dict(**attn, causal=1, window=9, sinks=4, **end))
tree_args = with_changes(dict(**attn, mask=P(GOOD), words=2, window=9, sinks=4, **end))


@pytest.mark.parametrize("which", ["sinks", "tree"])
def test_attention_refusals(w4a8, which):
    f, args = (w4a8.lib.w4a8_kv_attention_sinks, sinks_args) if which == "sinks" else (w4a8.lib.w4a8_kv_attention_tree, tree_args)
    for k in ("Q", "O", "cache", "table", "lens", "ws"):
        assert f(*args(**{k: None})) == 1, k
    for kw in (dict(qt=2), dict(ot=2), dict(qs=4088), dict(qs=4100), dict(Hq=30), dict(Hq=4), dict(scale=0.0), dict(scale=float("nan")), dict(window=-1),
               dict(sinks=-1), dict(rows=0), dict(batch=0), dict(cu=None), dict(D=96), dict(P=20), dict(mp=1 << 25)):
        assert f(*args(**kw)) == 2, kw
    for kw in (dict(Q=P(GOOD + 8)), dict(O=P(GOOD + 2)), dict(lse=P(GOOD + 2)), dict(cache=P(GOOD + 8)), dict(ws=P(GOOD + 128))):
        assert f(*args(**kw)) == 3, kw
    assert f(*args(wsb=w4a8.kv_attention_workspace_bytes(5, 2, 32, 8, 128) - 1)) == 4
    if which == "tree":
        assert f(*args(mask=None)) == 1
        for words in (0, -1, (1 << 20) + 1):
            assert f(*args(words=words)) == 2
        assert f(*args(mask=P(GOOD + 2))) == 3


accept_args = with_changes(dict(cache=P(GOOD), pages=4, P=64, H=8, D=128, table=P(GOOD), mp=2, lens=P(GOOD), cu=P(GOOD), batch=2, rows=5, acc=P(GOOD), most=3,
                                n=P(GOOD), out=None, ws=P(GOOD), wsb=256, st=None))


def test_accept_refusals(w4a8):
    f = w4a8.lib.w4a8_kv_accept
    for k in ("cache", "table", "lens", "acc", "n", "ws"):
        assert f(*accept_args(**{k: None})) == 1, k
    for kw in (dict(most=0), dict(pages=0), dict(P=20), dict(H=0), dict(D=80), dict(mp=0), dict(batch=0), dict(rows=0), dict(cu=None), dict(out=P(GOOD))):
        assert f(*accept_args(**kw)) == 2, kw
    for kw in (dict(cache=P(GOOD + 8)), dict(table=P(GOOD + 2)), dict(acc=P(GOOD + 2)), dict(n=P(GOOD + 1)), dict(out=P(GOOD + 2)), dict(ws=P(GOOD + 128))):
        assert f(*accept_args(**kw)) == 3, kw
    assert f(*accept_args(wsb=255)) == 4


def test_python_calls_refuse_before_they_touch_a_device(w4a8):
    import torch
    w = w4a8
    half, page = torch.zeros(1, 4, 64, dtype=torch.float16), torch.zeros(1, 16 * 72, dtype=torch.uint8)
    one, freq, slot = torch.ones(1, 1, dtype=torch.int32), torch.ones(32), torch.zeros(1, dtype=torch.int64)
    for call in (lambda: w.kv_plan(one[0], one[0], one[0], one, one[0], one[0], 16, 1, page), lambda: w.kv_plan(None, 3, one[0], one, one[0], one[0], 16, 1, page),
                 lambda: w.rope_kv_append(half, half, half, one[0], freq, page, slot, page), lambda: w.rope_kv_append(half, None, half, one[0], freq, page, slot, page),
                 lambda: w.kv_attention_sinks(half, page, one, one[0], 4, page, 8, 4), lambda: w.kv_attention_sinks(half, page, one, one[0], 4, page, "8", 4),
                 lambda: w.kv_attention_tree(half, page, one, one[0], 4, page, one), lambda: w.kv_attention_tree(half, page, one, one[0], 4, page, None),
                 lambda: w.kv_accept(page, one, one[0], one, one[0], 1, 64, page), lambda: w.kv_accept(page, one, one[0], one, one[0], None, 64, page)):
        with pytest.raises(TypeError):
            call()
