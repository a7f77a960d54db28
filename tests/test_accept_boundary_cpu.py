"""Refusals of the acceptance of paths with kept lengths: no device needed."""
from test_serving_boundary_cpu import GOOD, P, accept_args, w4a8, with_changes  # noqa: F401

base = dict(zip(("cache", "pages", "P", "H", "D", "table", "mp", "lens", "cu", "batch", "rows", "acc", "most", "n", "out", "ws", "wsb", "st"), accept_args()))
ex_args = with_changes({k: v for name, value in base.items() for k, v in ((("kept", P(GOOD)), (name, value)) if name == "out" else ((name, value),))})


def test_refusals(w4a8):  # noqa: F811
    f = w4a8.lib.w4a8_kv_accept_ex
    for k in ("cache", "table", "lens", "acc", "n", "ws"):
        assert f(*ex_args(**{k: None})) == 1, k
    for kw in (dict(most=0), dict(pages=0), dict(P=20), dict(H=0), dict(D=80), dict(mp=0), dict(batch=0), dict(rows=0), dict(cu=None), dict(out=P(GOOD))):
        assert f(*ex_args(**kw)) == 2, kw
    for kw in (dict(cache=P(GOOD + 8)), dict(kept=P(GOOD + 2)), dict(out=P(GOOD + 2)), dict(n=P(GOOD + 1)), dict(ws=P(GOOD + 128))):
        assert f(*ex_args(**kw)) == 3, kw
    assert f(*ex_args(wsb=255)) == 4
