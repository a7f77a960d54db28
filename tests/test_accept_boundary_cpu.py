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


def test_lengths_over_an_input(w4a8):  # noqa: F811
    """kv_lens_out shares an element or more with something that the call reads."""
    f, out = w4a8.lib.w4a8_kv_accept_ex, 0x80000
    apart = dict(table=P(GOOD), lens=P(GOOD + 0x1000), cu=P(GOOD + 0x2000), acc=P(GOOD + 0x3000), n=P(GOOD + 0x4000), kept=P(GOOD + 0x5000), out=P(out))
    sizes = dict(table=2 * 2, lens=2, cu=3, acc=2 * 3, n=2, kept=2)             # batch 2, 2 pages, 3 places
    for k, size in sizes.items():
        for shift in (1 - size, -1, 0, 1):
            if k == "kept" and shift == 0:
                continue
            assert f(*ex_args(**{**apart, k: P(out + 4 * shift)})) == 2, (k, shift)
    g = w4a8.lib.w4a8_kv_accept
    for k in ("lens", "acc", "n", "cu", "table"):
        assert g(*accept_args(**{**{x: v for x, v in apart.items() if x != "kept"}, k: P(out)})) == 2, k
