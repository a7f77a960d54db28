"""Page tables whose last positions lie at the end of 31 bits: the kernels count in groups of up to 64 tokens and up to
64 positions past the last, which have to stay in range."""
import ctypes

import pytest

import __graft_entry__ as entry

P = ctypes.c_void_p
GOOD = 0x10000          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    entry.build()
    import paper_2311_05161_b200 as mod
    return mod.lib


def calls(lib, page, most, table=GOOD):
    common = (4, page, 8, 128)
    return (lib.w4a8_kv_append(P(GOOD), P(GOOD), 0, 1024, 1024, P(GOOD), *common, P(table), most, P(GOOD), P(GOOD), 2, 5, P(GOOD), 1 << 20, None),
            lib.w4a8_kv_read(P(GOOD), *common, P(table), most, P(GOOD), P(GOOD), 2, 5, P(GOOD), P(GOOD), 0, P(GOOD), 1 << 20, None),
            lib.w4a8_kv_attention(P(GOOD), 0, 4096, P(GOOD), *common, P(table), most, P(GOOD), P(GOOD), 2, 5, 32, 0.1, 1, 0, P(GOOD), 0, None,
                                  P(GOOD), 1 << 30, None))


@pytest.mark.parametrize("page", [16, 64, 1024])
def test_the_last_positions_are_refused(lib, page):
    for most in ((1 << 31) // page, ((1 << 31) - 1024) // page + 1):
        assert calls(lib, page, most) == (2, 2, 2), most
    # as many as are allowed: the next check refuses (a table that is not aligned)
    assert calls(lib, page, ((1 << 31) - 1024) // page, GOOD + 2) == (3, 3, 3)
