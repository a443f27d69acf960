"""Sizes that 64 bits do not hold, refused before anything is launched."""
import ctypes

import paper_2011_09398_b200 as lce
from test_kv_abi import UNSUPPORTED, FAKE, attend, attention_desc, lib  # noqa: F401


def test_attention_of_more_rows_than_there_can_be(lib):  # noqa: F811
    for tokens in (1 << 31, 1 << 62, (1 << 63) - 1, (1 << 62) + 2):  # the second and the last times 4 heads are 0 and 8 in 64 bits
        d = attention_desc(tokens=tokens)
        assert attend(lib, d, starts=FAKE) == UNSUPPORTED, tokens
        assert lib.lce_kv_attention_workspace_bytes(ctypes.byref(d)) == 0, tokens
    assert lce.lce_kv_attention_workspace_bytes(lce.make_kv_desc(8, 16, 2, 64), 2, 100, 4, 3) > 0
