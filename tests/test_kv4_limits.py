"""Limits of the 4-bit attention at their edges, without a GPU."""
import ctypes

import paper_2605_22850_amd as oc


def test_query_heads_of_a_decode():
    """Row tiles of 32 query heads are a grid's second dimension, of at most 65535."""
    for nq, ok in ((65535 * 32, True), (65535 * 32 + 1, False), (1 << 22, False)):
        lay = oc.Layout(1, nq, 1, 64, 16, 16, 8).c()
        assert (oc.lib().oc_kv4_decode_workspace_bytes(ctypes.byref(lay), 1, 64) > 0) == ok
        if not ok:
            assert b"65535 * 32 query heads" in oc.lib().oc_last_error()
